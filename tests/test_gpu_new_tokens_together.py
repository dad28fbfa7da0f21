"""New tokens and the 4-bit cache where calls meet: pools and rows beyond 32-bit offsets, two contexts on two streams, recorded graphs that are replayed
between eager calls.  What a call gives here has to be, bit for bit, what the same call gives alone, on a small pool or eagerly: those are
held against the oracle elsewhere."""
import numpy as np
import pytest
import torch

from paper_2604_12056_amd import binding as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
G, D = 16, 128


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def context(Hq, Hkv, B, batch, max_pages):
    return L.losa_create(L.make_config(max_batch=batch, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, hidden_size=Hq * D, page_size=G, block_size=B,
                                       max_pages_per_seq=max_pages, max_topk_pages=max_pages), DEV)


def pools(n, Hkv, clear=True):
    make = torch.zeros if clear else torch.empty
    u8 = dict(dtype=torch.uint8, device=DEV)
    return (make((n, Hkv, G, D // 2), **u8), make((n, Hkv, G // 4, 16, D // 32, 4), **u8), make((n, Hkv, 2, G, D // 32), **u8),
            make((n, Hkv, 2, D), dtype=torch.bfloat16, device=DEV))


def rows(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)


def table(n):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    return L.Rotation(torch.cat((a.cos(), a.sin()), 1).float().to(DEV))


def test_pages_beyond_32_bit_offsets():
    """The same calls on a pool of 4.3 GB whose used pages lie at its two ends, and on a small one."""
    far, n, m = (1 << 22) + 8, 40, 600
    ids = {n: list(range(n)), far: [far - 1 - i if i % 2 else i for i in range(n)]}
    k, v, q = rows(1, m, 1, D), rows(2, m, 1, D), rows(3, 4, 2, D)
    ctx, rot, got = context(2, 1, 4, 1, n), table(m), {}
    for size in (n, far):
        pool = pools(size, 1, clear=size == n)
        table_of = (i32([0, n]), i32(ids[size]), i32([m]))
        kv = L.PackedKV(*pool, *table_of)
        L.losa_append_packed(ctx, kv, k, v, i32([0, m]), rot)
        o, lse, ko, vo = torch.zeros((4, 2, D), device=DEV), torch.zeros((4, 2), device=DEV), torch.zeros_like(k), torch.zeros_like(v)
        L.losa_sparse_attn_packed(ctx, kv, q, None, None, None, None, 0, o, lse)
        L.losa_read_packed(ctx, kv, i32([0, m]), ko, vo)
        used = (m + G - 1) // G
        got[size] = [o, lse, ko, vo, pool[3][table_of[1][:used].long()]]
        del pool, kv
        kp, vp = (torch.zeros((1, 1, 1), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        if size == far:      # a cache in bfloat16, 4.3 GB each way
            far16 = (1 << 20) + 8
            kp, vp = (torch.empty((far16, 1, G, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            at = i32([far16 - 1 - i if i % 2 else i for i in range(n)])
        else:
            kp, vp = (torch.empty((n, 1, G, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            at = i32(list(range(n)))
        meta = torch.empty((kp.shape[0], 1, 2, D), dtype=torch.bfloat16, device=DEV)
        L.losa_append_kv(ctx, L.PagedKV(kp, vp.view(-1, 1, D, G), meta, i32([0, n]), at, i32([m])), k, v, i32([0, m]), rot)
        full = m // G
        got[size] += [kp[at[:full].long()], vp[at[:full].long()], meta[at[:used].long()]]
    torch.cuda.synchronize()
    assert float(got[n][0].abs().max()) > 0
    for x, y in zip(got[n], got[far]):
        assert torch.equal(x, y)
    ctx.close()


def test_rows_beyond_32_bit_offsets():
    """Rows of new tokens, and of rotated ones, 2 GiB apart."""
    apart = 1 << 30                       # elements
    big = torch.empty(3 * apart + 2 * D, dtype=torch.bfloat16, device=DEV)
    k, v = big.as_strided((4, 1, D), (apart, D, 1)), big.as_strided((4, 1, D), (apart, D, 1), D)
    k.copy_(rows(4, 4, 1, D)), v.copy_(rows(5, 4, 1, D))
    ctx, rot, got = context(1, 1, 4, 1, 1), table(16), []
    for a, b in ((k, v), (k.contiguous(), v.contiguous())):
        kv = L.PackedKV(*pools(1, 1), i32([0, 1]), i32([0]), i32([4]))
        L.losa_append_packed(ctx, kv, a, b, i32([0, 4]), rot)
        L.losa_rotate(ctx, rot, i32([3, 2, 1, 0]), a, a)   # in place
        got.append([kv.k_codes, kv.v_codes, kv.scales, kv.meta, a.contiguous()])
    for x, y in zip(*got):
        assert torch.equal(x, y)
    ctx.close()


def test_many_tokens_are_turned_as_few_are():
    n = 9001
    ctx, rot, pos = context(3, 1, 4, 1, 1), table(512), torch.arange(n, dtype=torch.int32, device=DEV) % 512
    q, k = rows(6, n, 3, D), rows(7, n, 1, D)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    L.losa_rotate(ctx, rot, pos, q, qo, k, ko)
    for a in range(0, n, 1000):
        at = slice(a, min(a + 1000, n))
        qs, ks = torch.zeros_like(q[at]), torch.zeros_like(k[at])
        L.losa_rotate(ctx, rot, pos[at], q[at], qs, k[at], ks)
        assert torch.equal(qo[at], qs) and torch.equal(ko[at], ks)
    ctx.close()


class Cache:
    """A 4-bit cache, its context and what goes through them."""

    def __init__(self, seed, Hq=4, Hkv=2, B=8, lens=(70, 33, 200)):
        self.B, self.lens0 = B, list(lens)
        most = [(x + 3 * B + G - 1) // G for x in lens]
        self.ctx = context(Hq, Hkv, B, len(lens), max(most))
        n = sum(most)
        ids = np.random.default_rng(seed).permutation(n).tolist()
        self.kv = L.PackedKV(*pools(n, Hkv), i32(np.concatenate(([0], np.cumsum(most))).tolist()), i32(ids), i32(self.lens0))
        self.rot = table(max(lens) + 3 * B)
        self.prompt = rows(seed, sum(lens), Hkv, D), rows(seed + 1, sum(lens), Hkv, D)
        self.prompt_ptr, self.block_ptr = i32(np.concatenate(([0], np.cumsum(lens))).tolist()), i32([B * i for i in range(len(lens) + 1)])
        self.q, self.k, self.v = rows(seed + 2, len(lens) * B, Hq, D), rows(seed + 3, len(lens) * B, Hkv, D), rows(seed + 4, len(lens) * B, Hkv, D)
        self.pos = i32([x + i for x in lens for i in range(B)])
        self.qr, self.o, self.lse = torch.zeros_like(self.q), torch.zeros(self.q.shape, device=DEV), torch.zeros(self.q.shape[:2], device=DEV)
        self.ko, self.vo = torch.zeros_like(self.k), torch.zeros_like(self.v)
        torch.cuda.synchronize()

    def fill(self, stream=None):
        L.losa_append_packed(self.ctx, self.kv, *self.prompt, self.prompt_ptr, self.rot, stream=stream)

    def block(self, stream=None):
        """Tokens appended, queries turned, every query against every page, the new tokens read back.  (Twice gives the same.)"""
        L.losa_append_packed(self.ctx, self.kv, self.k, self.v, self.block_ptr, self.rot, max_new_tokens=self.B, stream=stream)
        L.losa_rotate(self.ctx, self.rot, self.pos, self.q, self.qr, stream=stream)
        L.losa_sparse_attn_packed(self.ctx, self.kv, self.qr, None, None, None, None, 0, self.o, self.lse, stream=stream)
        L.losa_read_packed(self.ctx, self.kv, self.block_ptr, self.ko, self.vo, max_tokens=self.B, stream=stream)

    def grow(self):
        self.kv.seq_lens.add_(self.B)

    def state(self):
        kv = self.kv
        return [x.clone() for x in (kv.k_codes, kv.v_codes, kv.scales, kv.meta, self.qr, self.o, self.lse, self.ko, self.vo)]


def alone(seed, blocks):
    c, out = Cache(seed), []
    c.fill()
    for _ in range(blocks):
        c.grow()
        c.block()
        out.append(c.state())
    torch.cuda.synchronize()
    c.ctx.close()
    return out


def test_two_contexts_on_two_streams():
    want = [alone(seed, 2) for seed in (10, 20)]
    caches, streams = [Cache(10), Cache(20)], [torch.cuda.Stream() for _ in range(2)]
    for c, s in zip(caches, streams):
        c.fill(stream=s.cuda_stream)
    got = [[], []]
    for _ in range(2):
        for c, s in zip(caches, streams):      # the handle given, and the current stream
            with torch.cuda.stream(s):
                c.grow()
            c.block(stream=s.cuda_stream)
        for c, s, x in zip(caches, streams, got):
            with torch.cuda.stream(s):
                x.append(c.state())
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):
            assert all(torch.equal(i, j) for i, j in zip(x, y))
    for c in caches:
        c.ctx.close()


def test_recorded_and_eager_calls_in_turn():
    """Two graphs of one context, which share its workspace, and eager calls between their replays."""
    want = alone(30, 3)
    c = Cache(30)
    c.fill()
    graphs = []
    side = torch.cuda.Stream()
    for f in (c.grow, c.block):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            f()
    other = Cache(40, lens=(5, 300))
    for i in range(3):
        graphs[0].replay()
        graphs[1].replay()
        if i == 1:                              # eagerly, over what the replay wrote: the same again
            torch.cuda.synchronize()
            c.block()
        other.fill()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want[i], c.state())), i
    c.ctx.close()
    other.ctx.close()


@pytest.mark.parametrize("shared", [False, True])
def test_stages_one_by_one_over_a_packed_cache(shared):
    """Active set, pages by the packed keys' bounds, attention: call by call what losa_step_packed does in one (or with one list per head).

    Tolerance: both results are within 4 ds + (n + 70) u of the exact ones, in units of the largest value, and lse within ds + (n + 70) u + 4 u |lse|
    (u = 2^-24, ds = (d + 4) u S + 4 u; derived in test_gpu_packed_attn.py).  n <= 224 tokens; S <= 2 |q| |k| / sqrt(d) + 16 <= 80, as rows of 128 normal
    numbers are shorter than 16 and rounding to 4 bits adds a third at most; |lse| < 32."""
    c = Cache(50)
    c.fill()
    B, batch, Hkv, most = c.B, 3, 2, 3
    h_prev, step = rows(51, batch * B, c.ctx.q_heads * D), rows(52, batch * B, c.ctx.q_heads * D)
    h_cur = h_prev + step * (torch.arange(batch * B, device=DEV) % 3 == 0)[:, None]
    assert c.q.float().norm(dim=2).max() < 16 and torch.cat((c.prompt[0], c.k)).float().norm(dim=2).max() < 16
    o, lse = torch.zeros_like(c.o), torch.zeros_like(c.lse)
    mask, count = torch.zeros(batch * B, dtype=torch.uint8, device=DEV), torch.zeros((batch, Hkv), dtype=torch.int32, device=DEV)
    L.losa_step_packed(c.ctx, c.kv, 1, h_cur, h_prev, c.q, L.LOSA_SEL_TOPK, 3.0, most, o, lse, mask, count)
    torch.cuda.synchronize()
    cap = max((n + 3 * B + G - 1) // G for n in c.lens0)
    delta, mask2 = torch.zeros(batch * B, device=DEV), torch.zeros_like(mask)
    idx, n = torch.full((batch, B), -1, dtype=torch.int32, device=DEV), torch.zeros(batch, dtype=torch.int32, device=DEV)
    L.losa_select_active(c.ctx, h_cur, h_prev, L.LOSA_SEL_TOPK, 3.0, delta, mask2, idx, n)
    pages, count2 = torch.full((batch, Hkv, cap), -1, dtype=torch.int32, device=DEV), torch.zeros_like(count)
    if shared:
        L.losa_score_pages_shared(c.ctx, c.kv.for_scoring(), c.q, idx, n, most, pages, count2, cap)
    else:
        L.losa_score_pages(c.ctx, c.kv.for_scoring(), c.q, idx, n, most, None, pages, count2, cap)
    L.losa_sparse_attn_packed(c.ctx, c.kv, c.q, idx, n, pages, count2, cap, c.o, c.lse)
    torch.cuda.synchronize()
    assert torch.equal(mask, mask2) and int(mask.sum()) == 3 * batch
    held = [(x + G - 1) // G for x in c.lens0]
    if shared:
        assert count2.tolist() == [[min(most, m)] * Hkv for m in held]
        assert bool(c.lse[mask.bool()].isfinite().all())
        return c.ctx.close()
    assert torch.equal(count, count2)
    biggest = torch.cat((c.prompt[1], c.v)).float().abs().max() * 4 / 3
    u, ds = 2.0 ** -24, (132 * 80 + 4) * 2.0 ** -24
    assert float((o - c.o).abs().max()) <= 2 * (4 * ds + 294 * u) * float(biggest)
    assert float((lse - c.lse)[mask.bool()].abs().max()) <= 2 * (ds + 294 * u + 4 * u * 32)
    assert not o[~mask.bool()].any() and not c.o[~mask.bool()].any()
    c.ctx.close()
