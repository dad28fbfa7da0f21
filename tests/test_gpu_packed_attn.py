"""Attention over a 4-bit cache (losa_sparse_attn_packed, losa_step_packed) against the CPU oracle in float64 over the numbers that the
codes stand for.

Tolerance, per (row, KV head), from the arithmetic.  With u = 2^-24 (half a step of float):
  score     d products summed in float, times a rounded scale, minus a reference, into an exponential of 1 ulp:
            |error| <= ds = (d + 4) u S + 4 u, S = scale * max_t sum_c |q_c k_tc| + |reference| <= 2 of those sums + 16
  o         numerators off by e^ds - 1 <= 2 ds each way, probabilities as two halves 2 u, n additions in float (n u), rescales and merge
            (64 u): |error| <= V (4 ds + (n + 70) u), V = max |v| over the head's tokens
  lse       ds + (n + 70) u + 4 u |lse|
Rows that are not active keep their bits."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from oracle import losa_oracle
from paper_2604_12056_amd import binding as L
from paper_2604_12056_amd import synth
from paper_2604_12056_amd.device_inputs import to_device, to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


class Rig:
    """A 4-bit cache of arbitrary numbers, slots behind the sequences' ends (and the spare pages) of arbitrary bytes."""

    def __init__(self, seed, Hq, Hkv, d, g, B, lens, dtype="bf16", spread=1.0, max_pages=None):
        self.rng = rng = np.random.default_rng(seed)
        self.Hq, self.Hkv, self.G, self.d, self.g, self.B, self.lens, self.dtype = Hq, Hkv, Hq // Hkv, d, g, B, lens, dtype
        batch, J = len(lens), d // 32
        pages = [(n + g - 1) // g for n in lens]
        n = sum(pages) + 3
        self.num_pages, self.pages = n, pages
        self.indptr = np.concatenate(([0], np.cumsum(pages))).astype(np.int32)
        self.indices = rng.permutation(n)[:sum(pages)].astype(np.int32)
        kc = rng.integers(0, 256, (n, Hkv, g, d // 2), dtype=np.uint8)
        vc = rng.integers(0, 256, (n, Hkv, g // 4, 16, J, 4), dtype=np.uint8)
        sc = rng.integers(0, 256, (n, Hkv, 2, g, J), dtype=np.uint8)
        for b, m in enumerate(lens):
            for p in range(pages[b]):
                fill = min(g, m - p * g)
                shape = (Hkv, 2, fill, J)
                sc[self.indices[self.indptr[b] + p], :, :, :fill] = rng.integers(int(124 - spread), int(127 + spread), shape)
        self.pool = orc.PackedPool(kc, vc, sc)
        q = rng.standard_normal((batch * B, Hq, d)).astype(np.float32) * 0.5
        self.q_s = synth.store(q, dtype)
        self.q = synth.load(self.q_s).astype(np.float64)
        self.cfg = L.make_config(max_batch=batch, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d, hidden_size=Hq * d, page_size=g, block_size=B,
                                 max_pages_per_seq=max_pages or max(max(pages), 1), max_topk_pages=max(max(pages), 1),
                                 dtype=L.LOSA_BF16 if dtype == "bf16" else L.LOSA_F32)
        self.ctx = L.losa_create(self.cfg, DEV)
        self.meta = torch.zeros((n, Hkv, 2, d), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device=DEV)
        self.upload()
        self.o0 = rng.standard_normal((batch * B, Hq, d)).astype(np.float32)
        self.l0 = rng.standard_normal((batch * B, Hq)).astype(np.float32)
        self.cache = {}

    def upload(self):
        self.kv = L.PackedKV(dev(self.pool.k_codes), dev(self.pool.v_codes), dev(self.pool.scales), self.meta, dev(self.indptr), dev(self.indices),
                             dev(np.array(self.lens, np.int32)))

    def page(self, b, p, h):
        """Keys and values of a logical page's tokens."""
        at = (b, p, h)
        if at not in self.cache:
            phys = int(self.indices[self.indptr[b] + p])
            if not 0 <= phys < self.num_pages:
                self.cache[at] = np.zeros((0, self.d)), np.zeros((0, self.d))
            else:
                kv = [self.pool.get(phys, h, r) for r in range(min(self.g, self.lens[b] - p * self.g))]
                self.cache[at] = np.stack([k for k, _ in kv]), np.stack([v for _, v in kv])
        return self.cache[at]

    def run(self, active=None, lists=None, cap=None, stream=None):
        """active: tokens of every sequence; lists[b][h]: logical pages.  Returns (o, lse) and the expectation."""
        batch = len(self.lens)
        o, l = dev(self.o0), dev(self.l0)
        idx = cnt = pages = count = None
        if active is not None:
            a = np.full((batch, self.B), -1, np.int32)
            for b, t in enumerate(active):
                a[b, :len(t)] = t
            idx, cnt = dev(a), dev(np.array([len(t) for t in active], np.int32))
        if lists is not None:
            cap = cap or max(1, max(len(x) for r in lists for x in r))
            a = np.full((batch, self.Hkv, cap), -1, np.int32)
            for b in range(batch):
                for h in range(self.Hkv):
                    a[b, h, :len(lists[b][h])] = lists[b][h][:cap]
            pages, count = dev(a), dev(np.array([[len(x) for x in r] for r in lists], np.int32))
        L.losa_sparse_attn_packed(self.ctx, self.kv, to_device(self.q_s, DEV), idx, cnt, pages, count, cap or 0, o, l, stream=stream)
        torch.cuda.synchronize()
        return o, l

    def check(self, o, l, active=None, lists=None, most_pages=1 << 30):
        o, l = o.cpu().numpy().astype(np.float64), l.cpu().numpy().astype(np.float64)
        scale = self.cfg.sm_scale or 1 / np.sqrt(self.d)
        idle = np.ones(len(o), bool)
        for b in range(len(self.lens)):
            tokens = range(self.B) if active is None else [t for t in active[b] if 0 <= t < self.B]
            at = [b * self.B + t for t in tokens]
            idle[at] = False
            if not at:
                continue
            for h in range(self.Hkv):
                listed = range(self.pages[b]) if lists is None else lists[b][h]
                kv = [self.page(b, p, h) for p in listed if 0 <= p < min(self.pages[b], most_pages)]
                k = np.concatenate([x for x, _ in kv] + [np.zeros((0, self.d))])
                v = np.concatenate([x for _, x in kv] + [np.zeros((0, self.d))])
                q = self.q[at, h * self.G:(h + 1) * self.G].reshape(-1, self.d)
                want, lse = orc.attention(q, k, v, scale)
                got = o[at, h * self.G:(h + 1) * self.G].reshape(-1, self.d)
                got_l = l[at, h * self.G:(h + 1) * self.G].reshape(-1)
                if len(k) == 0:
                    assert np.all(got == 0) and np.all(got_l == -np.inf)
                    continue
                S = 2 * scale * (np.abs(q) @ np.abs(k).T).max(1) + 16
                ds = (self.d + 4) * U * S + 4 * U
                n = len(k)
                tol = np.abs(v).max() * (4 * ds + (n + 70) * U)
                assert np.all(np.abs(got - want) <= tol[:, None]), (b, h, np.abs(got - want).max(), tol.min())
                assert np.all(np.abs(got_l - lse) <= ds + (n + 70) * U + 4 * U * np.abs(lse)), (b, h)
        rows = np.nonzero(idle)[0]
        assert np.array_equal(o[rows], self.o0[rows]) and np.array_equal(l[rows], self.l0[rows])

    def close(self):
        self.ctx.close()


LENS = (1, 0, 15, 16, 17, 33, 250)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [16, 32])
@pytest.mark.parametrize("Hq,Hkv,B", [(2, 2, 1), (7, 1, 1), (4, 2, 9), (12, 3, 12), (7, 1, 9), (4, 1, 16), (5, 1, 13), (8, 1, 29)])
def test_every_token_against_every_page(dtype, d, g, Hq, Hkv, B):
    """One to 232 query rows per KV head, sequences of no token to many, the last page part full."""
    rig = Rig(Hq * 31 + B, Hq, Hkv, d, g, B, LENS, dtype)
    rig.check(*rig.run())
    rig.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,g", [(64, 32), (128, 16), (128, 32)])
@pytest.mark.parametrize("Hq,Hkv,B", [(14, 2, 8), (28, 4, 5), (4, 1, 64), (8, 2, 1)])
def test_active_tokens_and_lists(dtype, d, g, Hq, Hkv, B):
    """Counts that only the device knows: no row to all of them; lists of no page, of one, ascending or not, with entries that are no page."""
    lens = (700, 33, 0, 401, 16)
    rig = Rig(Hq * 17 + B, Hq, Hkv, d, g, B, lens, dtype)
    rng = rig.rng
    for trial in range(3):
        active = [sorted(rng.permutation(B)[:n].tolist()) for n in rng.integers(0, B + 1, 5)]
        active[trial] = [] if trial else list(range(B))
        lists = [[sorted(rng.permutation(p)[:rng.integers(0, p + 1)].tolist()) for _ in range(Hkv)] for p in rig.pages]
        if trial == 1:
            lists[0] = [rng.permutation(rig.pages[0]).tolist() for _ in range(Hkv)]
        if trial == 2:
            lists[0][0] = [-1, 0, rig.pages[0], 2 ** 31 - 1, 3, -2 ** 31]
            lists[3][-1] = []
        rig.check(*rig.run(active, lists), active, lists)
        rig.check(*rig.run(active, None), active, None)
        rig.check(*rig.run(None, lists), None, lists)
    rig.close()


def test_token_ids_and_pages_that_do_not_exist_are_skipped():
    rig = Rig(4, 8, 2, 128, 16, 8, (90, 200), max_pages=20)
    rig.indices[2], rig.indices[int(rig.indptr[1]) + 5] = -3, rig.num_pages
    rig.upload()
    active = [[0, -5, 3, 8, 7], [2, 1]]
    rig.check(*rig.run(active), active)
    rig.kv.max_seq_pages = 4
    rig.check(*rig.run(active), active, most_pages=4)
    rig.close()


@pytest.mark.parametrize("d", [64, 128])
def test_long_lists_and_large_scores(d):
    """Many tiles a wavefront, references that move often, probabilities that vanish; heads of very different scales."""
    rig = Rig(6, 6, 2, d, 16, 7, (5003,), spread=3)
    rig.check(*rig.run())
    rig.close()
    rig = Rig(7, 6, 2, d, 32, 40, (3001, 5), spread=3)
    active = [[3, 17, 30], [39]]
    rig.check(*rig.run(active), active)
    rig.check(*rig.run())
    rig.close()


def test_scales_at_their_limits():
    """Values of 2^-23 and of 49152 beside each other, keys that are next to nothing."""
    rig = Rig(9, 4, 1, 128, 16, 4, (100,))
    sc = rig.pool.scales
    sc[:, :, 1] = rig.rng.choice([105, 140], sc[:, :, 1].shape)
    sc[:, :, 0] = rig.rng.choice([2, 60, 126], sc[:, :, 0].shape)
    rig.upload()
    rig.check(*rig.run())
    sc[:, :, 1] = 105
    rig.upload()
    rig.cache.clear()
    rig.check(*rig.run())
    rig.close()


def test_not_a_number_reaches_its_rows_only():
    """A value group that is NaN: its channels of every row.  A key group: every channel of the head.  Behind the end: nothing."""
    rig = Rig(10, 4, 2, 128, 16, 3, (40, 25))
    want, _ = rig.run()
    page = rig.indices[1]
    rig.pool.scales[page, 0, 1, 3, 2] = 255
    rig.upload()
    o, l = rig.run()
    nan = torch.isnan(o)
    assert bool(nan[:3, :2, 64:96].all()) and int(nan.sum()) == 3 * 2 * 32 and not bool(torch.isnan(l).any())
    assert torch.equal(o[~nan], want[~nan])
    rig.pool.scales[page, 0, 0, 3, 2] = 255
    rig.upload()
    o, l = rig.run()
    nan = torch.isnan(o)
    assert bool(nan[:3, :2].all()) and int(nan.sum()) == 3 * 2 * 128 and bool(torch.isnan(l[:3, :2]).all()) and int(torch.isnan(l).sum()) == 6
    rig.close()


def test_a_query_that_is_not_a_number_spoils_its_own_rows_only():
    for lens in ((40, 25), (2000, 0, 900)):
        rig = Rig(14, 6, 2, 64, 16, 3, lens)
        want, want_l = rig.run()
        rig.q_s[1, 4, 7] = 0x7FC0
        o, l = rig.run()
        assert bool(torch.isnan(o[1, 4]).all()) and bool(torch.isnan(l[1, 4])) and int(torch.isnan(o).sum()) == 64
        keep = torch.ones_like(l, dtype=torch.bool)
        keep[1, 4] = False
        assert torch.equal(o[keep], want[keep]) and torch.equal(l[keep], want_l[keep])
        rig.close()


@pytest.mark.parametrize("heads,batch", [(3, 70), (8, 40), (2, 200)])
def test_many_heads(heads, batch):
    """More lists than one wavefront has lanes, than are planned for, and rows that leave no room for partials."""
    rng = np.random.default_rng(heads)
    lens = tuple(int(x) for x in rng.integers(0, 90, batch))
    rig = Rig(heads, heads, heads, 64, 16, 2, lens)
    rig.check(*rig.run())
    active = [sorted(rng.permutation(2)[:rng.integers(0, 3)].tolist()) for _ in range(batch)]
    lists = [[sorted(rng.permutation(p)[:rng.integers(0, p + 1)].tolist()) for _ in range(heads)] for p in rig.pages]
    rig.check(*rig.run(active, lists), active, lists)
    rig.close()


def test_lists_of_very_different_lengths_and_rows():
    rig = Rig(15, 14, 2, 128, 16, 12, (6000, 0, 3, 700, 17))
    rng = rig.rng
    for trial in range(3):
        active = [sorted(rng.permutation(12)[:n].tolist()) for n in ((1, 12, 0, 5, 7), (12, 2, 12, 0, 1), (0, 0, 3, 0, 0))[trial]]
        rig.check(*rig.run(active), active)
        lists = [[sorted(rng.permutation(p)[:rng.integers(0, p + 1)].tolist()) for _ in range(2)] for p in rig.pages]
        rig.check(*rig.run(active, lists), active, lists)
    rig.close()


def test_the_same_call_twice_gives_the_same_bits():
    rig = Rig(12, 28, 4, 128, 16, 32, (3000, 1111))
    active = [[1, 4, 5, 9, 20, 31], [0]]
    first, again = rig.run(active), rig.run(active)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    first, again = rig.run(), rig.run()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda.current_stream().wait_stream(torch.cuda.default_stream())
        other = rig.run()
    assert torch.equal(first[0], other[0]) and torch.equal(first[1], other[1])
    rig.close()


@pytest.mark.parametrize("workgroups", [1, 3, 64, 1024])
def test_any_number_of_shares(workgroups):
    rig = Rig(13, 14, 2, 128, 16, 8, (900, 77))
    L.losa_set_tuning(rig.ctx, L.LOSA_TUNE_ATTN_WORKGROUPS, workgroups)
    rig.check(*rig.run())
    active = [[2, 7], [1, 3, 4]]
    rig.check(*rig.run(active), active)
    rig.close()


# ---- a cache's whole life: prompt, blocks, as a model uses the library

@pytest.mark.parametrize("dtype,g,mode,graph", [("bf16", 16, L.LOSA_SEL_TOPK, False), ("bf16", 32, L.LOSA_SEL_MASS, False), ("f32", 16, L.LOSA_SEL_TOPK, False),
                                                ("bf16", 16, L.LOSA_SEL_TOPK, True)])
def test_prompt_and_blocks_together(dtype, g, mode, graph):
    """A prompt is rotated and packed; then blocks: queries and keys rotated, a dense step, sparse steps, in-block attention, and the
    finished block appended.  Every step's active set and page lists, recomputed from what the library holds, and its
    attention, against the oracle.  Once as recorded graphs that are replayed."""
    rng = np.random.default_rng(21)
    Hq, Hkv, d, B, T, blocks, K = 8, 2, 128, 16, 3, 2, 3
    prompts = [75, 130]
    batch, G, H = 2, Hq // Hkv, 256
    total = [p + blocks * B for p in prompts]
    pages = [(n + g - 1) // g for n in total]
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    cfg = L.make_config(max_batch=batch, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d, hidden_size=H, page_size=g, block_size=B,
                        max_pages_per_seq=max(pages), max_topk_pages=K, dtype=L.LOSA_BF16 if dtype == "bf16" else L.LOSA_F32)
    ctx = L.losa_create(cfg, DEV)
    n = sum(pages)
    lens = torch.zeros(batch, dtype=torch.int32, device=DEV)
    kv = L.PackedKV(torch.full((n, Hkv, g, d // 2), 0x77, dtype=torch.uint8, device=DEV),
                    torch.full((n, Hkv, g // 4, 16, d // 32, 4), 0x77, dtype=torch.uint8, device=DEV),
                    torch.full((n, Hkv, 2, g, d // 32), 255, dtype=torch.uint8, device=DEV), torch.full((n, Hkv, 2, d), np.nan, dtype=tt, device=DEV),
                    dev(np.concatenate(([0], np.cumsum(pages))).astype(np.int32)), dev(rng.permutation(n).astype(np.int32)), lens)
    a = np.arange(max(total))[:, None] * 10000.0 ** (-np.arange(0, d, 2) / d)
    tab = np.concatenate((np.cos(a), np.sin(a)), 1).astype(np.float32)
    rot = L.Rotation(dev(tab))

    def tokens(m, heads):
        x = synth.store((rng.standard_normal((m, heads, d)) * np.exp(0.3 * rng.standard_normal((heads, d)))).astype(np.float32), dtype)
        return to_device(x, DEV), synth.load(x).astype(np.float64)

    k, kn = tokens(sum(prompts), Hkv)
    v, vn = tokens(sum(prompts), Hkv)
    lens.copy_(torch.tensor(prompts))
    L.losa_append_packed(ctx, kv, k, v, dev(np.array([0, prompts[0], sum(prompts)], np.int32)), rot, max_new_tokens=max(prompts))
    held = [[], []]        # what every sequence's tokens are after packing: (key, value) [Hkv, d]

    def hold(b, keys, values):
        for x, y in zip(keys, values):
            ck, cv = (orc.numbers(*orc.pack(z, lim)) for z, lim in ((x, orc.KEY_BYTES), (y, orc.VALUE_BYTES)))
            held[b].append((ck, cv))

    for b in range(batch):
        at = slice(0, prompts[0]) if b == 0 else slice(prompts[0], None)
        hold(b, orc.round_to(orc.rotate(kn[at], tab, range(prompts[b]), "halves"), dtype), vn[at])
    fixed = {"q": torch.zeros((batch * B, Hq, d), dtype=tt, device=DEV), "k": torch.zeros((batch * B, Hkv, d), dtype=tt, device=DEV)}
    v_b, raw_q, raw_k = torch.zeros_like(fixed["k"]), torch.zeros_like(fixed["q"]), torch.zeros_like(fixed["k"])
    h_cur, h_prev = (torch.zeros((batch * B, H), dtype=tt, device=DEV) for _ in range(2))
    pos = torch.zeros(batch * B, dtype=torch.int32, device=DEV)
    o_p, lse_p = torch.zeros((batch * B, Hq, d), device=DEV), torch.zeros((batch * B, Hq), device=DEV)
    mask, sel_count, out = torch.zeros(batch * B, dtype=torch.uint8, device=DEV), torch.zeros((batch, Hkv), dtype=torch.int32, device=DEV), torch.zeros_like(o_p)
    block_ptr = dev(np.arange(0, (batch + 1) * B, B).astype(np.int32))
    param = 5.0 if mode == L.LOSA_SEL_TOPK else 0.6

    def step(t):
        L.losa_rotate(ctx, rot, pos, raw_q, fixed["q"], raw_k, fixed["k"])
        L.losa_step_packed(ctx, kv, 0 if t == 0 else 1, h_cur, h_prev, fixed["q"], mode, param, K, o_p, lse_p, mask, sel_count)
        L.losa_block_merge(ctx, fixed["q"], fixed["k"], v_b, o_p, lse_p, out)

    def commit():
        lens.add_(B)
        L.losa_append_packed(ctx, kv, fixed["k"], v_b, block_ptr, max_new_tokens=B)

    calls = {}
    if graph:
        side = torch.cuda.Stream()
        for name, f in (("dense", lambda: step(0)), ("sparse", lambda: step(1)), ("commit", commit)):
            calls[name] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(calls[name], stream=side):
                f()
    hn = [rng.standard_normal((batch * B, H)).astype(np.float32)]
    scale = 1 / np.sqrt(d)
    for block in range(blocks):
        pos.copy_(torch.tensor([len(held[b]) + i for b in range(batch) for i in range(B)], dtype=torch.int32))
        for t in range(T):
            q, qn = tokens(batch * B, Hq)
            kb, kbn = tokens(batch * B, Hkv)
            vb, vbn = tokens(batch * B, Hkv)
            raw_q.copy_(q), raw_k.copy_(kb), v_b.copy_(vb)
            hn.append(hn[-1] + rng.standard_normal(hn[-1].shape).astype(np.float32) * rng.choice([0.5, 1e-3], (batch * B, 1)).astype(np.float32))
            h_prev.copy_(to_device(synth.store(hn[-2], dtype), DEV)), h_cur.copy_(to_device(synth.store(hn[-1], dtype), DEV))
            before = o_p.clone(), lse_p.clone()
            calls["dense" if t == 0 else "sparse"].replay() if graph else step(t)
            torch.cuda.synchronize()
            positions = pos.cpu().numpy()
            qr, kr = (orc.round_to(orc.rotate(x, tab, positions, "halves"), dtype) for x in (qn, kbn))
            o, l, final = (x.cpu().numpy().astype(np.float64) for x in (o_p, lse_p, out))
            delta = losa_oracle.locality_score(synth.load(synth.store(hn[-1], dtype)), synth.load(synth.store(hn[-2], dtype)))
            for b in range(batch):
                keys, values = np.stack([x for x, _ in held[b]]), np.stack([x for _, x in held[b]])
                m = (len(keys) + g - 1) // g
                A = list(range(B)) if t == 0 else list(losa_oracle.active_set(delta[b * B:(b + 1) * B], mode, param))
                if t:
                    assert np.array_equal(np.nonzero(mask.cpu().numpy()[b * B:(b + 1) * B])[0], A)
                for h in range(Hkv):
                    use = range(m)
                    if t:      # the union of the rows' best pages by the bounds of the packed keys
                        bounds = [orc.bound(None, keys[p * g:(p + 1) * g, h]) for p in range(m)]
                        lo, hi = (synth.load(synth.store(np.stack(x).astype(np.float32), dtype)).astype(np.float64) for x in zip(*bounds))
                        use = set()
                        for i in A:
                            for r in range(h * G, (h + 1) * G):
                                x = qr[b * B + i, r]
                                s = np.maximum(x * lo, x * hi).sum(1)
                                use |= set(np.argsort(-s, kind="stable")[:K].tolist())
                        assert int(sel_count[b, h]) == len(use)
                    sel = np.concatenate([np.arange(p * g, min((p + 1) * g, len(keys))) for p in sorted(use)])
                    for i in range(B):
                        for r in range(h * G, (h + 1) * G):
                            row = b * B + i
                            if i not in A:
                                assert np.array_equal(o[row, r], before[0][row, r].cpu().numpy()) and l[row, r] == float(before[1][row, r])
                                continue
                            want, lse = orc.attention(qr[row, r][None], keys[sel, h], values[sel, h], scale)
                            S = 2 * scale * (np.abs(keys[sel, h]) @ np.abs(qr[row, r])).max() + 16
                            ds = (d + 4) * U * S + 4 * U
                            assert np.abs(o[row, r] - want[0]).max() <= np.abs(values[sel, h]).max() * (4 * ds + (len(sel) + 70) * U)
                            assert abs(l[row, r] - lse[0]) <= ds + (len(sel) + 70) * U + 4 * U * abs(lse[0])
                    # merged with the block's own attention (the bound that losa_block_merge has elsewhere)
                    blk = slice(b * B, (b + 1) * B)
                    qh = qr[blk, h * G:(h + 1) * G].reshape(-1, d)
                    ob, lb = orc.attention(qh, kr[blk, h], vbn[blk, h], scale)
                    op, lp = o[blk, h * G:(h + 1) * G].reshape(-1, d), l[blk, h * G:(h + 1) * G].reshape(-1)
                    w = 1 / (1 + np.exp(lb - lp))
                    want = op * w[:, None] + ob * (1 - w[:, None])
                    assert np.abs(final[blk, h * G:(h + 1) * G].reshape(-1, d) - want).max() <= (2e-2 if dtype == "bf16" else 1e-4)
        calls["commit"].replay() if graph else commit()
        torch.cuda.synchronize()
        for b in range(batch):
            hold(b, kr[b * B:(b + 1) * B], vbn[b * B:(b + 1) * B])
        assert lens.tolist() == [len(x) for x in held]
        sizes = np.concatenate(([0], np.cumsum([len(x) for x in held]))).astype(np.int32)
        ko, vo = (torch.zeros((int(sizes[-1]), Hkv, d), dtype=tt, device=DEV) for _ in range(2))
        L.losa_read_packed(ctx, kv, dev(sizes), ko, vo)
        want = [np.stack([x[w] for s in held for x in s]) for w in range(2)]
        assert np.array_equal(synth.load(to_host(ko)), want[0]) and np.array_equal(synth.load(to_host(vo)), want[1])
    ctx.close()
