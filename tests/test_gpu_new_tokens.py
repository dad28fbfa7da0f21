"""Rotation and new tokens into a cache's pages (losa_rotate, losa_append_kv, losa_append_packed, losa_read_packed) against the CPU
oracle, bit for bit: a result is the exact one rounded once, codes and bounds follow from it, and nothing else is written.
The one exception is a float result next to a tie, where the kernel's pair of floats (2^-45) and the oracle's doubles may
round apart: float rotations are compared to one step of the type (2^-23 relative)."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2604_12056_amd import binding as L
from paper_2604_12056_amd import synth
from paper_2604_12056_amd.device_inputs import to_device, to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def config(dtype, Hq=8, Hkv=2, d=128, g=16, batch=3, max_pages=16, B=8):
    return L.make_config(max_batch=batch, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d, hidden_size=Hq * d, page_size=g, block_size=B,
                         max_pages_per_seq=max_pages, max_topk_pages=max_pages, dtype=L.LOSA_BF16 if dtype == "bf16" else L.LOSA_F32)


def table(rng, positions, rotary):
    a = rng.uniform(0, 6.3, (positions, rotary // 2))
    return np.concatenate((np.cos(a), np.sin(a)), 1).astype(np.float32)


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def rows(rng, n, heads, d, dtype, scale=None):
    """Storage array [n, heads, d] and its values."""
    x = rng.standard_normal((n, heads, d)) * np.exp(rng.standard_normal((heads, d)) if scale is None else scale)
    s = synth.store(x.astype(np.float32), dtype)
    return s, synth.load(s).astype(np.float64)


def host(t):
    return synth.load(to_host(t)).astype(np.float64)


def same(got, want, dtype, turned):
    if dtype == "f32" and turned:
        np.testing.assert_allclose(got, want, rtol=2.0 ** -23, atol=2.0 ** -140)
    else:
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rotary,style", [(128, 128, "halves"), (128, 64, "halves"), (128, 48, "halves"), (128, 16, "pairs"), (64, 64, "pairs"),
                                            (64, 32, "halves"), (128, 128, "pairs"), (128, 112, "halves")])
@pytest.mark.parametrize("tokens", [1, 5, 67])
def test_rotate(dtype, d, rotary, style, tokens):
    rng = np.random.default_rng(tokens * 7 + rotary)
    ctx = L.losa_create(config(dtype, d=d), DEV)
    fused, fv = rows(rng, tokens, 8 + 2 * 2, d, dtype)
    q, k = fv[:, :8], fv[:, 8:10]
    tab = table(rng, 50, rotary)
    pos = rng.integers(0, 50, tokens).astype(np.int32)
    off = rng.random(tokens) < 0.2
    pos[off] = rng.choice([-1, 50, 2 ** 31 - 1, -2 ** 31], off.sum())
    at = np.where(off, 0, pos)
    want_q, want_k = (orc.round_to(orc.rotate(x, tab, at, style), dtype) for x in (q, k))
    rot = L.Rotation(dev(tab), L.LOSA_ROTATE_HALVES if style == "halves" else L.LOSA_ROTATE_PAIRS)
    x = to_device(fused, DEV)
    # out of the fused projection into tensors of their own; rows of tokens that the table does not reach keep what they hold
    q_out, k_out = torch.full((tokens, 8, d), 7.0, dtype=x.dtype, device=DEV), torch.full((tokens, 2, d), 7.0, dtype=x.dtype, device=DEV)
    L.losa_rotate(ctx, rot, dev(pos), x[:, :8], q_out, x[:, 8:10], k_out)
    for got, want in ((q_out, want_q), (k_out, want_k)):
        assert np.all(host(got)[off] == 7.0)
        same(host(got)[~off], want[~off], dtype, True)
    # in place, each alone
    q_alone = torch.zeros_like(q_out)
    L.losa_rotate(ctx, rot, dev(pos), q=x[:, :8], q_out=q_alone)
    L.losa_rotate(ctx, rot, dev(pos), x[:, :8], x[:, :8], x[:, 8:10], x[:, 8:10])
    y = host(x)
    assert np.array_equal(y[off], fv[off]) and np.array_equal(y[:, 10:], fv[:, 10:])
    assert np.array_equal(y[~off, :8], host(q_out)[~off]) and np.array_equal(y[~off, 8:10], host(k_out)[~off])
    assert np.array_equal(host(q_alone)[~off], host(q_out)[~off]) and np.all(host(q_alone)[off] == 0)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotate_of_infinities_and_zeros(dtype):
    """What an ordinary product gives, no more NaN than that."""
    ctx = L.losa_create(config(dtype, Hq=2, Hkv=2, d=64), DEV)
    vals = np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 3.0e38, 1e-38, 1.0], np.float32)
    x = np.zeros((8, 2, 64), np.float32)
    x[:, 0, :32], x[:, 0, 32:] = vals[:, None], 1.0
    x[:, 1, :32], x[:, 1, 32:] = vals[:, None], vals[None, np.arange(32) % 8]
    s = synth.store(x, dtype)
    v = synth.load(s).astype(np.float64)
    tab = np.concatenate((np.full((8, 32), 0.6), np.full((8, 32), 0.8)), 1).astype(np.float32)
    want = orc.round_to(orc.rotate(v, tab, range(8), "halves"), dtype)
    q = to_device(s, DEV)
    L.losa_rotate(ctx, L.Rotation(dev(tab)), torch.arange(8, dtype=torch.int32, device=DEV), q, q)
    got = host(q)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    same(got[~np.isnan(want)], want[~np.isnan(want)], dtype, True)
    ctx.close()


class Cache:
    """Pools with arbitrary contents, a page table, and the same on the host."""

    def __init__(self, rng, dtype, packed, Hkv, d, g, before, new, spare_pages=1, lists=None):
        self.dtype, self.packed, self.Hkv, self.d, self.g = dtype, packed, Hkv, d, g
        self.lens = np.array([b + n for b, n in zip(before, new)], np.int32)
        pages = [(int(n) + g - 1) // g + spare_pages for n in self.lens]
        self.num_pages = sum(pages) + 2
        self.page_indptr = np.concatenate(([0], np.cumsum(pages))).astype(np.int32)
        self.page_indices = rng.permutation(self.num_pages)[:sum(pages)].astype(np.int32)
        self.indptr = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        n = self.num_pages
        if packed:
            J = d // 32
            self.pool = orc.PackedPool(rng.integers(0, 256, (n, Hkv, g, d // 2), dtype=np.uint8),
                                       rng.integers(0, 256, (n, Hkv, g // 4, 16, J, 4), dtype=np.uint8),
                                       rng.integers(110, 135, (n, Hkv, 2, g, J), dtype=np.uint8))
        else:
            self.k, self.v = (synth.store(rng.standard_normal((n, Hkv, g, d) if w == 0 else (n, Hkv, d, g)).astype(np.float32), dtype) for w in range(2))
        self.meta = synth.store(rng.standard_normal((n, Hkv, 2, d)).astype(np.float32), dtype)
        for b, held in enumerate(before):      # bounds of the pages that hold tokens already: exactly those of their keys
            for p in range((held + g - 1) // g):
                page = self.page_indices[self.page_indptr[b] + p]
                fill = min(g, held - p * g)
                for h in range(Hkv):
                    lo, hi = orc.bound(None, self.keys(page, h, fill))
                    self.meta[page, h] = synth.store(np.stack((lo, hi)).astype(np.float32), dtype)

    def keys(self, page, h, fill):
        if self.packed:
            return np.stack([self.pool.get(page, h, r)[0] for r in range(fill)])
        return synth.load(self.k[page, h, :fill]).astype(np.float64)

    def upload(self):
        self.d_meta = to_device(self.meta.copy(), DEV)
        args = [dev(self.page_indptr), dev(self.page_indices), dev(self.lens)]
        if self.packed:
            self.pools = [dev(x.copy()) for x in (self.pool.k_codes, self.pool.v_codes, self.pool.scales)]
            return L.PackedKV(*self.pools, self.d_meta, *args)
        self.pools = [to_device(x.copy(), DEV) for x in (self.k, self.v)]
        return L.PagedKV(*self.pools, self.d_meta, *args)

    def expect(self, k, v, tab=None, style="halves", positions=None, most_pages=1 << 30):
        """The host's pools and bounds after the tokens k, v (values [T, Hkv, d])."""
        joined = {}
        for row, slot, page, r, b in orc.places(self.indptr, self.page_indptr, self.page_indices, self.lens, self.g, self.num_pages, most_pages):
            key = k[row]
            if tab is not None:
                at = slot if positions is None else int(positions[row])
                if not 0 <= at < len(tab):
                    continue
                key = orc.round_to(orc.rotate(key[None], tab, [at], style), self.dtype)[0]
            held = self.lens[b] - (self.indptr[b + 1] - self.indptr[b]) > slot // self.g * self.g
            for h in range(self.Hkv):
                if self.packed:
                    self.pool.put(page, h, r, key[h], v[row, h])
                    key[h] = self.pool.get(page, h, r)[0]
                else:
                    self.k[page, h, r] = synth.store(key[h].astype(np.float32), self.dtype)
                    self.v[page, h, :, r] = synth.store(v[row, h].astype(np.float32), self.dtype)
            joined.setdefault(page, (held, []))[1].append(key)
        for page, (held, keys) in joined.items():
            for h in range(self.Hkv):
                fresh = np.stack([key[h] for key in keys])
                old = synth.load(self.meta[page, h]).astype(np.float64) if held else None
                self.meta[page, h] = synth.store(np.stack(orc.bound(old, fresh)).astype(np.float32), self.dtype)

    def check(self, turned=False):
        torch.cuda.synchronize()
        if self.packed:
            for got, want in zip(self.pools, (self.pool.k_codes, self.pool.v_codes, self.pool.scales)):
                np.testing.assert_array_equal(got.cpu().numpy(), want)
        else:
            same(host(self.pools[0]), synth.load(self.k).astype(np.float64), self.dtype, turned)
            np.testing.assert_array_equal(host(self.pools[1]), synth.load(self.v).astype(np.float64))
        same(host(self.d_meta), synth.load(self.meta).astype(np.float64), self.dtype, turned)


def append(ctx, c, kv, k, v, *a, **kw):
    (L.losa_append_packed if c.packed else L.losa_append_kv)(ctx, kv, k, v, dev(c.indptr), *a, **kw)


SHAPES = [  # heads, d, g, tokens before, new tokens
    (2, 128, 16, (0, 5, 16), (1, 1, 1)),
    (2, 128, 16, (0, 3, 40), (33, 13, 0)),
    (1, 64, 16, (7, 0, 15), (9, 16, 2)),
    (5, 64, 32, (0, 31, 70), (64, 33, 7)),
    (4, 128, 32, (1, 0, 0), (95, 0, 32)),
]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,d,g,before,new", SHAPES)
@pytest.mark.parametrize("rotary,style,fused,given", [(0, "halves", False, False), (-1, "halves", True, False), (32, "pairs", False, True),
                                                      (48, "halves", True, True)])
def test_append(packed, dtype, heads, d, g, before, new, rotary, style, fused, given):
    rng = np.random.default_rng(heads * 100 + g + rotary)
    c = Cache(rng, dtype, packed, heads, d, g, before, new)
    ctx = L.losa_create(config(dtype, Hq=heads, Hkv=heads, d=d, g=g), DEV)
    T = sum(new)
    stored, values = rows(rng, T, 3 * heads, d, dtype)
    k, v = values[:, heads:2 * heads], values[:, 2 * heads:]
    tab = pos = rot = None
    if rotary:
        tab = table(rng, 60 if given else 200, d if rotary < 0 else rotary)
        rot = L.Rotation(dev(tab), L.LOSA_ROTATE_HALVES if style == "halves" else L.LOSA_ROTATE_PAIRS)
        if given:
            pos = rng.integers(-2, 62, T).astype(np.int32)      # some that the table does not reach
    kv = c.upload()
    x = to_device(stored, DEV)
    kd, vd = x[:, heads:2 * heads], x[:, 2 * heads:]
    if not fused:
        kd, vd = kd.contiguous(), vd.contiguous()
    c.expect(k.copy(), v, tab, style, pos)
    for max_new in (0, max(new)):      # the same call again leaves the same pages
        append(ctx, c, kv, kd, vd, rot, None if pos is None else dev(pos), max_new_tokens=max_new)
        c.check(turned=rotary != 0)
    if packed:   # and the tokens read back
        outs = [torch.full((T, heads, d), 9.0, dtype=x.dtype, device=DEV) for _ in range(2)]
        L.losa_read_packed(ctx, kv, dev(c.indptr), *outs, max_tokens=max(new))
        want = np.full((2, T, heads, d), 9.0)
        for row, _, page, r, _ in orc.places(c.indptr, c.page_indptr, c.page_indices, c.lens, g, c.num_pages):
            for h in range(heads):
                want[0, row, h], want[1, row, h] = c.pool.get(page, h, r)
        np.testing.assert_array_equal(host(outs[0]), want[0])
        np.testing.assert_array_equal(host(outs[1]), want[1])
        alone = torch.zeros_like(outs[0])
        L.losa_read_packed(ctx, kv, dev(c.indptr), None, alone)
        assert torch.equal(alone, outs[1])
    ctx.close()


@pytest.mark.parametrize("packed", [False, True])
def test_append_leaves_out_what_has_no_place(packed):
    """Page ids outside the pool, pages that are not listed or beyond the caller's bound, lengths that do not hold the new tokens."""
    rng = np.random.default_rng(5)
    c = Cache(rng, "bf16", packed, 2, 128, 16, (4, 20, 0), (60, 50, 70), spare_pages=0)
    c.page_indices[1], c.page_indices[int(c.page_indptr[1]) + 2] = -7, c.num_pages
    c.page_indptr[3] -= 1                    # the last sequence's last page is not listed
    c.lens[2] = 55                           # fifteen of its tokens would lie before its first
    ctx = L.losa_create(config("bf16", Hq=2, Hkv=2), DEV)
    stored, values = rows(rng, 180, 4, 128, "bf16")
    kv = c.upload()
    kv.max_seq_pages = 4
    x = to_device(stored, DEV)
    c.expect(values[:, :2].copy(), values[:, 2:], most_pages=4)
    append(ctx, c, kv, x[:, :2], x[:, 2:])
    c.check()
    if packed:
        out = torch.full((180, 2, 128), 9.0, dtype=x.dtype, device=DEV)
        L.losa_read_packed(ctx, kv, dev(c.indptr), out, None)
        read = {row for row, *_ in orc.places(c.indptr, c.page_indptr, c.page_indices, c.lens, 16, c.num_pages, 4)}
        assert {i for i in range(180) if not np.all(host(out)[i] == 9.0)} == read
    # rows past num_tokens are never read: a table that says there are more
    c.indptr[3] += 1000
    append(ctx, c, kv, x[:, :2], x[:, 2:])
    torch.cuda.synchronize()
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packing_of_extreme_groups(dtype):
    """Zeros, infinities, NaN, the smallest and largest numbers, ties between codes and between scales."""
    rng = np.random.default_rng(11)
    groups = []
    for top in [0.0, 1e-45, 1e-38, 2.0 ** -125, 2.0 ** -24, 2.0 ** -22, 1.0, 3.4999, 3.5, 6.0, 6.984375, 7.0, 49152.0, 57344.0, 65504.0, 1e6, 3e38, np.inf, np.nan]:
        x = (rng.uniform(-1, 1, 32) * (top if np.isfinite(top) else 1.0)).astype(np.float32)
        x[rng.integers(32)] = top * rng.choice([-1.0, 1.0])
        groups.append(x)
    mid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], np.float32)
    for e in (-20, 0, 9):
        groups.append(np.concatenate((mid, -mid, mid / 2, -mid * 0.5)) * 2.0 ** e)
    n = len(groups)
    groups = np.stack(groups + [groups[0]] * (-n % 4)).reshape(-1, 1, 128).astype(np.float32)
    T = len(groups)
    s = synth.store(groups, dtype)
    values = synth.load(s).astype(np.float64)
    c = Cache(rng, dtype, True, 1, 128, 16, (0,), (T,))
    ctx = L.losa_create(config(dtype, Hq=1, Hkv=1, batch=1), DEV)
    kv = c.upload()
    c.expect(values.copy(), values)
    x = to_device(s, DEV)
    append(ctx, c, kv, x, x)
    c.check()
    out = torch.zeros((T, 1, 128), dtype=x.dtype, device=DEV), torch.zeros((T, 1, 128), dtype=x.dtype, device=DEV)
    L.losa_read_packed(ctx, kv, dev(c.indptr), *out)
    for t in range(T):
        page = c.page_indices[t // 16]
        for got, want in zip(out, c.pool.get(page, 0, t % 16)):
            np.testing.assert_array_equal(host(got)[t, 0], want)
    ctx.close()


def test_empty_calls_and_no_bounds():
    rng = np.random.default_rng(3)
    for packed in (False, True):
        c = Cache(rng, "bf16", packed, 2, 64, 16, (3, 0), (0, 0))
        ctx = L.losa_create(config("bf16", Hq=2, Hkv=2, d=64), DEV)
        kv = c.upload()
        none = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device=DEV)
        append(ctx, c, kv, none, none)
        c.check()
        c = Cache(rng, "bf16", packed, 2, 64, 16, (3, 0), (20, 1))
        stored, values = rows(rng, 21, 2, 64, "bf16")
        kv = c.upload()
        kv.meta = None
        meta = c.meta.copy()
        c.expect(values.copy(), values)
        c.meta = meta
        append(ctx, c, kv, to_device(stored, DEV), to_device(stored, DEV))
        c.check()
        ctx.close()


def test_append_agrees_with_page_bounds():
    """Bounds kept along the way are those that losa_page_bounds makes of the finished pages, whatever the steps were."""
    rng = np.random.default_rng(8)
    lens = (61, 16, 33)
    c = Cache(rng, "bf16", False, 2, 128, 16, (0, 0, 0), lens)
    ctx = L.losa_create(config("bf16", Hq=2, Hkv=2), DEV)
    kv = c.upload()
    stored, _ = rows(rng, sum(lens), 2, 128, "bf16")
    x, done = to_device(stored, DEV), np.zeros(3, int)
    starts = np.concatenate(([0], np.cumsum(lens)))[:3]
    while np.any(done < lens):
        n = np.minimum(rng.integers(0, 19, 3), np.array(lens) - done)
        take = np.concatenate([np.arange(s + d0, s + d0 + m) for s, d0, m in zip(starts, done, n)]).astype(np.int64)
        done = done + n
        kv.seq_lens = dev(done.astype(np.int32))
        part = x[torch.from_numpy(take).to(DEV)]
        L.losa_append_kv(ctx, kv, part, part, dev(np.concatenate(([0], np.cumsum(n))).astype(np.int32)), max_new_tokens=int(max(n.max(), 1)))
    kept = kv.meta.clone()
    L.losa_page_bounds(ctx, kv)
    torch.cuda.synchronize()
    used = np.concatenate([c.page_indices[c.page_indptr[b]:c.page_indptr[b] + (lens[b] + 15) // 16] for b in range(3)])
    assert np.array_equal(host(kept)[used], host(kv.meta)[used])
    ctx.close()
