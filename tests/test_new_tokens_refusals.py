"""Host-side refusals of the entry points that fill a cache and of the 4-bit cache's, without a GPU: nothing is launched."""
import ctypes as C
import os

import pytest
import torch

from paper_2604_12056_amd import binding as L

FAKE = 1 << 20   # an aligned address that is never looked at
INV, UNS, OK = L.LOSA_ERR_INVALID_ARG, L.LOSA_ERR_UNSUPPORTED, L.LOSA_OK


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.LIB_PATH):
        from paper_2604_12056_amd.build import build_library
        build_library(verbose=False)
    return L.load_library()


@pytest.fixture(params=[L.LOSA_BF16, L.LOSA_F32])
def ctx(lib, request):
    cfg = L.make_config(max_batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, hidden_size=1024, page_size=16, block_size=32,
                        max_pages_per_seq=64, max_topk_pages=16, dtype=request.param)
    out = C.c_void_p()
    assert lib.losa_create(C.byref(cfg), 4096, L.losa_workspace_bytes(cfg), C.byref(out)) == OK
    yield out.value
    lib.losa_destroy(out.value)


def _kv(**kw):
    return L.losa_kv(**{**dict(k_pages=FAKE, v_pages=FAKE, meta=FAKE, page_indptr=FAKE, page_indices=FAKE, seq_lens=FAKE, batch=2, num_pages=100,
                               max_seq_pages=0), **kw})


def _packed(**kw):
    return L.losa_packed_kv(**{**dict(k_codes=FAKE, v_codes=FAKE, scales=FAKE, meta=FAKE, page_indptr=FAKE, page_indices=FAKE, seq_lens=FAKE,
                                      batch=2, num_pages=100, max_seq_pages=0), **kw})


def _new(**kw):
    return L.losa_new_tokens(**{**dict(k=FAKE, v=FAKE, k_stride=0, v_stride=0, tok_indptr=FAKE, positions=None, num_tokens=5, max_new_tokens=0), **kw})


def _rot(**kw):
    return L.losa_rotation(**{**dict(cos_sin=FAKE, max_positions=10, rotary_dim=128, style=0), **kw})


BAD_CACHE = [dict(batch=0), dict(batch=3), dict(num_pages=0), dict(num_pages=(1 << 26) + 1), dict(max_seq_pages=65), dict(max_seq_pages=-1),
             dict(page_indptr=None), dict(page_indices=None), dict(seq_lens=None), dict(meta=FAKE + 4)]
BAD_NEW = [dict(k=None), dict(v=None), dict(tok_indptr=None), dict(num_tokens=-1), dict(max_new_tokens=-1), dict(k=FAKE + 8), dict(v=FAKE + 2),
           dict(k_stride=255), dict(v_stride=258), dict(k_stride=-256)]
BAD_ROT = [(dict(cos_sin=None), INV), (dict(cos_sin=FAKE + 4), INV), (dict(max_positions=0), INV), (dict(rotary_dim=0), INV),
           (dict(rotary_dim=144), INV), (dict(rotary_dim=24), UNS), (dict(style=2), INV)]


@pytest.mark.parametrize("call,cache", [("losa_append_kv", _kv), ("losa_append_packed", _packed)])
def test_new_tokens(lib, ctx, call, cache):
    f = getattr(lib, call)
    pools = [dict(k_pages=None), dict(v_pages=FAKE + 8)] if cache is _kv else [dict(k_codes=None), dict(v_codes=FAKE + 8), dict(scales=None),
                                                                                dict(scales=FAKE + 1)]
    for bad in BAD_CACHE + pools:
        assert f(ctx, None, C.byref(cache(**bad)), C.byref(_new()), None) == INV, bad
        assert len(lib.losa_last_error(ctx)) > 0
    for bad in BAD_NEW:
        assert f(ctx, None, C.byref(cache()), C.byref(_new(**bad)), None) == INV, bad
    for bad, status in BAD_ROT:
        assert f(ctx, None, C.byref(cache()), C.byref(_new()), C.byref(_rot(**bad))) == status, bad
    assert f(ctx, None, None, C.byref(_new()), None) == INV and f(ctx, None, C.byref(cache()), None, None) == INV
    assert f(None, None, C.byref(cache()), C.byref(_new()), None) == INV
    assert f(ctx, None, C.byref(cache()), C.byref(_new(num_tokens=0, k=None, v=None, tok_indptr=None)), None) == OK   # nothing to do


def test_rotate(lib, ctx):
    def call(rot=None, positions=FAKE, tokens=5, q=(FAKE, 0, FAKE, 0), k=(FAKE, 0, FAKE, 0)):
        return lib.losa_rotate(ctx, None, C.byref(rot or _rot()), positions, tokens, *q, *k)
    none = (None, 0, None, 0)
    for bad, status in BAD_ROT:
        assert call(rot=_rot(**bad)) == status, bad
    assert lib.losa_rotate(ctx, None, None, FAKE, 5, FAKE, 0, FAKE, 0, *none) == INV
    assert lib.losa_rotate(None, None, C.byref(_rot()), FAKE, 5, FAKE, 0, FAKE, 0, *none) == INV
    assert call(tokens=-1) == INV and call(positions=None) == INV
    assert call(q=(FAKE, 0, None, 0)) == INV and call(k=(None, 0, FAKE, 0)) == INV
    assert call(q=(FAKE, 1023, FAKE, 0)) == INV and call(q=(FAKE, 0, FAKE, 1026)) == INV and call(k=(FAKE, 128, FAKE, 0)) == INV
    assert call(q=(FAKE + 4, 0, FAKE, 0)) == INV and call(k=(FAKE, 0, FAKE + 8, 0)) == INV
    assert call(tokens=0) == OK and call(q=none, k=none) == OK


def test_packed_reads(lib, ctx):
    read, attn, step = lib.losa_read_packed, lib.losa_sparse_attn_packed, lib.losa_step_packed
    for bad in BAD_CACHE + [dict(k_codes=None), dict(v_codes=None), dict(scales=None), dict(scales=FAKE + 8)]:
        kv = C.byref(_packed(**bad))
        assert read(ctx, None, kv, FAKE, 5, 0, FAKE, FAKE) == INV, bad
        assert attn(ctx, None, kv, FAKE, None, None, None, None, 0, FAKE, FAKE) == INV, bad
        assert step(ctx, None, kv, 1, FAKE, FAKE, FAKE, 0, 5.0, 4, FAKE, FAKE, None, None) == INV, bad
    kv = C.byref(_packed())
    assert read(ctx, None, kv, FAKE, -1, 0, FAKE, FAKE) == INV and read(ctx, None, kv, FAKE, 5, -1, FAKE, FAKE) == INV
    assert read(ctx, None, kv, None, 5, 0, FAKE, FAKE) == INV and read(ctx, None, kv, FAKE, 5, 0, FAKE + 8, None) == INV
    assert read(None, None, kv, FAKE, 5, 0, FAKE, FAKE) == INV
    assert read(ctx, None, kv, FAKE, 0, 0, FAKE, FAKE) == OK and read(ctx, None, kv, FAKE, 5, 0, None, None) == OK
    assert attn(ctx, None, kv, FAKE, FAKE, None, None, None, 0, FAKE, FAKE) == INV      # half a pair
    assert attn(ctx, None, kv, FAKE, None, None, FAKE, None, 4, FAKE, FAKE) == INV
    assert attn(ctx, None, kv, FAKE, None, None, FAKE, FAKE, 0, FAKE, FAKE) == INV      # no capacity
    assert attn(ctx, None, kv, None, None, None, None, None, 0, FAKE, FAKE) == INV
    assert attn(None, None, kv, FAKE, None, None, None, None, 0, FAKE, FAKE) == INV
    assert step(ctx, None, kv, 1, None, None, FAKE, 0, 5.0, 4, FAKE, FAKE, None, None) == INV
    assert step(ctx, None, kv, -1, FAKE, FAKE, FAKE, 0, 5.0, 4, FAKE, FAKE, None, None) == INV
    assert step(ctx, None, kv, 1, FAKE, FAKE, FAKE, 9, 5.0, 4, FAKE, FAKE, None, None) == INV
    assert step(ctx, None, kv, 1, FAKE, FAKE, FAKE, 0, 5.0, 99, FAKE, FAKE, None, None) == INV
    assert step(ctx, None, C.byref(_packed(meta=None)), 1, FAKE, FAKE, FAKE, 0, 5.0, 4, FAKE, FAKE, None, None) == INV


def test_binding_refuses_rows_it_cannot_describe():
    cfg = L.make_config(max_batch=1, num_q_heads=4, num_kv_heads=2, head_dim=64, hidden_size=256, page_size=16, block_size=4,
                        max_pages_per_seq=4, max_topk_pages=1)
    ctx = L.Context(None, None, cfg)
    x = torch.zeros((6, 8, 64), dtype=torch.bfloat16)
    assert L._row_stride(x[:, 2:4], ctx, 6, 2, "k") == 512 and L._row_stride(x[:1, 2:4], ctx, 1, 2, "k") == 0
    assert L._row_stride(x[::2, 2:4], ctx, 3, 2, "k") == 1024
    for bad in (x, x[:, ::4], x[:, 2:4].float(), x[:, 2:4].transpose(0, 1), x[:1, :2].expand(6, 2, 64), x[..., :32][:, :2], x[:5, :2], x[0]):
        with pytest.raises(L.LosaError) as e:
            L._row_stride(bad, ctx, 6, 2, "k")
        assert e.value.status == INV
    rot = L.Rotation(torch.zeros((8, 64)))
    with pytest.raises(L.LosaError):
        L.losa_rotate(ctx, rot, torch.zeros(5, dtype=torch.int32), x[:, :4], x[:, :4].clone())   # five positions, six tokens
    for k, v, positions in ((x[:, :2], x[:5, :2], None), (x[:, :2], x[:, :2], torch.zeros(5, dtype=torch.int32))):
        with pytest.raises(L.LosaError):
            L._new_tokens(ctx, k, v, torch.zeros(2, dtype=torch.int32), positions, 0)
