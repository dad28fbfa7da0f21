"""CPU oracle (numpy, float64) of what fills a paged cache and of the cache in 4 bits, written from the definitions in
include/losa.h: position rotation, new tokens into pages, page bounds, the MXFP4 format.  Test infrastructure only; it shares
no code with the HIP path."""
from __future__ import annotations

import numpy as np

NUMBERS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
KEY_BYTES, VALUE_BYTES, NAN_BYTE = (2, 252), (105, 140), 255


def round_to(x: np.ndarray, dtype: str) -> np.ndarray:
    """float64 -> the nearest number of the storage type (by way of float32 for bfloat16), as float64."""
    with np.errstate(over="ignore", invalid="ignore"):
        f = np.asarray(x, np.float64).astype(np.float32)
    if dtype == "f32":
        return f.astype(np.float64)
    u = f.view(np.uint32).astype(np.uint64)
    r = (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(f), np.nan, r).astype(np.float64)


def rotate(x: np.ndarray, table: np.ndarray, positions, style: str) -> np.ndarray:
    """x [tokens, heads, d] with the angles of table[positions] ([cosines | sines]); not rounded."""
    y, r = np.array(x, np.float64), table.shape[1]
    for n, p in enumerate(positions):
        for i in range(r // 2):
            c, s = float(table[p, i]), float(table[p, r // 2 + i])
            a, b = (i, i + r // 2) if style == "halves" else (2 * i, 2 * i + 1)
            x1, x2 = y[n, :, a].copy(), y[n, :, b].copy()
            with np.errstate(invalid="ignore"):
                y[n, :, a], y[n, :, b] = x1 * c - x2 * s, x2 * c + x1 * s
    return y


def pack(x: np.ndarray, limits):
    """[..., d] -> (codes [..., d], scale bytes [..., d/32])."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    top = np.abs(g).max(-1)
    bad = ~np.isfinite(top)
    safe = np.where(bad | (top == 0), 1.0, top)
    e = np.floor(np.log2(safe)).astype(int)
    e = np.where(2.0 ** e > safe, e - 1, np.where(2.0 ** (e + 1) <= safe, e + 1, e))    # (log2's last bit)
    byte = e - 2 + 127
    byte = np.where(safe >= 7 * 2.0 ** (byte - 127.0), byte + 1, byte)
    byte = np.where(top == 0, limits[0], np.clip(byte, *limits))
    with np.errstate(invalid="ignore"):
        y = np.abs(g) / 2.0 ** (byte[..., None] - 127.0)
    y = np.where(bad[..., None], 0.0, np.minimum(y, 8.0))      # (far beyond 6 all numbers are equally far in float64)
    away = np.abs(y[..., None] - NUMBERS)                      # nearest number; of two equally near ones the even code
    code = np.argmin(away + 1e-300 * (np.arange(8) % 2), axis=-1)
    near = np.sort(away, axis=-1)
    tie = near[..., 0] == near[..., 1]
    first = np.argmin(away, axis=-1)
    code = np.where(tie, first + first % 2, code)
    code = code + 8 * ((np.signbit(g)) & ~bad[..., None])
    return code.reshape(x.shape), np.where(bad, NAN_BYTE, byte)


def numbers(code: np.ndarray, byte: np.ndarray) -> np.ndarray:
    """Codes [..., d] and scale bytes [..., d/32] -> float64 [..., d]."""
    v = NUMBERS[code % 8] * np.where(code >= 8, -1.0, 1.0)
    scale = np.where(byte == NAN_BYTE, np.nan, 2.0 ** (byte.astype(np.float64) - 127.0))
    return (v.reshape(*byte.shape, 32) * scale[..., None]).reshape(code.shape)


class PackedPool:
    """The pools of a 4-bit cache as the library lays them out (numpy uint8), token by token."""

    def __init__(self, k_codes, v_codes, scales):
        self.k_codes, self.v_codes, self.scales = k_codes, v_codes, scales

    def put(self, page, head, row, key, value):
        """One token: key and value of T, already turned and rounded."""
        for x, limits, which in ((key, KEY_BYTES, 0), (value, VALUE_BYTES, 1)):
            code, byte = pack(np.asarray(x, np.float64), limits)
            self.scales[page, head, which, row] = byte
            if which == 0:
                self.k_codes[page, head, row] = code[0::2] | code[1::2] << 4
            else:
                for j in range(len(byte)):
                    low, high = code[32 * j:32 * j + 16], code[32 * j + 16:32 * j + 32]
                    self.v_codes[page, head, row // 4, :, j, row % 4] = low | high << 4

    def get(self, page, head, row):
        """(key, value) of one token, float64 [d] each."""
        kc = self.k_codes[page, head, row].astype(int)
        code = np.stack((kc & 15, kc >> 4), 1).reshape(-1)
        vc = self.v_codes[page, head, row // 4, :, :, row % 4].astype(int).T      # [d/32, 16]
        vcode = np.concatenate((vc & 15, vc >> 4), 1).reshape(-1)
        return (numbers(code, self.scales[page, head, 0, row].astype(int)),
                numbers(vcode, self.scales[page, head, 1, row].astype(int)))


def places(indptr, page_indptr, page_indices, seq_lens, g, num_pages, most_pages=1 << 30):
    """(row of the new tokens, place in the sequence, page, row in it, sequence) of every new token that has a place."""
    for b in range(len(seq_lens)):
        n = int(indptr[b + 1]) - int(indptr[b])
        for i in range(n):
            slot = int(seq_lens[b]) - n + i
            p = slot // g
            if slot < 0 or p >= min(int(page_indptr[b + 1]) - int(page_indptr[b]), most_pages):
                continue
            page = int(page_indices[int(page_indptr[b]) + p])
            if 0 <= page < num_pages:
                yield int(indptr[b]) + i, slot, page, slot % g, b


def bound(old, fresh):
    """Bounds of a page from its old ones (None: it held no token) and the keys [n, d] that join it; NaN are passed over."""
    all_k = fresh if old is None else np.concatenate((old, fresh))
    return np.fmin.reduce(all_k), np.fmax.reduce(all_k)


def attention(q, k, v, scale):
    """(o, lse) of query rows [M, d] over keys and values [n, d]; no token: zeros and -inf."""
    if len(k) == 0:
        return np.zeros((len(q), v.shape[-1])), np.full(len(q), -np.inf)
    s = scale * q @ k.T
    m = s.max(1, keepdims=True)
    e = np.exp(s - m)
    l = e.sum(1, keepdims=True)
    return e @ v / l, (m + np.log(l))[:, 0]
