// What the kernels that bring new tokens into a paged cache share: the position rotation of 16 bytes of a row, and which
// page and which of its rows a workgroup fills.
#pragma once
#include "losa_device.h"
#include "losa_internal.h"

namespace losa {

// Bytes that a launch reads, or writes, once: they need displace nothing in the caches.  (What each is worth is said where it is used.)
typedef __attribute__((ext_vector_type(4))) uint32_t words4_t;
__device__ __forceinline__ uint4 load_once(const void* p) {
  const words4_t x = __builtin_nontemporal_load(reinterpret_cast<const words4_t*>(p));
  return make_uint4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ uint32_t load_once(const uint32_t* p) { return __builtin_nontemporal_load(p); }
__device__ __forceinline__ void store_once(void* p, const uint4& v) {
  __builtin_nontemporal_store((words4_t){v.x, v.y, v.z, v.w}, reinterpret_cast<words4_t*>(p));
}

// ---- the rotation.  (x1, x2) of an angle (c, s) becomes (x1 c - x2 s, x2 c + x1 s).
//
// Both products and the difference are taken with their rounding errors (a product's by one fused multiply-add, a
// sum's by Knuth's two-sum), so the result is the exact one rounded once, but for 2^-45 or so: a key that is coded in 4 bits right
// after may lie next to a border between two codes, where a float's last bit would decide.  Some ten vector operations
// a channel, where a quarter-rate conversion to double and back would take longer than the bytes.
__device__ __forceinline__ float turned(float x1, float c, float x2, float s) {   // x1 c + x2 s
#pragma clang fp contract(off)
  const float a = x1 * c, b = x2 * s;
  const float ea = __builtin_fmaf(x1, c, -a), eb = __builtin_fmaf(x2, s, -b);
  const float sum = a + b, t = sum - a;
  const float err = (a - (sum - t)) + (b - t);
  // (An infinity's error term is no number, so the maximum below passes over it; a number's is above -3 * 2^103.)
  return sum + __builtin_fmaxf(err + (ea + eb), -0x1p105f);
}

// A unit is two 16-byte chunks of a row and the V angles that turn them: halves style channels u V .. and half a turn's width
// further, pairs style 2 V neighbours.  Units past rotary_dim are 2 V neighbours that pass through.
struct Unit {
  int first, second;   // channels its two chunks start at
  int angle;           // its first angle; negative: passes through
};
template <int V>
__device__ __forceinline__ Unit unit_of(int u, int rotary, bool pairs) {
  const int turning = rotary / (2 * V);
  if (u >= turning) return {rotary + (u - turning) * 2 * V, rotary + (u - turning) * 2 * V + V, -1};
  return pairs ? Unit{u * 2 * V, u * 2 * V + V, u * V} : Unit{u * V, rotary / 2 + u * V, u * V};
}

// Chunks `a` and `b` of a unit, widened, turned in place by the angles' cosines and sines.
template <int V>
__device__ __forceinline__ void turn_unit(float (&a)[V], float (&b)[V], const float (&c)[V], const float (&s)[V], bool pairs) {
  if (!pairs) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float x1 = a[e], x2 = b[e];
      a[e] = turned(x1, c[e], x2, -s[e]);
      b[e] = turned(x2, c[e], x1, s[e]);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < V; e += 2) {
    const float x1 = a[e], x2 = a[e + 1], y1 = b[e], y2 = b[e + 1];
    const float ca = c[e / 2], sa = s[e / 2], cb = c[V / 2 + e / 2], sb = s[V / 2 + e / 2];
    a[e] = turned(x1, ca, x2, -sa);
    a[e + 1] = turned(x2, ca, x1, sa);
    b[e] = turned(y1, cb, y2, -sb);
    b[e + 1] = turned(y2, cb, y1, sb);
  }
}

template <int V>
__device__ __forceinline__ void load_floats(const float* p, float (&f)[V]) {
#pragma unroll
  for (int e = 0; e < V; e += 4) {
    const float4 x = *reinterpret_cast<const float4*>(p + e);
    f[e] = x.x;
    f[e + 1] = x.y;
    f[e + 2] = x.z;
    f[e + 3] = x.w;
  }
}

// Floats to one 16-byte vector of T, rounded to nearest, ties to even.
__device__ __forceinline__ uint4 round16(const float (&f)[8], bf16_t) {
  typedef __attribute__((ext_vector_type(8))) float f8;
  typedef __attribute__((ext_vector_type(8))) __bf16 b8;
  const f8 x = {f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]};
  return __builtin_bit_cast(uint4, __builtin_convertvector(x, b8));
}
__device__ __forceinline__ uint4 round16(const float (&f)[4], float) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// ---- the page a workgroup fills
// Rows lo .. hi-1 of a page take the new tokens from row `source` of k and v on; the first of them is token `slot` of the sequence.
struct Fill {
  int entry, lo, hi, source, slot;   // entry: the page's place in page_indices
};
// The `tile`-th page of sequence b that gets new tokens; hi <= lo where there is none.
// The sequence's last n tokens are the new ones; tokens whose page is not listed or beyond the launch's bound are left out.
// (Whether the page is in the pool is the caller's to check, with other loads already on their way.)
__device__ __forceinline__ Fill fill_of(const KvView& kv, const Shape& sh, const int32_t* indptr, int num_tokens, int b, int tile) {
  const int t0 = max(indptr[b], 0), t1 = min(indptr[b + 1], num_tokens), len = max(kv.seq_lens[b], 0);
  const int base = kv.page_indptr[b], listed = kv.page_indptr[b + 1] - base;
  const int n = t1 - t0, first = len - n, begin = max(first, 0), shift = sh.g == 16 ? 4 : 5;
  const int p = (begin >> shift) + tile;
  if (n <= 0 || p >= min(min(listed, sh.max_pages), kv.seq_page_limit)) return {0, 0, 0, 0, 0};
  const int lo = max(begin - (p << shift), 0), hi = min(len - (p << shift), sh.g), slot = (p << shift) + lo;
  return {base + p, lo, hi, t0 + (slot - first), slot};
}
// Pages that n tokens can touch at most.
inline int pages_touched(int n, int g) { return n <= 0 ? 0 : (int)(((long)n + 2 * g - 2) / g); }

// Elementwise minimum and maximum over rows [lo, hi) of which `ok` says which hold a token, of the page-head tile `rows` (T [g][d]
// in LDS, written by this wavefront), combined with what the page's bounds say where it held tokens before, to `meta`.
// A lane takes the channels of one dword.  Minima and maxima pass over NaN as losa_page_bounds does.
template <typename T, int D>
__device__ __forceinline__ void bounds_from_lds(const T* rows, uint32_t ok, int lo, int hi, bool held, T* meta, int lane) {
  constexpr int E = 4 / sizeof(T);   // channels of a dword
  if (!ok) return;
#pragma unroll
  for (int w = 0; w < D / E; w += 64) {
    const int at = w + lane;
    if (at >= D / E) break;
    float mn[E], mx[E];
    const auto take = [&](uint32_t bits, float (&f)[E]) {
      if constexpr (E == 2) {
        f[0] = __uint_as_float(bits << 16);
        f[1] = __uint_as_float(bits & 0xFFFF0000u);
      } else {
        f[0] = __uint_as_float(bits);
      }
    };
    if (held) {
      take(reinterpret_cast<const uint32_t*>(meta)[at], mn);
      take(reinterpret_cast<const uint32_t*>(meta + D)[at], mx);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) mn[e] = mx[e] = __uint_as_float(0x7FC00000u);
    }
    for (int t = lo; t < hi; ++t) {
      if (!((ok >> t) & 1)) continue;   // (uniform)
      float f[E];
      take(reinterpret_cast<const uint32_t*>(rows + t * D)[at], f);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        mn[e] = fminf(mn[e], f[e]);
        mx[e] = fmaxf(mx[e], f[e]);
      }
    }
    const auto give = [&](const float (&f)[E]) -> uint32_t {
      if constexpr (E == 2)
        return (__float_as_uint(f[0]) >> 16) | (__float_as_uint(f[1]) & 0xFFFF0000u);
      else
        return __float_as_uint(f[0]);
    };
    reinterpret_cast<uint32_t*>(meta)[at] = give(mn);
    reinterpret_cast<uint32_t*>(meta + D)[at] = give(mx);
  }
}

}  // namespace losa
