// Position rotation of queries and keys, and new tokens' way into the pages of a cache.
//
// Both are bound by the bytes they move: a rotated channel is 14 vector operations (see turned) on two bytes in and two out, half of the time
// that the bytes take.
#include <algorithm>

#include "losa_device.h"
#include "losa_internal.h"
#include "new_tokens.h"

namespace losa {

// ---- rotation alone.  A thread has one unit (two 16-byte chunks) of a head of a token; a token's heads are neighbours, so that a workgroup reads
// and writes whole stretches and a token's angles are asked for by the same compute unit.  8191 tokens of 40 heads of 128 floats: 61.5 us, 5.5 TB/s
// (a large copy reaches 5.1); a head's tokens as neighbours 80, rows past the caches 67, those and results 74, measured in turn.
struct RotateSide {
  const void* x;
  void* y;
  long x_stride, y_stride;
  int heads;
};
constexpr int kRotateTokens = 4096;   // of one blockIdx.y: their units are counted in 32 bits
template <typename T>
__global__ __launch_bounds__(256) void rotate_kernel(Rotation rot, const int32_t* __restrict__ positions, int tokens, int d, RotateSide q,
                                                     RotateSide k) {
  constexpr int V = Vec16<T>::n;
  const uint32_t units = d / (2 * V), heads = q.heads + k.heads;   // units: 4 .. 16
  const uint32_t item = blockIdx.x * 256 + threadIdx.x, row = item / units;
  const long t = (long)blockIdx.y * kRotateTokens + row / heads;
  if (row / heads >= kRotateTokens || t >= tokens) return;
  const int h = (int)(row % heads), at = positions[t];
  const Unit u = unit_of<V>((int)(item % units), rot.rotary, rot.pairs);
  const T* from = h < q.heads ? (const T*)q.x + t * q.x_stride + h * d : (const T*)k.x + t * k.x_stride + (h - q.heads) * d;
  uint4 a = *reinterpret_cast<const uint4*>(from + u.first), b = *reinterpret_cast<const uint4*>(from + u.second);
  if ((unsigned)at >= (unsigned)rot.max_positions) return;
  if (u.angle >= 0) {
    float c[V], s[V], fa[V], fb[V];
    const float* angles = rot.table + (size_t)at * rot.rotary + u.angle;
    load_floats<V>(angles, c);
    load_floats<V>(angles + rot.rotary / 2, s);
    widen16(a, fa, T());
    widen16(b, fb, T());
    turn_unit<V>(fa, fb, c, s, rot.pairs);
    a = round16(fa, T());
    b = round16(fb, T());
  }
  T* to = h < q.heads ? (T*)q.y + t * q.y_stride + h * d : (T*)k.y + t * k.y_stride + (h - q.heads) * d;
  *reinterpret_cast<uint4*>(to + u.first) = a;
  *reinterpret_cast<uint4*>(to + u.second) = b;
}

template <typename T>
static hipError_t launch_rotate_t(hipStream_t st, int d, const Rotation& rot, const int32_t* positions, int tokens, const RotateSide& q,
                                  const RotateSide& k) {
  const long items = (long)std::min(tokens, kRotateTokens) * (q.heads + k.heads) * (d / (2 * Vec16<T>::n));
  rotate_kernel<T><<<dim3((unsigned)((items + 255) / 256), (tokens + kRotateTokens - 1) / kRotateTokens), 256, 0, st>>>(rot, positions, tokens, d, q, k);
  return hipGetLastError();
}

hipError_t launch_rotate(hipStream_t st, int dtype, int d, const Rotation& rot, const int32_t* positions, int tokens, const void* q,
                         long q_stride, void* q_out, long q_out_stride, int q_heads, const void* k, long k_stride, void* k_out,
                         long k_out_stride, int k_heads) {
  const RotateSide qs = {q, q_out, q_stride, q_out_stride, q ? q_heads : 0}, ks = {k, k_out, k_stride, k_out_stride, k ? k_heads : 0};
  return dtype == LOSA_BF16 ? launch_rotate_t<bf16_t>(st, d, rot, positions, tokens, qs, ks)
                            : launch_rotate_t<float>(st, d, rot, positions, tokens, qs, ks);
}

// ---- new tokens into pages.  A wavefront has 16 tokens of a page and KV head, a workgroup four of them: a page of four heads, or of two
// where a page has 32 tokens.  All of a wavefront's reads leave before it uses any.
//
// Keys: d / (2 V) lanes per token, a unit each, turned where there is a rotation, written as they lie (token-major) and left in
// LDS, out of which a lane takes the bounds of its channels.
// Values: a lane has one dword of channels and reads eight tokens of it (a token's row is one contiguous read of the wavefront), which makes
// each channel's eight tokens 16 or 32 contiguous bytes of the channel-major page.  Where all 16 rows get a token they are written
// in order by way of LDS (38.4 against 41.4 us at the size below), else one by one: rows that get no token are not written.
// 32768 tokens of 4 heads of 128 bfloat16, keys rotated: 32 us, 4.8 TB/s (a copy of as many bytes reaches 5.0); without reading rows once, 37.
template <typename T, int D, int GP>
__global__ __launch_bounds__(256) void append_kernel(KvView kv, Shape sh, NewTokens in, Rotation rot) {
  constexpr int V = Vec16<T>::n, LPT = D / (2 * V), TPP = 64 / LPT, PASSES = 16 / TPP;   // keys: lanes per token, tokens per pass
  constexpr int HALVES = GP / 16, HEADS = 4 / HALVES;
  constexpr int E = 4 / sizeof(T), WPT = D / E, LPR = WPT < 64 ? WPT : 64;   // values: channels of a dword, dwords and lanes per token
  constexpr int SETS = 64 / LPR, OCTETS = 2 / SETS, COLS = WPT / LPR;        // octets of tokens side by side, one after the other; dwords of a lane per token
  __shared__ __attribute__((aligned(16))) T lds[HEADS][GP * D];
  __shared__ uint32_t arrived[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = wave % HALVES, hl = wave / HALVES, h = blockIdx.z * HEADS + hl, head = min(h, sh.Hkv - 1);
  const Fill f = fill_of(kv, sh, in.indptr, in.num_tokens, blockIdx.y, blockIdx.x);
  if (f.hi <= f.lo) return;
  const int phys = kv.page_indices[f.entry];
  const Unit u = unit_of<V>(lane % LPT, rot.table ? rot.rotary : 0, rot.pairs);

  // reads: rows that are not there read one that is
  const int most = f.hi - f.lo - 1;
  uint4 a[PASSES], b[PASSES];
  int row[PASSES];
  bool ok[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    row[i] = 16 * half + i * TPP + lane / LPT;
    ok[i] = row[i] >= f.lo && row[i] < f.hi && h < sh.Hkv;
    const T* from = (const T*)in.k + (size_t)(f.source + max(0, min(row[i] - f.lo, most))) * in.k_stride + head * D;
    a[i] = load_once(from + u.first);
    b[i] = load_once(from + u.second);
  }
  const int col = lane % LPR, set = lane / LPR;
  uint32_t x[OCTETS][COLS][8];
#pragma unroll
  for (int o = 0; o < OCTETS; ++o)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = 16 * half + 8 * (o * SETS + set) + e;
      const T* from = (const T*)in.v + (size_t)(f.source + max(0, min(t - f.lo, most))) * in.v_stride + head * D;
#pragma unroll
      for (int w = 0; w < COLS; ++w) x[o][w][e] = load_once(reinterpret_cast<const uint32_t*>(from) + w * 64 + col);
    }
  float c[PASSES][V], s[PASSES][V];
  if (rot.table) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int new_row = max(0, min(row[i] - f.lo, most));
      const int at = in.positions ? in.positions[f.source + new_row] : f.slot + new_row;
      const bool known = (unsigned)at < (unsigned)rot.max_positions;
      ok[i] = ok[i] && known;
      const float* angles = rot.table + (size_t)(known ? at : 0) * rot.rotary + max(u.angle, 0);
      load_floats<V>(angles, c[i]);
      load_floats<V>(angles + rot.rotary / 2, s[i]);
    }
  }
  if ((unsigned)phys >= (unsigned)kv.num_pages) return;
  const size_t tile = (size_t)phys * sh.Hkv + head;

  uint32_t there = 0;   // rows of these 16 that hold a token now
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const unsigned long long who = __ballot(ok[i]);
#pragma unroll
    for (int t = 0; t < TPP; ++t) there |= (uint32_t)((who >> (t * LPT)) & 1) << (i * TPP + t);
  }

  T* const mine = lds[hl] + 16 * half * D;   // this wavefront's own
  T* const vpage = (T*)kv.v_pages + tile * (GP * D) + 16 * half;
  constexpr int CHUNKS = sizeof(T);          // 16-byte chunks of a channel's 16 tokens
#pragma unroll
  for (int o = 0; o < OCTETS; ++o) {
    const int octet = o * SETS + set;
    const uint32_t mask = (there >> (8 * octet)) & 0xFFu;
#pragma unroll
    for (int w = 0; w < COLS; ++w) {
      const uint32_t(&y)[8] = x[o][w];
      const int channel = (w * 64 + col) * E;
      if (there == 0xFFFFu) {
        uint4* dst = reinterpret_cast<uint4*>(mine) + channel * CHUNKS + octet * (CHUNKS / 2);
        if constexpr (E == 2) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t pick = e ? 0x07060302u : 0x05040100u;
            dst[e * CHUNKS] = make_uint4(__builtin_amdgcn_perm(y[1], y[0], pick), __builtin_amdgcn_perm(y[3], y[2], pick),
                                         __builtin_amdgcn_perm(y[5], y[4], pick), __builtin_amdgcn_perm(y[7], y[6], pick));
          }
        } else {
          dst[0] = make_uint4(y[0], y[1], y[2], y[3]);
          dst[1] = make_uint4(y[4], y[5], y[6], y[7]);
        }
      } else {
        T* dst = vpage + channel * GP + 8 * octet;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if ((mask >> e) & 1) {
            if constexpr (E == 2) {
              dst[e] = (T)(y[e] & 0xFFFFu);
              dst[GP + e] = (T)(y[e] >> 16);
            } else {
              reinterpret_cast<uint32_t*>(dst)[e] = y[e];
            }
          }
      }
    }
  }
  if (there == 0xFFFFu) {
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < D * CHUNKS / 64; ++i) {
      const int id = i * 64 + lane;
      *reinterpret_cast<uint4*>(vpage + (id / CHUNKS) * GP + (id % CHUNKS) * (16 / CHUNKS)) = reinterpret_cast<const uint4*>(mine)[id];
    }
    wave_lds_fence();   // the keys go there next
  }

#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    if (rot.table && u.angle >= 0) {
      float fa[V], fb[V];
      widen16(a[i], fa, T());
      widen16(b[i], fb, T());
      turn_unit<V>(fa, fb, c[i], s[i], rot.pairs);
      a[i] = round16(fa, T());
      b[i] = round16(fb, T());
    }
    if (ok[i]) {
      T* dst = (T*)kv.k_pages + tile * (GP * D) + row[i] * D;
      *reinterpret_cast<uint4*>(dst + u.first) = a[i];
      *reinterpret_cast<uint4*>(dst + u.second) = b[i];
      if (kv.meta) {
        *reinterpret_cast<uint4*>(lds[hl] + row[i] * D + u.first) = a[i];
        *reinterpret_cast<uint4*>(lds[hl] + row[i] * D + u.second) = b[i];
      }
    }
  }
  if (!kv.meta) return;
  there <<= 16 * half;
  if constexpr (HALVES == 1) {
    wave_lds_fence();
  } else {
    if (lane == 0) arrived[wave] = there;
    __syncthreads();
    there = arrived[hl * 2] | arrived[hl * 2 + 1];
    if (half) return;
  }
  if (h < sh.Hkv) bounds_from_lds<T, D>(lds[hl], there, f.lo, f.hi, f.lo > 0, (T*)kv.meta + tile * 2 * D, lane);
}

hipError_t launch_append(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, int batch, int max_new, const NewTokens& in,
                         const Rotation& rot) {
  const int per_group = sh.g == 32 ? 2 : 4;
  const dim3 grid(pages_touched(max_new, sh.g), batch, (sh.Hkv + per_group - 1) / per_group);
  auto launch = [&](auto kern) {
    kern<<<grid, 256, 0, st>>>(kv, sh, in, rot);
    return hipGetLastError();
  };
  if (dtype == LOSA_BF16) {
    if (sh.d == 128) return sh.g == 16 ? launch(append_kernel<bf16_t, 128, 16>) : launch(append_kernel<bf16_t, 128, 32>);
    return sh.g == 16 ? launch(append_kernel<bf16_t, 64, 16>) : launch(append_kernel<bf16_t, 64, 32>);
  }
  if (sh.d == 128) return sh.g == 16 ? launch(append_kernel<float, 128, 16>) : launch(append_kernel<float, 128, 32>);
  return sh.g == 16 ? launch(append_kernel<float, 64, 16>) : launch(append_kernel<float, 64, 32>);
}

}  // namespace losa
