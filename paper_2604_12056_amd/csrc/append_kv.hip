// Position rotation of queries and keys, and new tokens' way into the pages of a cache.
//
// Both only move bytes: a rotated channel is six operations of arithmetic on two bytes in and two out.
#include "losa_device.h"
#include "losa_internal.h"
#include "new_tokens.h"

namespace losa {

// ---- rotation alone.  A thread has one unit (two 16-byte chunks) of HPT heads of a token: the angles are read once for them,
// and the loads of all heads leave together.
struct RotateSide {
  const void* x;
  void* y;
  long x_stride, y_stride;
  int heads;
};
template <typename T, int HPT>
__global__ __launch_bounds__(256) void rotate_kernel(Rotation rot, const int32_t* __restrict__ positions, int tokens, int d, RotateSide q,
                                                     RotateSide k) {
  constexpr int V = Vec16<T>::n;
  const int units = d / (2 * V);   // a power of two: 4 .. 16
  const long item = (long)blockIdx.x * 256 + threadIdx.x;
  const long t = item / units;
  const Unit u = unit_of<V>((int)(item % units), rot.rotary, rot.pairs);
  if (t >= tokens) return;
  const int at = positions[t], head0 = blockIdx.y * HPT, heads = q.heads + k.heads;
  uint4 a[HPT], b[HPT];
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const int h = min(head0 + i, heads - 1);
    const T* row = h < q.heads ? (const T*)q.x + t * q.x_stride + h * d : (const T*)k.x + t * k.x_stride + (h - q.heads) * d;
    a[i] = *reinterpret_cast<const uint4*>(row + u.first);
    b[i] = *reinterpret_cast<const uint4*>(row + u.second);
  }
  if ((unsigned)at >= (unsigned)rot.max_positions) return;
  float c[V], s[V];
  const float* angles = rot.table + (size_t)at * rot.rotary + max(u.angle, 0);
  load_floats<V>(angles, c);
  load_floats<V>(angles + rot.rotary / 2, s);
#pragma unroll
  for (int i = 0; i < HPT; ++i) {
    const int h = head0 + i;
    if (h >= heads) return;
    if (u.angle >= 0) {
      float fa[V], fb[V];
      widen16(a[i], fa, T());
      widen16(b[i], fb, T());
      turn_unit<V>(fa, fb, c, s, rot.pairs);
      a[i] = round16(fa, T());
      b[i] = round16(fb, T());
    }
    T* row = h < q.heads ? (T*)q.y + t * q.y_stride + h * d : (T*)k.y + t * k.y_stride + (h - q.heads) * d;
    *reinterpret_cast<uint4*>(row + u.first) = a[i];
    *reinterpret_cast<uint4*>(row + u.second) = b[i];
  }
}

template <typename T>
static hipError_t launch_rotate_t(hipStream_t st, int d, const Rotation& rot, const int32_t* positions, int tokens, const RotateSide& q,
                                  const RotateSide& k) {
  const long items = (long)tokens * (d / (2 * Vec16<T>::n));
  const int heads = q.heads + k.heads;
  const unsigned groups = (unsigned)((items + 255) / 256);
  rotate_kernel<T, 1><<<dim3(groups, heads), 256, 0, st>>>(rot, positions, tokens, d, q, k);
  return hipGetLastError();
}

hipError_t launch_rotate(hipStream_t st, int dtype, int d, const Rotation& rot, const int32_t* positions, int tokens, const void* q,
                         long q_stride, void* q_out, long q_out_stride, int q_heads, const void* k, long k_stride, void* k_out,
                         long k_out_stride, int k_heads) {
  const RotateSide qs = {q, q_out, q_stride, q_out_stride, q ? q_heads : 0}, ks = {k, k_out, k_stride, k_out_stride, k ? k_heads : 0};
  return dtype == LOSA_BF16 ? launch_rotate_t<bf16_t>(st, d, rot, positions, tokens, qs, ks)
                            : launch_rotate_t<float>(st, d, rot, positions, tokens, qs, ks);
}

// ---- new tokens into pages.  A workgroup fills one page, each of its four wavefronts every fourth KV head of it.
//
// Keys: d / (2 V) lanes per token, a unit each, turned where there is a rotation, written as they lie (token-major) and left in
// LDS, out of which a lane takes the bounds of its channels.
// Values: a lane has one dword of channels, reads eight tokens of it (a token's row is one contiguous read of the wavefront) and
// writes each channel's eight tokens as 16 or 32 contiguous bytes of the channel-major page: the transposition costs no
// LDS and no lane exchange.  Rows that get no token are not written.
template <typename T, int D, int GP>
__global__ __launch_bounds__(256) void append_kernel(KvView kv, Shape sh, NewTokens in, Rotation rot) {
  constexpr int V = Vec16<T>::n, LPT = D / (2 * V), TPP = 64 / LPT;   // lanes per token, tokens per pass
  __shared__ __attribute__((aligned(16))) T lds[4][GP * D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Fill f = fill_of(kv, sh, in.indptr, in.num_tokens, blockIdx.y, blockIdx.x);
  if (f.hi <= f.lo) return;
  const int phys = kv.page_indices[f.entry];
  if ((unsigned)phys >= (unsigned)kv.num_pages) return;
  const Unit u = unit_of<V>(lane % LPT, rot.table ? rot.rotary : 0, rot.pairs);
  for (int j = wave; j < sh.Hkv; j += 4) {
    const size_t tile = (size_t)phys * sh.Hkv + j;
    uint32_t there = 0;   // rows that hold a token now
    T* rows = lds[wave];
#pragma unroll
    for (int pass = 0; pass < GP / TPP; ++pass) {
      const int t = pass * TPP + lane / LPT;
      const bool mine = t >= f.lo && t < f.hi;
      const int src = f.source + (t - f.lo);
      int at = 0;
      if (mine && rot.table) at = in.positions ? in.positions[src] : f.slot + (t - f.lo);
      const bool ok = mine && (!rot.table || (unsigned)at < (unsigned)rot.max_positions);
      if (ok) {
        const T* row = (const T*)in.k + (size_t)src * in.k_stride + j * D;
        uint4 a = *reinterpret_cast<const uint4*>(row + u.first), b = *reinterpret_cast<const uint4*>(row + u.second);
        if (u.angle >= 0) {
          float fa[V], fb[V], c[V], s[V];
          const float* angles = rot.table + (size_t)at * rot.rotary + u.angle;
          load_floats<V>(angles, c);
          load_floats<V>(angles + rot.rotary / 2, s);
          widen16(a, fa, T());
          widen16(b, fb, T());
          turn_unit<V>(fa, fb, c, s, rot.pairs);
          a = round16(fa, T());
          b = round16(fb, T());
        }
        T* dst = (T*)kv.k_pages + tile * (GP * D) + t * D;
        *reinterpret_cast<uint4*>(dst + u.first) = a;
        *reinterpret_cast<uint4*>(dst + u.second) = b;
        *reinterpret_cast<uint4*>(rows + t * D + u.first) = a;
        *reinterpret_cast<uint4*>(rows + t * D + u.second) = b;
      }
      const unsigned long long who = __ballot(ok);
#pragma unroll
      for (int i = 0; i < TPP; ++i) there |= (uint32_t)((who >> (i * LPT)) & 1) << (pass * TPP + i);
    }
    wave_lds_fence();
    if (kv.meta) bounds_from_lds<T, D>(rows, there, f.lo, f.hi, f.lo > 0, (T*)kv.meta + tile * 2 * D, lane);

    // values: E channels of a lane, eight tokens a time
    constexpr int E = 4 / sizeof(T), WPT = D / E;   // dwords per token
    constexpr int SETS = WPT >= 64 ? 1 : 64 / WPT;  // octets of tokens side by side
    const T* vrow = (const T*)in.v + (size_t)f.source * in.v_stride + j * D;
    T* vpage = (T*)kv.v_pages + tile * (GP * D);
    for (int w = 0; w < WPT; w += 64) {
      const int at = WPT >= 64 ? w + lane : lane % WPT;
#pragma unroll
      for (int o = 0; o < GP / 8; o += SETS) {
        const int t0 = 8 * (o + (WPT >= 64 ? 0 : lane / WPT));
        const uint32_t mask = (there >> t0) & 0xFFu;
        uint32_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          x[i] = ((mask >> i) & 1) ? reinterpret_cast<const uint32_t*>(vrow + (long)(t0 + i - f.lo) * in.v_stride)[at] : 0u;
        if constexpr (E == 2) {
          if (mask == 0xFFu) {
            uint4 lo, hi;
            lo.x = __builtin_amdgcn_perm(x[1], x[0], 0x05040100u);
            lo.y = __builtin_amdgcn_perm(x[3], x[2], 0x05040100u);
            lo.z = __builtin_amdgcn_perm(x[5], x[4], 0x05040100u);
            lo.w = __builtin_amdgcn_perm(x[7], x[6], 0x05040100u);
            hi.x = __builtin_amdgcn_perm(x[1], x[0], 0x07060302u);
            hi.y = __builtin_amdgcn_perm(x[3], x[2], 0x07060302u);
            hi.z = __builtin_amdgcn_perm(x[5], x[4], 0x07060302u);
            hi.w = __builtin_amdgcn_perm(x[7], x[6], 0x07060302u);
            *reinterpret_cast<uint4*>(vpage + (2 * at) * GP + t0) = lo;
            *reinterpret_cast<uint4*>(vpage + (2 * at + 1) * GP + t0) = hi;
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if ((mask >> i) & 1) {
                vpage[(2 * at) * GP + t0 + i] = (T)(x[i] & 0xFFFFu);
                vpage[(2 * at + 1) * GP + t0 + i] = (T)(x[i] >> 16);
              }
          }
        } else {
          if (mask == 0xFFu) {
            uint4* dst = reinterpret_cast<uint4*>(vpage + at * GP + t0);
            dst[0] = make_uint4(x[0], x[1], x[2], x[3]);
            dst[1] = make_uint4(x[4], x[5], x[6], x[7]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if ((mask >> i) & 1) reinterpret_cast<uint32_t*>(vpage)[at * GP + t0 + i] = x[i];
          }
        }
      }
    }
    wave_lds_fence();   // the next head's keys go where this one's bounds were read
  }
}

hipError_t launch_append(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, int batch, int max_new, const NewTokens& in,
                         const Rotation& rot) {
  const dim3 grid(pages_touched(max_new, sh.g), batch);
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
