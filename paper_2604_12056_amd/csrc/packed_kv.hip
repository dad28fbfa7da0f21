// New tokens into a 4-bit cache, and tokens out of it.
//
// A lane has one token's group of 32 channels: what a scale is made of, and the 16 bytes that come of it.  With 128 channels the
// 64 lanes are the sixteen tokens of a page or of half of one, and 16 bytes a lane are what a page-head tile holds in lane order.
// A workgroup has one page, each of its four wavefronts every fourth KV head of it.
#include "losa_device.h"
#include "losa_internal.h"
#include "new_tokens.h"
#include "packed_format.h"

namespace losa {

// 32 channels of a row, widened.
template <typename T>
__device__ __forceinline__ void load32(const T* p, float (&x)[32]) {
  constexpr int V = Vec16<T>::n;
#pragma unroll
  for (int e = 0; e < 32; e += V) {
    float f[V];
    widen16(*reinterpret_cast<const uint4*>(p + e), f, T());
#pragma unroll
    for (int i = 0; i < V; ++i) x[e + i] = f[i];
  }
}

// Channels c .. c + 31 of `row`, turned by the angles of one position (`angles`: cosines, then sines) and rounded to T, as a cache of T would
// hold them.  Eight channels are turned by a whole half or not at all, as rotary_dim is a multiple of 16.
template <typename T>
__device__ __forceinline__ void load32_turned(const T* row, int c, const float* angles, const Rotation& rot, float (&x)[32]) {
  load32<T>(row + c, x);
  const int half = rot.rotary / 2;
#pragma unroll
  for (int e = 0; e < 32; e += 8) {
    const int ch = c + e;
    if (ch >= rot.rotary) continue;
    float y[8];
    if (rot.pairs) {
      float cs[4], sn[4];
      load_floats<4>(angles + ch / 2, cs);
      load_floats<4>(angles + half + ch / 2, sn);
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        y[i] = turned(x[e + i], cs[i / 2], x[e + i + 1], -sn[i / 2]);
        y[i + 1] = turned(x[e + i + 1], cs[i / 2], x[e + i], sn[i / 2]);
      }
    } else {
      const bool second = ch >= half;
      const int at = second ? ch - half : ch;
      float cs[8], sn[8], other[8];
      load_floats<8>(angles + at, cs);
      load_floats<8>(angles + half + at, sn);
      constexpr int V = Vec16<T>::n;
#pragma unroll
      for (int i = 0; i < 8; i += V) {
        float f[V];
        widen16(*reinterpret_cast<const uint4*>(row + (second ? at : at + half) + i), f, T());
#pragma unroll
        for (int k = 0; k < V; ++k) other[i + k] = f[k];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = turned(x[e + i], cs[i], other[i], second ? sn[i] : -sn[i]);
    }
    constexpr int V = Vec16<T>::n;
#pragma unroll
    for (int i = 0; i < 8; i += V) {
      float f[V];
#pragma unroll
      for (int k = 0; k < V; ++k) f[k] = y[i + k];
      widen16(round16(f, T()), f, T());
#pragma unroll
      for (int k = 0; k < V; ++k) x[e + i + k] = f[k];
    }
  }
}

// Codes of 32 numbers: byte i of the result holds x[FIRST i] and x[FIRST i + SECOND] (keys: neighbours; values: 16 apart).
template <int FIRST, int SECOND>
__device__ __forceinline__ uint4 codes_of(const float (&x)[32], int byte) {
  const float scale = power_of(byte);
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t c = 0;
    c = put_codes<0>(c, x[FIRST * (4 * k)], x[FIRST * (4 * k) + SECOND], scale);
    c = put_codes<1>(c, x[FIRST * (4 * k + 1)], x[FIRST * (4 * k + 1) + SECOND], scale);
    c = put_codes<2>(c, x[FIRST * (4 * k + 2)], x[FIRST * (4 * k + 2) + SECOND], scale);
    c = put_codes<3>(c, x[FIRST * (4 * k + 3)], x[FIRST * (4 * k + 3) + SECOND], scale);
    w[k] = byte == kScaleNaN ? 0u : c;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T, int D, int GP>
__global__ __launch_bounds__(256) void append_packed_kernel(KvView kv, Shape sh, NewTokens in, Rotation rot, PackedView out) {
  constexpr int J = D / 32, TPP = 64 / J < GP ? 64 / J : GP;   // groups per token, tokens per pass
  __shared__ __attribute__((aligned(16))) T lds[4][GP * D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Fill f = fill_of(kv, sh, in.indptr, in.num_tokens, blockIdx.y, blockIdx.x);
  if (f.hi <= f.lo) return;
  const int j = lane % J;
  for (int h = wave; h < sh.Hkv; h += 4) {
    const size_t tile = (size_t)f.phys * sh.Hkv + h;
    uint8_t* scales = out.scales + tile * (2 * GP * J);
    uint8_t* vcodes = out.v + tile * (GP * D / 2);
    uint32_t there = 0;
#pragma unroll
    for (int pass = 0; pass < GP / TPP; ++pass) {
      const int t = pass * TPP + lane / J;
      const bool mine = t >= f.lo && t < f.hi;   // (lanes past the page's rows have none)
      const int src = f.source + (t - f.lo);
      int at = 0;
      if (mine && rot.table) at = in.positions ? in.positions[src] : f.slot + (t - f.lo);
      const bool ok = mine && (!rot.table || (unsigned)at < (unsigned)rot.max_positions);
      if (ok) {
        float x[32];
        const T* row = (const T*)in.k + (size_t)src * in.k_stride + h * D;
        if (rot.table)
          load32_turned<T>(row, j * 32, rot.table + (size_t)at * rot.rotary, rot, x);
        else
          load32<T>(row + j * 32, x);
        const int byte = scale_byte(largest(x), kKeyScaleMin, kKeyScaleMax);
        const uint4 c = codes_of<2, 1>(x, byte);
        *reinterpret_cast<uint4*>(out.k + tile * (GP * D / 2) + t * (D / 2) + j * 16) = c;
        scales[t * J + j] = (uint8_t)byte;
        // the numbers that now stand for the key, for the page's bounds
        const float scale = power_of(byte);
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint4 n = make_uint4(codes_to_bf16<0>(w[k], scale), codes_to_bf16<1>(w[k], scale), codes_to_bf16<2>(w[k], scale),
                                     codes_to_bf16<3>(w[k], scale));
          uint4* dst = reinterpret_cast<uint4*>(&lds[wave][t * D + j * 32 + 8 * k]);
          if constexpr (sizeof(T) == 2) {
            dst[0] = n;
          } else {
            dst[0] = make_uint4(n.x << 16, n.x & 0xFFFF0000u, n.y << 16, n.y & 0xFFFF0000u);
            dst[1] = make_uint4(n.z << 16, n.z & 0xFFFF0000u, n.w << 16, n.w & 0xFFFF0000u);
          }
        }
        load32<T>((const T*)in.v + (size_t)src * in.v_stride + h * D + j * 32, x);
        const int vbyte = scale_byte(largest(x), kValueScaleMin, kValueScaleMax);
        const uint4 vc = codes_of<1, 16>(x, vbyte);
        scales[GP * J + t * J + j] = (uint8_t)vbyte;
        const uint32_t vw[4] = {vc.x, vc.y, vc.z, vc.w};
        uint8_t* dst = vcodes + ((t >> 2) * 16 * J + j) * 4 + (t & 3);
#pragma unroll
        for (int r = 0; r < 16; ++r) dst[r * J * 4] = (uint8_t)(vw[r / 4] >> (8 * (r % 4)));
      }
      const unsigned long long who = __ballot(ok);
#pragma unroll
      for (int i = 0; i < TPP; ++i) there |= (uint32_t)((who >> (i * J)) & 1) << (pass * TPP + i);
    }
    wave_lds_fence();
    if (kv.meta) bounds_from_lds<T, D>(lds[wave], there, f.lo, f.hi, f.lo > 0, (T*)kv.meta + tile * 2 * D, lane);
    wave_lds_fence();   // the next head's keys go where this one's bounds were read
  }
}

// 32 numbers, as dwords of two bfloat16 each, to a row of T.
template <typename T>
__device__ __forceinline__ void store32(T* dst, const uint32_t (&w)[16]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint4* to = reinterpret_cast<uint4*>(dst + 8 * k);
    if constexpr (sizeof(T) == 2) {
      to[0] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    } else {
      to[0] = make_uint4(w[4 * k] << 16, w[4 * k] & 0xFFFF0000u, w[4 * k + 1] << 16, w[4 * k + 1] & 0xFFFF0000u);
      to[1] = make_uint4(w[4 * k + 2] << 16, w[4 * k + 2] & 0xFFFF0000u, w[4 * k + 3] << 16, w[4 * k + 3] & 0xFFFF0000u);
    }
  }
}

template <typename T, int D, int GP>
__global__ __launch_bounds__(256) void read_packed_kernel(KvView kv, Shape sh, const int32_t* indptr, int num_tokens, PackedView in,
                                                          T* __restrict__ k_out, T* __restrict__ v_out) {
  constexpr int J = D / 32, TPP = 64 / J < GP ? 64 / J : GP;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Fill f = fill_of(kv, sh, indptr, num_tokens, blockIdx.y, blockIdx.x);
  if (f.hi <= f.lo) return;
  const int j = lane % J;
  for (int h = wave; h < sh.Hkv; h += 4) {
    const size_t tile = (size_t)f.phys * sh.Hkv + h;
    const uint8_t* scales = in.scales + tile * (2 * GP * J);
#pragma unroll
    for (int pass = 0; pass < GP / TPP; ++pass) {
      const int t = pass * TPP + lane / J;
      if (t < f.lo || t >= f.hi) continue;
      const size_t row = ((size_t)(f.source + (t - f.lo)) * sh.Hkv + h) * D + j * 32;
      uint32_t w[16];
      if (k_out) {
        const uint4 c = *reinterpret_cast<const uint4*>(in.k + tile * (GP * D / 2) + t * (D / 2) + j * 16);
        const float scale = power_of(scales[t * J + j]);
        const uint32_t cw[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          w[4 * k] = codes_to_bf16<0>(cw[k], scale);
          w[4 * k + 1] = codes_to_bf16<1>(cw[k], scale);
          w[4 * k + 2] = codes_to_bf16<2>(cw[k], scale);
          w[4 * k + 3] = codes_to_bf16<3>(cw[k], scale);
        }
        store32<T>(k_out + row, w);
      }
      if (v_out) {
        const uint8_t* src = in.v + tile * (GP * D / 2) + ((t >> 2) * 16 * J + j) * 4 + (t & 3);
        const float scale = power_of(scales[GP * J + t * J + j]);
        uint32_t n[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) n[r] = src[r * J * 4];
#pragma unroll
        for (int r = 0; r < 16; ++r) n[r] = codes_to_bf16<0>(n[r], scale);   // channels r and 16 + r
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          w[r / 2] = __builtin_amdgcn_perm(n[r + 1], n[r], 0x05040100u);
          w[8 + r / 2] = __builtin_amdgcn_perm(n[r + 1], n[r], 0x07060302u);
        }
        store32<T>(v_out + row, w);
      }
    }
  }
}

// The instantiation of a kernel template for a context's type, head dimension and page size.
#define LOSA_OF_SHAPE(kernel)                                                                                                  \
  (dtype == LOSA_BF16 ? (sh.d == 128 ? (sh.g == 16 ? launch(kernel<bf16_t, 128, 16>) : launch(kernel<bf16_t, 128, 32>))         \
                                     : (sh.g == 16 ? launch(kernel<bf16_t, 64, 16>) : launch(kernel<bf16_t, 64, 32>)))          \
                      : (sh.d == 128 ? (sh.g == 16 ? launch(kernel<float, 128, 16>) : launch(kernel<float, 128, 32>))           \
                                     : (sh.g == 16 ? launch(kernel<float, 64, 16>) : launch(kernel<float, 64, 32>))))

hipError_t launch_append_packed(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, int batch, int max_new, const NewTokens& in,
                                const Rotation& rot, const PackedView& out) {
  const dim3 grid(pages_touched(max_new, sh.g), batch);
  auto launch = [&](auto kern) {
    kern<<<grid, 256, 0, st>>>(kv, sh, in, rot, out);
    return hipGetLastError();
  };
  return LOSA_OF_SHAPE(append_packed_kernel);
}

template <typename T>
static T* typed(void* p) { return static_cast<T*>(p); }

hipError_t launch_read_packed(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, int batch, int max_tokens, const int32_t* indptr,
                              int num_tokens, const PackedView& in, void* k_out, void* v_out) {
  const dim3 grid(pages_touched(max_tokens, sh.g), batch);
  auto go = [&](auto kern, auto* k, auto* v) {
    kern<<<grid, 256, 0, st>>>(kv, sh, indptr, num_tokens, in, k, v);
    return hipGetLastError();
  };
  if (dtype == LOSA_BF16) {
    auto launch = [&](auto kern) { return go(kern, typed<bf16_t>(k_out), typed<bf16_t>(v_out)); };
    if (sh.d == 128) return sh.g == 16 ? launch(read_packed_kernel<bf16_t, 128, 16>) : launch(read_packed_kernel<bf16_t, 128, 32>);
    return sh.g == 16 ? launch(read_packed_kernel<bf16_t, 64, 16>) : launch(read_packed_kernel<bf16_t, 64, 32>);
  }
  auto launch = [&](auto kern) { return go(kern, typed<float>(k_out), typed<float>(v_out)); };
  if (sh.d == 128) return sh.g == 16 ? launch(read_packed_kernel<float, 128, 16>) : launch(read_packed_kernel<float, 128, 32>);
  return sh.g == 16 ? launch(read_packed_kernel<float, 64, 16>) : launch(read_packed_kernel<float, 64, 32>);
}

}  // namespace losa
