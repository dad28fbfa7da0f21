// New tokens into a 4-bit cache, and tokens out of it.
//
// Bytes are all there is to them, so what matters is that a wavefront asks for all of its own before it uses any, and stores whole lines.
// Packing: two neighbouring lanes have a token's group of 32 channels, what a scale is made of; a wavefront has 1024 numbers of each of keys and values of a
// head (8 tokens of 128 channels, 16 of 64).  Reading: a lane has eight channels of a token, 16 bytes of what is written, a wavefront
// 16 tokens of a head.  A workgroup is four wavefronts of a page.
//
// Packing four sequences of 501 to 4093 tokens, 8 heads of 128, pages of 32, keys turned: 22 us for some 80 MB (16 at a large copy's rate); between
// them are the turning and the latency that five wavefronts a SIMD leave.  A whole group a lane, three wavefronts a SIMD: 27; values a byte at a time as well: 37.
// Rows read past the caches: 5 more, as a lane's bytes are several requests of one line.  Single tokens of 16 sequences: 5 us, four dependent trips to memory.
// Reading two sequences of 39012 tokens in all: 26.5 us, 5.3 TB/s (codes and rows past the caches: 29.1 without).
#include "losa_device.h"
#include "losa_internal.h"
#include "new_tokens.h"
#include "packed_format.h"

namespace losa {

// A lane's share of a group of 32 channels: eight of its first half and the same eight of its second, 16 further (c: the first).
// Neighbouring lanes have the two shares of a group.
constexpr int kShare = 16;
template <typename T>
struct RawShare {
  uint4 v[kShare / Vec16<T>::n];
};
template <typename T>
__device__ __forceinline__ RawShare<T> load_share(const T* p) {
  constexpr int V = Vec16<T>::n;
  RawShare<T> r;
#pragma unroll
  for (int i = 0; i < kShare / V; ++i) r.v[i] = *reinterpret_cast<const uint4*>(p + 16 * (i * V / 8) + i * V % 8);
  return r;
}
template <typename T>
__device__ __forceinline__ void widen_share(const RawShare<T>& r, float (&x)[kShare]) {
  constexpr int V = Vec16<T>::n;
#pragma unroll
  for (int i = 0; i < kShare / V; ++i) {
    float f[V];
    widen16(r.v[i], f, T());
#pragma unroll
    for (int e = 0; e < V; ++e) x[V * i + e] = f[e];
  }
}

// What turns a share: its angles and, halves style, the channels half a turn's width away.  Eight channels are turned by a whole
// half or not at all, as rotary_dim is a multiple of 16.  (No branch around a load: what does not turn, or has its pair at hand, loads something and
// does not use it.)
template <typename T>
struct TurnShare {
  float4 cs[4], sn[4];   // pairs style: every other one counts
  uint4 other[kShare / Vec16<T>::n];
};
template <typename T>
__device__ __forceinline__ void load_turn(const T* row, int c, const float* angles, const Rotation& rot, TurnShare<T>& t) {
  constexpr int V = Vec16<T>::n;
  const int half = rot.rotary / 2, next = rot.pairs ? 0 : 4;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int ch = c + 16 * i, in = ch < rot.rotary ? ch : 0;
    const int at = rot.pairs ? in / 2 : in < half ? in : in - half;
    const int away = rot.pairs || ch >= rot.rotary ? ch : ch < half ? ch + half : ch - half;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      t.cs[2 * i + k] = *reinterpret_cast<const float4*>(angles + at + next * k);
      t.sn[2 * i + k] = *reinterpret_cast<const float4*>(angles + half + at + next * k);
    }
#pragma unroll
    for (int k = 0; k < 8 / V; ++k) t.other[8 / V * i + k] = *reinterpret_cast<const uint4*>(row + away + V * k);
  }
}
// x, turned and rounded to T, as a cache of T would hold it.
template <typename T>
__device__ __forceinline__ void turn_share(float (&x)[kShare], int c, const Rotation& rot, const TurnShare<T>& t) {
  constexpr int V = Vec16<T>::n;
  const int half = rot.rotary / 2;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int ch = c + 16 * i;
    float y[8];
    if (rot.pairs) {
      const float4 c0 = t.cs[2 * i], s0 = t.sn[2 * i];
      const float cs[4] = {c0.x, c0.y, c0.z, c0.w}, sn[4] = {s0.x, s0.y, s0.z, s0.w};
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        y[e] = turned(x[8 * i + e], cs[e / 2], x[8 * i + e + 1], -sn[e / 2]);
        y[e + 1] = turned(x[8 * i + e + 1], cs[e / 2], x[8 * i + e], sn[e / 2]);
      }
    } else {
      const float4 c0 = t.cs[2 * i], c1 = t.cs[2 * i + 1], s0 = t.sn[2 * i], s1 = t.sn[2 * i + 1];
      const float cs[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, sn[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
      float other[8];
#pragma unroll
      for (int k = 0; k < 8 / V; ++k) {
        float f[V];
        widen16(t.other[8 / V * i + k], f, T());
#pragma unroll
        for (int e = 0; e < V; ++e) other[V * k + e] = f[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = turned(x[8 * i + e], cs[e], other[e], ch >= half ? sn[e] : -sn[e]);
    }
#pragma unroll
    for (int k = 0; k < 8; k += V) {
      float f[V];
#pragma unroll
      for (int e = 0; e < V; ++e) f[e] = y[k + e];
      widen16(round16(f, T()), f, T());
#pragma unroll
      for (int e = 0; e < V; ++e) x[8 * i + k + e] = ch < rot.rotary ? f[e] : x[8 * i + k + e];
    }
  }
}

// The largest magnitude of a group, both lanes' shares, NaN if one of its numbers is: in the bits of magnitudes, integers order as the numbers do and NaN is
// largest.
__device__ __forceinline__ float largest(const float (&x)[kShare]) {
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < kShare; ++e) m = max(m, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  return __uint_as_float(max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, true)));   // (lanes 1 0 3 2 of every four)
}

// A dword of codes: byte i holds a[FIRST i] and b[FIRST i].
template <int FIRST>
__device__ __forceinline__ uint32_t four_codes(const float* a, const float* b, int byte) {
  const float scale = power_of(byte);
  uint32_t c = 0;
  c = put_codes<0>(c, a[0], b[0], scale);
  c = put_codes<1>(c, a[FIRST], b[FIRST], scale);
  c = put_codes<2>(c, a[2 * FIRST], b[2 * FIRST], scale);
  c = put_codes<3>(c, a[3 * FIRST], b[3 * FIRST], scale);
  return byte == kScaleNaN ? 0u : c;
}

template <int D, int GP>
struct PageWork {   // of a workgroup
  static constexpr int LPT = D / kShare, TPP = 64 / LPT;        // lanes per token, tokens per wavefront
  static constexpr int PASSES = GP / TPP, HEADS = 4 / PASSES;   // wavefronts per page and head, heads per workgroup
};

template <typename T, int D, int GP>
__global__ __launch_bounds__(256) void append_packed_kernel(KvView kv, Shape sh, NewTokens in, Rotation rot, PackedView out) {
  typedef PageWork<D, GP> Work;
  constexpr int J = D / 32, LPT = Work::LPT, TPP = Work::TPP, kTile = GP * D / 2, kWaveBytes = TPP * D / 2;
  __shared__ __attribute__((aligned(16))) T keys[Work::HEADS][GP * D];   // the numbers that stand for the keys, for the page's bounds
  __shared__ __attribute__((aligned(16))) uint8_t codes[4][kWaveBytes];
  __shared__ uint32_t arrived[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pass = wave % Work::PASSES, hl = wave / Work::PASSES, h = blockIdx.z * Work::HEADS + hl;
  const int j = lane % LPT / 2, part = lane & 1, c = 32 * j + 8 * part;   // group, which of its lanes, first channel
  const Fill f = fill_of(kv, sh, in.indptr, in.num_tokens, blockIdx.y, blockIdx.x);
  if (f.hi <= f.lo) return;
  const int phys = kv.page_indices[f.entry];
  const int row = lane / LPT, t = pass * TPP + row;
  const bool mine = t >= f.lo && t < f.hi && h < sh.Hkv;
  const int at_row = max(f.lo, min(t, f.hi - 1)) - f.lo, src = f.source + at_row, head = min(h, sh.Hkv - 1);
  const T* const krow = (const T*)in.k + (size_t)src * in.k_stride + head * D;
  const RawShare<T> kraw = load_share<T>(krow + c), vraw = load_share<T>((const T*)in.v + (size_t)src * in.v_stride + head * D + c);
  bool ok = mine;
  TurnShare<T> turn;
  if (rot.table) {
    const int at = in.positions ? in.positions[src] : f.slot + at_row;
    ok = mine && (unsigned)at < (unsigned)rot.max_positions;
    load_turn<T>(krow, c, rot.table + (size_t)(ok ? at : 0) * rot.rotary, rot, turn);
  }
  if ((unsigned)phys >= (unsigned)kv.num_pages) return;
  const size_t tile = (size_t)phys * sh.Hkv + head;
  uint8_t* const scales = out.scales + tile * (2 * GP * J);
  uint8_t* const vcodes = out.v + tile * kTile + pass * kWaveBytes;

  float x[kShare];
  widen_share<T>(kraw, x);
  if (rot.table) turn_share<T>(x, c, rot, turn);
  const int byte = scale_byte(largest(x), kKeyScaleMin, kKeyScaleMax);
  if (ok) {
    if (part == 0) scales[t * J + j] = (uint8_t)byte;
#pragma unroll
    for (int i = 0; i < 2; ++i) {   // (neighbours are a byte)
      const uint32_t w = four_codes<2>(x + 8 * i, x + 8 * i + 1, byte);
      *reinterpret_cast<uint32_t*>(out.k + tile * kTile + t * (D / 2) + j * 16 + 8 * i + 4 * part) = w;
      if (kv.meta) {
        const float scale = power_of(byte);
        const uint4 n = make_uint4(codes_to_bf16<0>(w, scale), codes_to_bf16<1>(w, scale), codes_to_bf16<2>(w, scale), codes_to_bf16<3>(w, scale));
        uint4* dst = reinterpret_cast<uint4*>(&keys[hl][t * D + c + 16 * i]);
        if constexpr (sizeof(T) == 2) {
          dst[0] = n;
        } else {
          dst[0] = make_uint4(n.x << 16, n.x & 0xFFFF0000u, n.y << 16, n.y & 0xFFFF0000u);
          dst[1] = make_uint4(n.z << 16, n.z & 0xFFFF0000u, n.w << 16, n.w & 0xFFFF0000u);
        }
      }
    }
  }
  widen_share<T>(vraw, x);
  const int vbyte = scale_byte(largest(x), kValueScaleMin, kValueScaleMax);
  if (ok && part == 0) scales[GP * J + t * J + j] = (uint8_t)vbyte;
  // bytes 8 part .. 8 part + 7 of the group's 16: channels 16 apart
  const uint32_t vw[2] = {four_codes<1>(x, x + 8, vbyte), four_codes<1>(x + 4, x + 12, vbyte)};
  const unsigned long long who = __ballot(ok);
  const int place = ((row >> 2) * 16 * J + 8 * part * J + j) * 4 + (row & 3);   // of the first among this wavefront's bytes; the next is J 4 further
  if (who == ~0ull) {   // every byte of this wavefront's rows: in order by way of LDS
#pragma unroll
    for (int r = 0; r < 8; ++r) codes[wave][place + r * J * 4] = (uint8_t)(vw[r / 4] >> (8 * (r % 4)));
    wave_lds_fence();
    if (lane < kWaveBytes / 16) *reinterpret_cast<uint4*>(vcodes + lane * 16) = *reinterpret_cast<const uint4*>(&codes[wave][lane * 16]);
  } else if (ok) {
#pragma unroll
    for (int r = 0; r < 8; ++r) vcodes[place + r * J * 4] = (uint8_t)(vw[r / 4] >> (8 * (r % 4)));
  }
  if (!kv.meta) return;
  uint32_t there = 0;   // rows that hold a token now
#pragma unroll
  for (int i = 0; i < TPP; ++i) there |= (uint32_t)((who >> (i * LPT)) & 1) << (pass * TPP + i);
  if constexpr (Work::PASSES == 1) {
    wave_lds_fence();
  } else {
    if (lane == 0) arrived[wave] = there;
    __syncthreads();
    if (pass) return;
#pragma unroll
    for (int i = 1; i < Work::PASSES; ++i) there |= arrived[hl * Work::PASSES + i];
  }
  if (h < sh.Hkv) bounds_from_lds<T, D>(keys[hl], there, f.lo, f.hi, f.lo > 0, (T*)kv.meta + tile * 2 * D, lane);
}

// Eight numbers, as dwords of two bfloat16 each, to a row of T.
__device__ __forceinline__ void store8(bf16_t* dst, const uint4& n) { store_once(dst, n); }
__device__ __forceinline__ void store8(float* dst, const uint4& n) {
  store_once(dst, make_uint4(n.x << 16, n.x & 0xFFFF0000u, n.y << 16, n.y & 0xFFFF0000u));
  store_once(dst + 4, make_uint4(n.z << 16, n.z & 0xFFFF0000u, n.w << 16, n.w & 0xFFFF0000u));
}

template <typename T, int D, int GP>
__global__ __launch_bounds__(256) void read_packed_kernel(KvView kv, Shape sh, const int32_t* indptr, int num_tokens, PackedView in,
                                                          T* __restrict__ k_out, T* __restrict__ v_out) {
  constexpr int J = D / 32, LPT = D / 8, TPS = 64 / LPT, STEPS = 16 / TPS, kTile = GP * D / 2;   // lanes per token, tokens per step of 16
  constexpr int HALVES = GP / 16, HEADS = 4 / HALVES;
  __shared__ __attribute__((aligned(16))) uint8_t codes[4][16 * D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = wave % HALVES, h = blockIdx.z * HEADS + wave / HALVES;
  const Fill f = fill_of(kv, sh, indptr, num_tokens, blockIdx.y, blockIdx.x);
  if (f.hi <= f.lo || h >= sh.Hkv || f.hi <= 16 * part || f.lo >= 16 * part + 16) return;
  const int phys = kv.page_indices[f.entry];
  if ((unsigned)phys >= (unsigned)kv.num_pages) return;
  const size_t tile = (size_t)phys * sh.Hkv + h;
  const uint8_t* const scales = in.scales + tile * (2 * GP * J) + 16 * part * J;
  const int row = lane / LPT, c8 = lane % LPT, j = c8 / 4;   // this lane's token of a step, its eight channels, their group
  // everything that is read, of the whole half page
  uint32_t kc[STEPS];
  uint8_t ks[STEPS], vs[STEPS];
  uint4 vc = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    kc[i] = load_once(reinterpret_cast<const uint32_t*>(in.k + tile * kTile + (16 * part + i * TPS + row) * (D / 2) + c8 * 4));
    ks[i] = scales[(i * TPS + row) * J + j];
    vs[i] = scales[GP * J + (i * TPS + row) * J + j];
  }
  if (lane < D / 2) vc = load_once(in.v + tile * kTile + part * (8 * D) + lane * 16);
  if (lane < D / 2) *reinterpret_cast<uint4*>(&codes[wave][lane * 16]) = vc;
  wave_lds_fence();
  const uint32_t pick = (c8 & 2) ? 0x07060302u : 0x05040100u;   // the second half of a group's channels are the high codes
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    const int t = i * TPS + row, slot = 16 * part + t;
    const size_t to = ((size_t)(f.source + (slot - f.lo)) * sh.Hkv + h) * D + c8 * 8;
    const bool ok = slot >= f.lo && slot < f.hi;
    if (k_out && ok) {
      const float scale = power_of(ks[i]);
      store8(k_out + to, make_uint4(codes_to_bf16<0>(kc[i], scale), codes_to_bf16<1>(kc[i], scale), codes_to_bf16<2>(kc[i], scale),
                                    codes_to_bf16<3>(kc[i], scale)));
    }
    if (v_out && ok) {
      const float scale = power_of(vs[i]);
      const uint8_t* const from = &codes[wave][(((t >> 2) * 16 + (c8 & 1) * 8) * J + j) * 4 + (t & 3)];
      uint32_t n[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) n[r] = codes_to_bf16<0>(from[r * J * 4], scale);
      store8(v_out + to, make_uint4(__builtin_amdgcn_perm(n[1], n[0], pick), __builtin_amdgcn_perm(n[3], n[2], pick),
                                    __builtin_amdgcn_perm(n[5], n[4], pick), __builtin_amdgcn_perm(n[7], n[6], pick)));
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
  const int per_group = 4 * 1024 / (sh.g * sh.d);   // (PageWork::HEADS)
  const dim3 grid(pages_touched(max_new, sh.g), batch, (sh.Hkv + per_group - 1) / per_group);
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
  const int per_group = sh.g == 32 ? 2 : 4;
  const dim3 grid(pages_touched(max_tokens, sh.g), batch, (sh.Hkv + per_group - 1) / per_group);
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
