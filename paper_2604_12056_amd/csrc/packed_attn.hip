// Split-K paged prefix attention over a 4-bit cache (packed_format.h) on the gfx950 matrix cores.
//
// A wavefront has R*16 query rows of one KV head and walks 32-token tiles of the head's page list:
//
//   S^T = K_tile . Q^T      v_mfma_f32_16x16x32_bf16.  A lane reads 16 bytes of a 16-token subtile, a token's channels 32 qd .. 32 qd + 31
//                           (64 channels a head: 16 of them), all under one scale: sixteen conversions with that scale make the bfloat16
//                           operands of four products, exactly.  Product s contracts the channels 8 s .. 8 s + 7 of every such run; the
//                           query rows are laid out for that once.
//   O^T += V_tile^T . P^T   v_mfma_f32_16x16x32_f16.  S^T leaves the matrix core as the second operand (lane = query row, four tokens of
//                           each subtile).  The value operand wants the same tokens of one channel: a lane reads 16 bytes, four
//                           tokens' codes of the channels l16 + 16 i; a conversion gives two channels of a token under that token's scale, two
//                           permutations pair the tokens up.
//
// Numbers: keys are exact in bfloat16, values in half precision.  Probabilities enter the second product as a pair of halves, hi rounded to
// nearest and lo = p - hi rounded again (22 bits: error 2^-23 of p, against 2^-17 of a bfloat16 pair at the same cost); their sum is kept
// in float from the unrounded p.  Float mode splits a query into three bfloat16 terms, which hold its 24 bits.
// p is taken against a reference 2^7 below the row's maximum that may lag it by 2^8 (see kLag), so p < 2^15 is inside a half's
// range and what lo cannot hold is below 2^-25, 2^-32 of the largest p.
#include <math.h>

#include "losa_device.h"
#include "losa_internal.h"
#include "packed_format.h"

namespace losa {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef uint32_t u32x4v_t __attribute__((ext_vector_type(4)));

constexpr float kNegBig = -1.0e30f;   // finite stand-in for "no token seen yet"
constexpr float kLag = 8.0f, kHeadroom = 7.0f;

__device__ __forceinline__ float over_lane_groups_max(float v) {
  return __uint_as_float(across_rows(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ float over_lane_groups_sum(float v) {
  return __uint_as_float(across_rows(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// 16 or 8 bytes of codes per lane, as dwords
template <int N>
__device__ __forceinline__ void load_dwords(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const u32x4v_t x = __builtin_nontemporal_load(reinterpret_cast<const u32x4v_t*>(p));
    w[0] = x[0];
    w[1] = x[1];
    w[2] = x[2];
    w[3] = x[3];
  } else {
    typedef uint32_t u32x2v_t __attribute__((ext_vector_type(2)));
    const u32x2v_t x = __builtin_nontemporal_load(reinterpret_cast<const u32x2v_t*>(p));
    w[0] = x[0];
    w[1] = x[1];
  }
}

// Query rows row0 .. row0 + 16 R - 1 of a (sequence, KV head): what a workgroup does.
template <int D, int GP, int R, int NQ, int NBUF>
__device__ __forceinline__ void packed_attn_body(const KvView& kv, const Shape& sh, const AttnInputs& in, const PackedView& pk, int nchunk, int nrb,
                                                 int row0, const Partials& part, float scale_log2e, float* lds) {
  constexpr int KS = D / 32, NT = D / 16, J = D / 32, W = D / 32;   // products per score, channel tiles, groups, dwords a lane reads of a subtile
  constexpr int CPL = D / 4;                                        // channels of a token that a lane has
  constexpr int PPT = 32 / GP, TPR = 64 / PPT;                      // pages per tile, tiles per fetch of page entries
  constexpr int kTileBytes = GP * D / 2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, qd = lane >> 4;
  const int chunk = blockIdx.x, j = blockIdx.y / nrb, b = blockIdx.z, head = b * sh.Hkv + j;

  const Sequence seq = sequence(kv, sh, b);
  const int M = min(active_rows(in, kv, sh, b), min(sh.rows_max, part.rows));
  const int U = min(in.list ? min(in.sel_count[head], in.cap) : seq.pages, sh.max_pages);
  const int ntiles = (U + PPT - 1) / PPT;
  if (row0 >= M || chunk >= ntiles) return;
  // tiles are dealt round-robin to the workgroups, and a workgroup's to its wavefronts
  const int tfirst = chunk + nchunk * wave, tstep = nchunk * 4;
  const int ntw = tfirst < ntiles ? (ntiles - 1 - tfirst) / tstep + 1 : 0;

  // ---- query rows, in the order the keys' channels are contracted in
  bf16x8_t qf[R][NQ][KS];
#pragma unroll
  for (int mt = 0; mt < R; ++mt) {
    const int r = row0 + mt * 16 + l16, a = row_token(sh, min(r, sh.rows_max - 1));
    const int tok = in.active_idx ? in.active_idx[(size_t)b * sh.B + a] : a;
    const bool keep = r < M && (unsigned)tok < (unsigned)sh.B;
    const size_t at = (((size_t)b * sh.B + (keep ? tok : 0)) * sh.Hq + j * sh.G + (min(r, sh.rows_max - 1) - a * sh.G)) * D + qd * CPL;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (NQ == 1) {
        uint4 x = *reinterpret_cast<const uint4*>((const bf16_t*)in.q + at + ks * 8);
        if (!keep) x = make_uint4(0u, 0u, 0u, 0u);
        qf[mt][0][ks] = __builtin_bit_cast(bf16x8_t, x);
      } else {
        const float4 x0 = *reinterpret_cast<const float4*>((const float*)in.q + at + ks * 8), x1 = *reinterpret_cast<const float4*>((const float*)in.q + at + ks * 8 + 4);
        float x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (!keep) x[e] = 0.f;
            const __bf16 t = (__bf16)x[e];
            qf[mt][n][ks][e] = t;
            x[e] -= (float)t;
          }
      }
    }
  }

  float m_run[R], l_run[R], up_thr[R];
  const float inv_scale_log2e = 1.0f / scale_log2e;
  f32x4_t o[R][NT];
#pragma unroll
  for (int mt = 0; mt < R; ++mt) {
    m_run[mt] = kNegBig;
    up_thr[mt] = -INFINITY;
    l_run[mt] = 0.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) o[mt][nt] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  }

  // ---- pages of this wavefront's next TPR tiles, one per lane
  int pg_phys = 0, pg_valid = 0;
  auto fetch_pages = [&](int n0) {
    const int at = (tfirst + (n0 + lane / PPT) * tstep) * PPT + lane % PPT;
    int logical = -1, phys = -1;
    if (at < U) logical = in.list ? in.list[(size_t)head * in.cap + at] : at;
    if ((unsigned)logical < (unsigned)seq.pages) phys = kv.page_indices[seq.base + logical];
    const bool ok = (unsigned)phys < (unsigned)kv.num_pages;
    pg_phys = ok ? phys : 0;
    pg_valid = ok ? min(GP, seq.tokens - logical * GP) : 0;
  };

  struct Tile {
    uint32_t k[2][W], v[2][W], vs[2][4];   // vs: scales of the lane's four tokens, a byte per group (64 channels: two tokens a dword)
    uint32_t ks[2];
    int nv[2];   // valid tokens of the two subtiles
  };
  // A tile that does not exist is read like one, from the pool's first page, so that the loads in flight are the same number always.
  auto load_tile = [&](Tile& t, int n, int ne) {
    const bool real = n < ne;
    const int slot = (n * PPT) & 63;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int at = GP == 16 ? slot + s : slot;
      const int phys = real ? __builtin_amdgcn_readlane(pg_phys, at) : 0, valid = real ? __builtin_amdgcn_readlane(pg_valid, at) : 0;
      t.nv[s] = GP == 16 ? valid : valid - 16 * s;
      const int row = GP == 16 ? 0 : 16 * s;
      const size_t tile = (size_t)phys * sh.Hkv + j;
      load_dwords<W>(pk.k + tile * kTileBytes + (row + l16) * (D / 2) + qd * (CPL / 2), t.k[s]);
      load_dwords<W>(pk.v + tile * kTileBytes + ((row / 4 + qd) * 16 + l16) * (J * 4), t.v[s]);
      const uint8_t* sc = pk.scales + tile * (2 * GP * J);
      t.ks[s] = sc[(row + l16) * J + qd * CPL / 32];
      if constexpr (J == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(sc + GP * J + (row + qd * 4) * J);
        t.vs[s][0] = x.x;
        t.vs[s][1] = x.y;
        t.vs[s][2] = x.z;
        t.vs[s][3] = x.w;
      } else {
        const uint2 x = *reinterpret_cast<const uint2*>(sc + GP * J + (row + qd * 4) * J);
        t.vs[s][0] = x.x & 0xFFFFu;
        t.vs[s][1] = x.x >> 16;
        t.vs[s][2] = x.y & 0xFFFFu;
        t.vs[s][3] = x.y >> 16;
      }
    }
  };

  auto compute_tile = [&](Tile& t, bool first) {
    // scores
    f32x4_t sc[R][2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float ks_scale = power_of(t.ks[s]);
#pragma unroll
      for (int mt = 0; mt < R; ++mt) sc[mt][s] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const uint4 kf = make_uint4(codes_to_bf16<0>(t.k[s][ks], ks_scale), codes_to_bf16<1>(t.k[s][ks], ks_scale),
                                    codes_to_bf16<2>(t.k[s][ks], ks_scale), codes_to_bf16<3>(t.k[s][ks], ks_scale));
#pragma unroll
        for (int mt = 0; mt < R; ++mt)
#pragma unroll
          for (int n = NQ - 1; n >= 0; --n)
            sc[mt][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf), qf[mt][n][ks], sc[mt][s], 0, 0, 0);
      }
    }
    const bool full = t.nv[0] >= 16 && t.nv[1] >= 16;
    if (!full) {   // slots behind the sequence's end may hold anything
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool there = qd * 4 + e < t.nv[s];
          t.vs[s][e] = there ? t.vs[s][e] : 0u;   // (the smallest scale: nothing, in half precision)
#pragma unroll
          for (int mt = 0; mt < R; ++mt) sc[mt][s][e] = there ? sc[mt][s][e] : -INFINITY;
        }
    }
    // the rows' references: moved only where a maximum has overtaken one by kLag
    float tm[R];
    bool any_up = false;
#pragma unroll
    for (int mt = 0; mt < R; ++mt) {
      const f32x4_t a = sc[mt][0], c = sc[mt][1];
      tm[mt] = fmaxf(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])), fmaxf(fmaxf(c[0], c[1]), fmaxf(c[2], c[3])));
      any_up |= tm[mt] > up_thr[mt];
    }
    if (__any(any_up)) {
#pragma unroll
      for (int mt = 0; mt < R; ++mt) {
        const float cand = over_lane_groups_max(tm[mt]) * scale_log2e - kHeadroom;
        const bool up = cand > m_run[mt] + kLag;
        const float alpha = up ? __builtin_amdgcn_exp2f(m_run[mt] - cand) : 1.0f;
        m_run[mt] = up ? cand : m_run[mt];
        up_thr[mt] = (m_run[mt] + kHeadroom + kLag) * inv_scale_log2e;
        l_run[mt] *= alpha;
        if (!first) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[mt][nt] *= alpha;
        }
      }
    }
    f16x8_t p_hi[R], p_lo[R];
#pragma unroll
    for (int mt = 0; mt < R; ++mt) {
      const float neg_m = -m_run[mt];
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const f32x2_t p = {__builtin_amdgcn_exp2f(fmaf(sc[mt][e >> 2][e & 3], scale_log2e, neg_m)),
                           __builtin_amdgcn_exp2f(fmaf(sc[mt][e >> 2][(e & 3) + 1], scale_log2e, neg_m))};
        sum += p[0] + p[1];
        const f16x2_t hi = __builtin_convertvector(p, f16x2_t);
        const f32x2_t rest = {p[0] - (float)hi[0], p[1] - (float)hi[1]};
        const f16x2_t lo = __builtin_convertvector(rest, f16x2_t);
        p_hi[mt][e] = hi[0];
        p_hi[mt][e + 1] = hi[1];
        p_lo[mt][e] = lo[0];
        p_lo[mt][e + 1] = lo[1];
      }
      l_run[mt] += sum;
    }
    // values: group g's codes become the operands of channel tiles 2 g (low codes) and 2 g + 1
#pragma unroll
    for (int g = 0; g < J; ++g) {
      uint4 va, vb;
      uint32_t* const a = &va.x;
      uint32_t* const c = &vb.x;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = power_of((t.vs[s][e] >> (8 * g)) & 0xFFu);
        const uint32_t n0 = codes_to_f16<0>(t.v[s][g], f[0]), n1 = codes_to_f16<1>(t.v[s][g], f[1]);
        const uint32_t n2 = codes_to_f16<2>(t.v[s][g], f[2]), n3 = codes_to_f16<3>(t.v[s][g], f[3]);
        a[2 * s] = __builtin_amdgcn_perm(n1, n0, 0x05040100u);
        a[2 * s + 1] = __builtin_amdgcn_perm(n3, n2, 0x05040100u);
        c[2 * s] = __builtin_amdgcn_perm(n1, n0, 0x07060302u);
        c[2 * s + 1] = __builtin_amdgcn_perm(n3, n2, 0x07060302u);
      }
#pragma unroll
      for (int mt = 0; mt < R; ++mt) {
        o[mt][2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, va), p_hi[mt], o[mt][2 * g], 0, 0, 0);
        o[mt][2 * g + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, vb), p_hi[mt], o[mt][2 * g + 1], 0, 0, 0);
      }
#pragma unroll
      for (int mt = 0; mt < R; ++mt) {
        o[mt][2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, va), p_lo[mt], o[mt][2 * g], 0, 0, 0);
        o[mt][2 * g + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, vb), p_lo[mt], o[mt][2 * g + 1], 0, 0, 0);
      }
    }
  };

  Tile tb[NBUF];
  for (int nb = 0; nb < ntw; nb += TPR) {
    const int ne = min(ntw, nb + TPR);
    fetch_pages(nb);
#pragma unroll
    for (int k = 0; k < NBUF - 1; ++k) load_tile(tb[k], nb + k, ne);
    for (int n = nb; n < ne; n += NBUF) {
#pragma unroll
      for (int k = 0; k < NBUF; ++k) {
        load_tile(tb[(k + NBUF - 1) % NBUF], n + k + NBUF - 1, ne);
        if (n + k < ne) compute_tile(tb[k], n + k == 0);
      }
    }
  }

  // ---- the four wavefronts' states become one partial: everybody's in LDS, then a quarter of the channels each, in a fixed order
  constexpr int kSlot = R * NT * 64 * 4 + 2 * R * 16;   // O as [row tile][channel tile][lane] vectors, then references and sums
  float* mine = lds + wave * kSlot;
#pragma unroll
  for (int mt = 0; mt < R; ++mt) {
    const float l = over_lane_groups_sum(l_run[mt]);
    if (qd == 0) {
      mine[R * NT * 256 + mt * 16 + l16] = m_run[mt];
      mine[R * NT * 256 + R * 16 + mt * 16 + l16] = l;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f32x4_t*>(mine + ((mt * NT + nt) * 64 + lane) * 4) = o[mt][nt];
  }
  __syncthreads();
  const uint32_t item = (uint32_t)head * nchunk + chunk;
#pragma unroll
  for (int mt = 0; mt < R; ++mt) {
    const int r = row0 + mt * 16 + l16;
    if (r >= M) continue;
    float m[4], l[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      m[w] = lds[w * kSlot + R * NT * 256 + mt * 16 + l16];
      l[w] = lds[w * kSlot + R * NT * 256 + R * 16 + mt * 16 + l16];
    }
    const float m_all = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
    float wgt[4], l_all = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      wgt[w] = __builtin_amdgcn_exp2f(m[w] - m_all);
      l_all = fmaf(l[w], wgt[w], l_all);
    }
    const uint32_t prow = item * part.rows + r;
    if (wave == 0 && qd == 0) {
      part.m[prow] = m_all;
      part.l[prow] = l_all;
    }
#pragma unroll
    for (int k = 0; k < NT / 4; ++k) {
      const int nt = wave * (NT / 4) + k;
      f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) acc += *reinterpret_cast<const f32x4_t*>(lds + w * kSlot + ((mt * NT + nt) * 64 + lane) * 4) * wgt[w];
      *reinterpret_cast<f32x4_t*>(part.o + (size_t)prow * D + nt * 16 + qd * 4) = acc;
    }
  }
}

template <int R, int D>
constexpr size_t packed_lds_bytes() { return 4 * (R * (D / 16) * 256 + 2 * R * 16) * sizeof(float); }

// Rows that the host knows: blocks of R row tiles.
template <int D, int GP, int R, int NQ>
__global__ __launch_bounds__(256) void packed_attn_kernel(KvView kv, Shape sh, AttnInputs in, PackedView pk, int nchunk, int nrb, Partials part,
                                                          float scale_log2e) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  packed_attn_body<D, GP, R, NQ, 3>(kv, sh, in, pk, nchunk, nrb, (int)(blockIdx.y % nrb) * (R * 16), part, scale_log2e, lds);
}
// Rows counted on the device: every block of MOST row tiles takes the form made for the rows it has.
template <int D, int GP, int MOST, int NQ>
__global__ __launch_bounds__(256) void packed_attn_counted_kernel(KvView kv, Shape sh, AttnInputs in, PackedView pk, int nchunk, int nrb, Partials part,
                                                                  float scale_log2e) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int row0 = (int)(blockIdx.y % nrb) * (MOST * 16), left = active_rows(in, kv, sh, blockIdx.z) - row0;
  if (left <= 0) return;
  if (left <= 16)
    packed_attn_body<D, GP, 1, NQ, 3>(kv, sh, in, pk, nchunk, nrb, row0, part, scale_log2e, lds);
  else if (left <= 32 || MOST == 2)
    packed_attn_body<D, GP, 2, NQ, 3>(kv, sh, in, pk, nchunk, nrb, row0, part, scale_log2e, lds);
  else if constexpr (MOST > 2) {
    if (left <= 48)
      packed_attn_body<D, GP, 3, NQ, 3>(kv, sh, in, pk, nchunk, nrb, row0, part, scale_log2e, lds);
    else
      packed_attn_body<D, GP, 4, NQ, 3>(kv, sh, in, pk, nchunk, nrb, row0, part, scale_log2e, lds);
  }
}

template <int D, int GP, int R, int NQ, bool COUNTED>
static hipError_t launch_one(hipStream_t st, const KvView& kv, const Shape& sh, int batch, const AttnInputs& in, const PackedView& pk, int nchunk,
                             int rows, const Partials& part) {
  constexpr size_t lds_bytes = packed_lds_bytes<R, D>();
  void (*kern)(KvView, Shape, AttnInputs, PackedView, int, int, Partials, float);
  if constexpr (COUNTED)
    kern = packed_attn_counted_kernel<D, GP, R, NQ>;
  else
    kern = packed_attn_kernel<D, GP, R, NQ>;
  static bool attr_set = false;   // per instantiation
  if (lds_bytes > 48 * 1024 && !attr_set) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_bytes);
    if (e != hipSuccess) return e;
    attr_set = true;
  }
  const int nrb = (rows + R * 16 - 1) / (R * 16);
  kern<<<dim3(nchunk, sh.Hkv * nrb, batch), 256, lds_bytes, st>>>(kv, sh, in, pk, nchunk, nrb, part, sh.sm_scale * 1.4426950408889634f);
  return hipGetLastError();
}

template <int D, int GP>
static hipError_t launch_dg(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, int batch, const AttnInputs& in, const PackedView& pk,
                            int nchunk, int rows, bool known, const Partials& part) {
  if (dtype != LOSA_BF16) {
    if (rows <= 16) return launch_one<D, GP, 1, 3, false>(st, kv, sh, batch, in, pk, nchunk, rows, part);
    return known ? launch_one<D, GP, 2, 3, false>(st, kv, sh, batch, in, pk, nchunk, rows, part)
                 : launch_one<D, GP, 2, 3, true>(st, kv, sh, batch, in, pk, nchunk, rows, part);
  }
  if (rows <= 16) return launch_one<D, GP, 1, 1, false>(st, kv, sh, batch, in, pk, nchunk, rows, part);
  if (!known) return launch_one<D, GP, 4, 1, true>(st, kv, sh, batch, in, pk, nchunk, rows, part);
  if (rows <= 32) return launch_one<D, GP, 2, 1, false>(st, kv, sh, batch, in, pk, nchunk, rows, part);
  if (rows <= 48) return launch_one<D, GP, 3, 1, false>(st, kv, sh, batch, in, pk, nchunk, rows, part);
  return launch_one<D, GP, 4, 1, false>(st, kv, sh, batch, in, pk, nchunk, rows, part);
}

hipError_t launch_packed_attn(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, int batch, const AttnInputs& in, const PackedView& pk,
                              int nchunk, int rows, bool rows_known, const Partials& part) {
  if (batch <= 0 || nchunk <= 0 || rows <= 0) return hipSuccess;
  if (sh.d == 128)
    return sh.g == 16 ? launch_dg<128, 16>(st, dtype, kv, sh, batch, in, pk, nchunk, rows, rows_known, part)
                      : launch_dg<128, 32>(st, dtype, kv, sh, batch, in, pk, nchunk, rows, rows_known, part);
  return sh.g == 16 ? launch_dg<64, 16>(st, dtype, kv, sh, batch, in, pk, nchunk, rows, rows_known, part)
                    : launch_dg<64, 32>(st, dtype, kv, sh, batch, in, pk, nchunk, rows, rows_known, part);
}

}  // namespace losa
