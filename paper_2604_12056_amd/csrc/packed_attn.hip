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

#include <algorithm>

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

__device__ __forceinline__ void load_floats8(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// Scale bytes of four consecutive tokens' values: a dword per token, a byte per group.
template <int J>
__device__ __forceinline__ void load_scales(const uint8_t* p, uint32_t (&w)[4]) {
  if constexpr (J == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x;
    w[1] = x.y;
    w[2] = x.z;
    w[3] = x.w;
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x & 0xFFFFu;
    w[1] = x.x >> 16;
    w[2] = x.y & 0xFFFFu;
    w[3] = x.y >> 16;
  }
}

// Group g's codes of four tokens under their scales: the halves of channel tiles 2 g (low codes) and 2 g + 1, tokens side by side.
__device__ __forceinline__ void value_operands(uint32_t codes, const uint32_t (&scales)[4], int g, uint2& lo, uint2& hi) {
  float f[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = power_of((scales[e] >> (8 * g)) & 0xFFu);
  const uint32_t n0 = codes_to_f16<0>(codes, f[0]), n1 = codes_to_f16<1>(codes, f[1]);
  const uint32_t n2 = codes_to_f16<2>(codes, f[2]), n3 = codes_to_f16<3>(codes, f[3]);
  lo.x = __builtin_amdgcn_perm(n1, n0, 0x05040100u);
  lo.y = __builtin_amdgcn_perm(n3, n2, 0x05040100u);
  hi.x = __builtin_amdgcn_perm(n1, n0, 0x07060302u);
  hi.y = __builtin_amdgcn_perm(n3, n2, 0x07060302u);
}

// Numerators of a lane's four tokens of two subtiles as pairs of halves; returns their sum.
__device__ __forceinline__ float numerators(const f32x4_t& a, const f32x4_t& b, float scale_log2e, float neg_m, f16x8_t& p_hi, f16x8_t& p_lo) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const f32x4_t& s = e < 4 ? a : b;
    const f32x2_t p = {__builtin_amdgcn_exp2f(fmaf(s[e & 3], scale_log2e, neg_m)), __builtin_amdgcn_exp2f(fmaf(s[(e & 3) + 1], scale_log2e, neg_m))};
    sum += p[0] + p[1];
    const f16x2_t hi = __builtin_convertvector(p, f16x2_t);
    const f32x2_t rest = {p[0] - (float)hi[0], p[1] - (float)hi[1]};
    const f16x2_t lo = __builtin_convertvector(rest, f16x2_t);
    p_hi[e] = hi[0];
    p_hi[e + 1] = hi[1];
    p_lo[e] = lo[0];
    p_lo[e + 1] = lo[1];
  }
  return sum;
}

// ---- who does what.  The tiles of all (sequence, KV head) lists, one list behind the other and weighted with what a tile of so many query rows costs, are
// cut into equal shares, one per workgroup: lists of any lengths keep every compute unit busy to the end.  A share that ends inside a list leaves a
// partial, and the merge kernel joins a list's partials; a list that lies in one share is finished by its workgroup.
// Every workgroup works the cut out for itself from the counts (one memory round trip and a prefix sum): lists in the order of their
// heads, list h at [start, start + tiles * unit).  Tile t is workgroup (start + t * unit) / share's.  The partial of workgroup w for list h is item w + h.
// Beyond kPlannedHeads lists every one has a workgroup of its own.
struct Segment {
  int b, j, head, M;       // M: query rows
  int pages, t0, t1;       // listed pages, and the tiles [t0, t1) of them that are this workgroup's
  int item;                // partial; negative: the list is finished here
};
__device__ __forceinline__ int row_blocks(int M, int most) { return (M + most - 1) / most; }
// What a tile costs: converting it once per block of rows, and every 16 rows about as much as half of that.
__device__ __forceinline__ int unit_cost(int M, int block) { return M <= 0 ? 0 : 2 * row_blocks(M, block) + row_blocks(M, 16); }

// BLOCK: query rows that convert a tile once.  f(segment) for every list of this workgroup, in order.
template <int GP, int BLOCK, typename F>
__device__ __forceinline__ void for_each_segment(const KvView& kv, const Shape& sh, const AttnInputs& in, const Partials& part, const PackedOut& out, int heads,
                                                 int workgroups, int least_tiles, int* plan, F f) {
  constexpr int PPT = 32 / GP;
  const int lane = threadIdx.x & 63;
  auto list_of = [&](int h, int& M, int& pages) {
    const int b = h / sh.Hkv;
    M = min(active_rows(in, kv, sh, b), min(sh.rows_max, part.rows));
    const Sequence seq = sequence_of(kv, sh, b);
    pages = in.list ? max(0, min(min(in.sel_count[h], in.cap), sh.max_pages)) : seq.pages;
  };
  if (workgroups == 0) {   // a list each
    Segment s;
    s.head = blockIdx.x;
    s.b = s.head / sh.Hkv;
    s.j = s.head % sh.Hkv;
    list_of(s.head, s.M, s.pages);
    s.t0 = 0;
    s.t1 = (s.pages + PPT - 1) / PPT;
    s.item = -1;
    if (s.M > 0) f(s);
    return;
  }
  // the plan, [start | tiles | unit | pages] per head in LDS: every wavefront makes it, all of them the same
  int total = 0, most_unit = 1;
  for (int h0 = 0; h0 < heads; h0 += 64) {
    const int h = h0 + lane;
    int M = 0, pages = 0;
    if (h < heads) list_of(h, M, pages);
    const int unit = unit_cost(M, BLOCK), tiles = M > 0 ? (pages + PPT - 1) / PPT : 0, cost = tiles * unit;
    const int incl = wave_inclusive_scan(cost);
    if (h < heads) reinterpret_cast<int4*>(plan)[h] = make_int4(total + incl - cost, tiles, unit, pages);
    total += __builtin_amdgcn_readlane(incl, 63);
    most_unit = max(most_unit, (int)wave_max_u32((uint32_t)unit));
  }
  wave_lds_fence();
  const int w = blockIdx.x, share = max((total + workgroups - 1) / workgroups, least_tiles * most_unit);
  if (w == 0) {
    for (int h = threadIdx.x; h < heads; h += blockDim.x) {
      const int4 p = reinterpret_cast<const int4*>(plan)[h];
      const int first = p.x / share, last = (p.x + (p.y - 1) * p.z) / share;
      out.table[h] = make_int2(first + h, p.y > 0 ? last - first + 1 : 0);
    }
  }
  const int begin = w * share, end = begin + share;
  int first = heads;
  for (int h0 = 0; h0 < heads; h0 += 64) {   // the first list that reaches into the share
    const int h = h0 + lane;
    const int4 p = reinterpret_cast<const int4*>(plan)[min(h, heads - 1)];
    const unsigned long long in_it = __ballot(h < heads && p.y > 0 && p.x + p.y * p.z > begin);
    if (in_it) {
      first = h0 + __builtin_ctzll(in_it);
      break;
    }
  }
  for (int h = first; h < heads; ++h) {
    const int4 p = reinterpret_cast<const int4*>(plan)[h];
    const int start = __builtin_amdgcn_readfirstlane(p.x), tiles = __builtin_amdgcn_readfirstlane(p.y), unit = __builtin_amdgcn_readfirstlane(p.z);
    if (start >= end) break;
    if (tiles == 0) continue;
    Segment s;
    s.t0 = begin <= start ? 0 : (begin - start + unit - 1) / unit;
    s.t1 = min(tiles, (end - start + unit - 1) / unit);
    if (s.t0 >= s.t1) continue;
    s.head = h;
    s.b = h / sh.Hkv;
    s.j = h - s.b * sh.Hkv;
    s.M = min(active_rows(in, kv, sh, s.b), min(sh.rows_max, part.rows));
    s.pages = __builtin_amdgcn_readfirstlane(p.w);
    s.item = s.t0 == 0 && s.t1 == tiles ? -1 : w + h;
    f(s);
  }
}

// A vector of four channels of row r of a segment, numerators against `m` with sum `l`: a partial's, or the finished output.
template <int D>
__device__ __forceinline__ void store_state(const Shape& sh, const AttnInputs& in, const Partials& part, const PackedOut& out, const Segment& s, int r, int channel,
                                            f32x4_t acc, float m, float l) {
  if (s.item >= 0) {
    const uint32_t prow = (uint32_t)s.item * part.rows + r;
    if (channel == 0) {
      part.m[prow] = m;
      part.l[prow] = l;
    }
    *reinterpret_cast<f32x4_t*>(part.o + (size_t)prow * D + channel) = acc;
    return;
  }
  const int a = row_token(sh, r), tok = in.active_idx ? in.active_idx[(size_t)s.b * sh.B + a] : a;
  if ((unsigned)tok >= (unsigned)sh.B) return;
  const size_t orow = ((size_t)s.b * sh.B + tok) * sh.Hq + s.j * sh.G + (r - a * sh.G);
  const bool any = m > -1.0e29f || l != l;   // no valid token at all: the neutral element of a merge.  (Scores that are all NaN move no reference)
  *reinterpret_cast<f32x4_t*>(out.o_p + orow * D + channel) = any ? acc / l : (f32x4_t){0.f, 0.f, 0.f, 0.f};
  if (channel == 0) out.lse_p[orow] = any ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// Query rows row0 .. row0 + 16 R - 1 of a (sequence, KV head): what a workgroup of up to 64 rows does.  Its WAVES wavefronts deal the share's tiles out, two
// wavefronts to a SIMD, so that one's matrix products run beside the other's vector work.  That takes 256 registers a lane at most:
//   a tile's codes have no second buffer: the next tile's keys are requested when this one's have been converted, its values after
//     the last product (what is on its way per compute unit is still some 24 KiB);
//   the query fragments are read from LDS for every tile where there are more than two row tiles (or float queries).
// Four row tiles do not fit.  They are two sets of two (SETS): a wavefront of each set takes every tile, which reads its codes from
// the cache the second time and converts them twice, 128 of some 240 vector instructions a tile.
constexpr int kSlots = 4;   // LDS images of a wavefront's state (of a set): half of the wavefronts hand theirs over, twice; with two sets all have one
template <int R, int D, int NQ, int SETS = 1>
struct DealtLds {
  static constexpr bool kQueries = R > 2 || NQ > 1;
  static constexpr int kState = R * (D / 16) * 256 + 2 * R * 16;                    // floats: O as [row tile][channel tile][lane] vectors, references, sums
  static constexpr int kQueryFloats = kQueries ? NQ * R * (D / 32) * 256 : 0;
  static constexpr int kBytes = (kQueryFloats + SETS * kSlots * kState) * (int)sizeof(float);
};
template <int D, int GP, int R, int NQ, int SETS = 1>
__device__ __forceinline__ void packed_attn_body(const KvView& kv, const Shape& sh, const AttnInputs& in, const PackedView& pk, const Segment& seg, int row_base,
                                                 const Partials& part, const PackedOut& out, float scale_log2e, float* lds) {
  constexpr int WAVES = 2 * kSlots / SETS;   // of a set
  constexpr int KS = D / 32, NT = D / 16, J = D / 32, W = D / 32;   // products per score, channel tiles, groups, dwords a lane reads of a subtile
  constexpr int CPL = D / 4;                                        // channels of a token that a lane has
  constexpr int PPT = 32 / GP, TPR = 64 / PPT;                      // pages per tile, tiles per fetch of page entries
  constexpr int kTileBytes = GP * D / 2;
  typedef DealtLds<R, D, NQ, SETS> Lds;
  static_assert(SETS == 1 || !Lds::kQueries, "the sets' queries are not the same");
  constexpr bool kTight = D == 128 && Lds::kQueries;   // registers are short
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));   // (what derives from it is worked out per segment, not kept in registers over all of them)
  const int in_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = in_group % WAVES, set = in_group / WAVES;
  const int l16 = lane & 15, qd = lane >> 4;
  const int b = seg.b, j = seg.j, M = seg.M, row0 = row_base + set * (R * 16);
  const Sequence seq = sequence(kv, sh, b);
  // tiles are dealt round-robin to the wavefronts
  const int tfirst = seg.t0 + wave, ntw = tfirst < seg.t1 ? (seg.t1 - 1 - tfirst) / WAVES + 1 : 0;

  // ---- pages of this wavefront's next TPR tiles, one per lane
  int pg_phys = 0, pg_valid = 0;
  auto fetch_pages = [&](int n0) {
    const int at = (tfirst + (n0 + lane / PPT) * WAVES) * PPT + lane % PPT;
    int logical = -1, phys = -1;
    if (at < seg.pages) logical = in.list ? in.list[(size_t)seg.head * in.cap + at] : at;
    if ((unsigned)logical < (unsigned)seq.pages) phys = kv.page_indices[seq.base + logical];
    const bool ok = (unsigned)phys < (unsigned)kv.num_pages;
    pg_phys = ok ? phys : 0;
    pg_valid = ok ? min(GP, seq.tokens - logical * GP) : 0;
  };
  struct Keys {
    uint32_t c[2][W], s[2];
  } k;
  struct Values {
    uint32_t c[2][W], s[2][4];   // s: scales of the lane's four tokens, a byte per group
  } v;
  int nv[2] = {0, 0}, nv_next[2] = {0, 0};   // valid tokens of the two subtiles
  // tile n (where there is none, the pool's first page: nothing is made of it)
  auto page_of = [&](int n, int s) {
    const int at = GP == 16 ? (2 * n + s) & 63 : n & 63;
    return n < ntw ? __builtin_amdgcn_readlane(pg_phys, at) : 0;
  };
  auto load_keys = [&](int n) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const size_t tile = (size_t)page_of(n, s) * sh.Hkv + j;
      const int row = (GP == 16 ? 0 : 16 * s) + l16;
      load_dwords<W>(pk.k + tile * kTileBytes + row * (D / 2) + qd * (CPL / 2), k.c[s]);
      k.s[s] = pk.scales[tile * (2 * GP * J) + row * J + qd * CPL / 32];
      nv_next[s] = __builtin_amdgcn_readlane(pg_valid, GP == 16 ? (2 * n + s) & 63 : n & 63) - (GP == 16 ? 0 : 16 * s);
    }
  };
  auto load_values = [&](int n) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const size_t tile = (size_t)page_of(n, s) * sh.Hkv + j;
      const int quad = (GP == 16 ? 0 : 4 * s) + qd;
      load_dwords<W>(pk.v + tile * kTileBytes + (quad * 16 + l16) * (J * 4), v.c[s]);
      load_scales<J>(pk.scales + tile * (2 * GP * J) + GP * J + quad * 4 * J, v.s[s]);
    }
  };
  fetch_pages(0);
  load_keys(0);
  load_values(0);

  // ---- query rows, in the order the keys' channels are contracted in: fragment (row tile, term, product)
  bf16x8_t qf[Lds::kQueries ? 1 : R][NQ][KS];
  auto query = [&](int mt, int ks, bf16x8_t (&term)[NQ]) {
    const int r = row0 + mt * 16 + l16, rr = min(r, sh.rows_max - 1), a = row_token(sh, rr);
    const int tok = in.active_idx ? in.active_idx[(size_t)b * sh.B + a] : a;
    const bool keep = r < M && (unsigned)tok < (unsigned)sh.B;
    const size_t at = (((size_t)b * sh.B + (keep ? tok : 0)) * sh.Hq + j * sh.G + (rr - a * sh.G)) * D + qd * CPL + ks * 8;
    if constexpr (NQ == 1) {
      uint4 x = *reinterpret_cast<const uint4*>((const bf16_t*)in.q + at);
      if (!keep) x = make_uint4(0u, 0u, 0u, 0u);
      term[0] = __builtin_bit_cast(bf16x8_t, x);
    } else {
      float x[8];
      load_floats8((const float*)in.q + at, x);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (!keep) x[e] = 0.f;
          const __bf16 t = (__bf16)x[e];
          term[n][e] = t;
          x[e] -= (float)t;
        }
    }
  };
  const bf16x8_t* const q_lds = reinterpret_cast<const bf16x8_t*>(lds);
  if constexpr (Lds::kQueries) {
    for (int f = wave; f < R * KS; f += WAVES) {
      bf16x8_t term[NQ];
      query(f / KS, f % KS, term);
#pragma unroll
      for (int n = 0; n < NQ; ++n) reinterpret_cast<bf16x8_t*>(lds)[(f * NQ + n) * 64 + lane] = term[n];
    }
    __syncthreads();
  } else {
#pragma unroll
    for (int mt = 0; mt < R; ++mt)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8_t term[NQ];
        query(mt, ks, term);
#pragma unroll
        for (int n = 0; n < NQ; ++n) qf[mt][n][ks] = term[n];
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

  for (int n = 0; n < ntw; ++n) {
    nv[0] = nv_next[0];
    nv[1] = nv_next[1];
    if ((n + 1) % TPR == 0) fetch_pages(n + 1);   // (the entries are decoded behind the branch, so nothing waits where it joins)
    // scores, a subtile at a time (the barriers keep what is read or converted ahead, and so the registers, to that)
    f32x4_t sc[R][2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const float scale = power_of(k.s[s]);
      bf16x8_t kf[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        kf[ks] = __builtin_bit_cast(bf16x8_t, make_uint4(codes_to_bf16<0>(k.c[s][ks], scale), codes_to_bf16<1>(k.c[s][ks], scale),
                                                         codes_to_bf16<2>(k.c[s][ks], scale), codes_to_bf16<3>(k.c[s][ks], scale)));
      if (s == 1) load_keys(n + 1);
#pragma unroll
      for (int mt = 0; mt < R; ++mt) {
        sc[mt][s] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int t = NQ - 1; t >= 0; --t) {
            bf16x8_t q;
            if constexpr (Lds::kQueries)
              q = q_lds[((mt * KS + ks) * NQ + t) * 64 + lane];
            else
              q = qf[mt][t][ks];
            sc[mt][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[ks], q, sc[mt][s], 0, 0, 0);
          }
      }
      if constexpr (kTight) __builtin_amdgcn_sched_barrier(0);
    }
    if (!(nv[0] >= 16 && nv[1] >= 16)) {   // slots behind the sequence's end may hold anything
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool there = qd * 4 + e < nv[s];
          v.s[s][e] = there ? v.s[s][e] : 0u;   // (the smallest scale: nothing, in half precision)
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
        if (n > 0) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[mt][nt] *= alpha;
        }
      }
    }
    f16x8_t p_hi[R], p_lo[R];
#pragma unroll
    for (int mt = 0; mt < R; ++mt) l_run[mt] += numerators(sc[mt][0], sc[mt][1], scale_log2e, -m_run[mt], p_hi[mt], p_lo[mt]);
#pragma unroll
    for (int g = 0; g < J; ++g) {
      uint2 lo[2], hi[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) value_operands(v.c[s][g], v.s[s], g, lo[s], hi[s]);
      const f16x8_t va = __builtin_bit_cast(f16x8_t, make_uint4(lo[0].x, lo[0].y, lo[1].x, lo[1].y));
      const f16x8_t vb = __builtin_bit_cast(f16x8_t, make_uint4(hi[0].x, hi[0].y, hi[1].x, hi[1].y));
      if (g == J - 1) load_values(n + 1);
      if constexpr (kTight) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int mt = 0; mt < R; ++mt) {
        o[mt][2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, p_hi[mt], o[mt][2 * g], 0, 0, 0);
        o[mt][2 * g + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vb, p_hi[mt], o[mt][2 * g + 1], 0, 0, 0);
      }
#pragma unroll
      for (int mt = 0; mt < R; ++mt) {
        o[mt][2 * g] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, p_lo[mt], o[mt][2 * g], 0, 0, 0);
        o[mt][2 * g + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vb, p_lo[mt], o[mt][2 * g + 1], 0, 0, 0);
      }
    }
  }

  // ---- the wavefronts' states become one partial, in a fixed order: the second half of them hands its states to the first through LDS, those hand theirs
  // to everybody, and each wavefront makes some of the partial's vectors
#pragma unroll
  for (int mt = 0; mt < R; ++mt) l_run[mt] = over_lane_groups_sum(l_run[mt]);
  float* const states = lds + Lds::kQueryFloats;
  float* const slot = states + (SETS == 1 ? wave % kSlots : in_group) * Lds::kState;
  auto publish = [&]() {
#pragma unroll
    for (int mt = 0; mt < R; ++mt) {
      if (qd == 0) {
        slot[R * NT * 256 + mt * 16 + l16] = m_run[mt];
        slot[R * NT * 256 + R * 16 + mt * 16 + l16] = l_run[mt];
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) *reinterpret_cast<f32x4_t*>(slot + ((mt * NT + nt) * 64 + lane) * 4) = o[mt][nt];
    }
  };
  if constexpr (SETS == 1) {
    if (wave >= kSlots) publish();
    __syncthreads();
    if (wave < kSlots) {
#pragma unroll
      for (int mt = 0; mt < R; ++mt) {
        const float m = slot[R * NT * 256 + mt * 16 + l16], l = slot[R * NT * 256 + R * 16 + mt * 16 + l16];
        const float m_all = fmaxf(m_run[mt], m), mine = __builtin_amdgcn_exp2f(m_run[mt] - m_all), theirs = __builtin_amdgcn_exp2f(m - m_all);
        m_run[mt] = m_all;
        l_run[mt] = fmaf(l_run[mt], mine, l * theirs);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[mt][nt] = o[mt][nt] * mine + *reinterpret_cast<const f32x4_t*>(slot + ((mt * NT + nt) * 64 + lane) * 4) * theirs;
      }
      publish();   // (where this wavefront alone has just read)
    }
  } else {
    publish();
  }
  __syncthreads();
  for (int piece = in_group; piece < SETS * R * NT; piece += SETS * WAVES) {
    const int of = piece / (R * NT), vec = piece % (R * NT), mt = vec / NT, nt = vec % NT, r = row_base + of * (R * 16) + mt * 16 + l16;
    if (r >= M) continue;
    float m[kSlots], l[kSlots], m_all = kNegBig;
    f32x4_t x[kSlots];
#pragma unroll
    for (int w = 0; w < kSlots; ++w) {
      const float* from = states + (of * kSlots + w) * Lds::kState;
      m[w] = from[R * NT * 256 + mt * 16 + l16];
      l[w] = from[R * NT * 256 + R * 16 + mt * 16 + l16];
      x[w] = *reinterpret_cast<const f32x4_t*>(from + (vec * 64 + lane) * 4);
      m_all = fmaxf(m_all, m[w]);
    }
    float l_all = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kSlots; ++w) {
      const float wgt = __builtin_amdgcn_exp2f(m[w] - m_all);
      l_all = fmaf(l[w], wgt, l_all);
      acc += x[w] * wgt;
    }
    store_state<D>(sh, in, part, out, seg, r, nt * 16 + qd * 4, acc, m_all, l_all);
  }
  __syncthreads();   // the LDS is the next segment's
}

// ---- more than 64 query rows: the eight wavefronts of a workgroup have R*16 rows each and share the tiles.
//
// Two tiles of the workgroup's share are a stage of 64 tokens, four subtiles.  Every wavefront reads one subtile's codes, of keys or of values, converts
// them once for all rows and leaves them in LDS as the matrix core's operands, 16 bytes a lane, in lane order.  Two LDS buffers and
// a barrier per stage; the codes of the next kAhead stages are on their way in registers.
template <int D>
constexpr int kStageBytes = 64 * D * 2 * 2;   // keys, then values
constexpr int kAhead = 2;

template <int D, int GP, int R>
__device__ __forceinline__ void packed_rows_body(const KvView& kv, const Shape& sh, const AttnInputs& in, const PackedView& pk, const Segment& seg, int row_base,
                                                 const Partials& part, const PackedOut& out, float scale_log2e, char* lds) {
  constexpr int KS = D / 32, NT = D / 16, J = D / 32, W = D / 32, CPL = D / 4, PPT = 32 / GP, TPR = 64 / PPT;
  constexpr int kTileBytes = GP * D / 2;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));   // (see the other form)
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, qd = lane >> 4;
  const int b = seg.b, j = seg.j, M = seg.M, row0 = row_base + wave * (R * 16);
  const Sequence seq = sequence(kv, sh, b);
  const int stages = (seg.t1 - seg.t0 + 1) / 2;

  bf16x8_t qf[R][KS];
#pragma unroll
  for (int mt = 0; mt < R; ++mt) {
    const int r = row0 + mt * 16 + l16, rr = min(r, sh.rows_max - 1), a = row_token(sh, rr);
    const int tok = in.active_idx ? in.active_idx[(size_t)b * sh.B + a] : a;
    const bool keep = r < M && (unsigned)tok < (unsigned)sh.B;
    const bf16_t* row = (const bf16_t*)in.q + (((size_t)b * sh.B + (keep ? tok : 0)) * sh.Hq + j * sh.G + (rr - a * sh.G)) * D + qd * CPL;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint4 x = *reinterpret_cast<const uint4*>(row + ks * 8);
      if (!keep) x = make_uint4(0u, 0u, 0u, 0u);
      qf[mt][ks] = __builtin_bit_cast(bf16x8_t, x);
    }
  }

  // pages of the share's next TPR tiles, one per lane
  int pg_phys = 0, pg_valid = 0;
  auto fetch_pages = [&](int n0) {
    const int tile = seg.t0 + n0 + lane / PPT, at = tile * PPT + lane % PPT;
    int logical = -1, phys = -1;
    if (tile < seg.t1 && at < seg.pages) logical = in.list ? in.list[(size_t)seg.head * in.cap + at] : at;
    if ((unsigned)logical < (unsigned)seq.pages) phys = kv.page_indices[seq.base + logical];
    const bool ok = (unsigned)phys < (unsigned)kv.num_pages;
    pg_phys = ok ? phys : 0;
    pg_valid = ok ? min(GP, seq.tokens - logical * GP) : 0;
  };
  // valid tokens of subtile s of stage i (of the TPR tiles at hand)
  auto valid_of = [&](int i, int s) {
    const int at = (2 * i + s / 2) * PPT;
    return GP == 16 ? __builtin_amdgcn_readlane(pg_valid, (at + s % 2) & 63) : __builtin_amdgcn_readlane(pg_valid, at & 63) - 16 * (s % 2);
  };

  struct Raw {
    uint32_t c[W], vs[4], ks;   // codes of keys or of values
  };
  const bool has_keys = wave < 4;
  const int mysub = wave & 3;
  auto load_stage = [&](Raw& x, int i) {   // (past the end: the pool's first page, as nothing depends on it)
    const int at = ((2 * i + mysub / 2) * PPT + (GP == 16 ? mysub % 2 : 0)) & 63;
    const size_t tile = (size_t)__builtin_amdgcn_readlane(pg_phys, at) * sh.Hkv + j;
    const int row = GP == 16 ? 0 : 16 * (mysub % 2);
    const uint8_t* sc = pk.scales + tile * (2 * GP * J);
    const uint8_t* keys = pk.k + tile * kTileBytes + (row + l16) * (D / 2) + qd * (CPL / 2);
    const uint8_t* values = pk.v + tile * kTileBytes + ((row / 4 + qd) * 16 + l16) * (J * 4);
    load_dwords<W>(has_keys ? keys : values, x.c);
    x.ks = sc[(row + l16) * J + qd * CPL / 32];   // (one of the two in vain: no branch around a load)
    load_scales<J>(sc + GP * J + (row + qd * 4) * J, x.vs);
  };
  auto convert_stage = [&](Raw& x, int i, char* buf) {
    if (has_keys) {
      const float scale = power_of(x.ks);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        *reinterpret_cast<uint4*>(buf + ((mysub * KS + ks) * 64 + lane) * 16) =
            make_uint4(codes_to_bf16<0>(x.c[ks], scale), codes_to_bf16<1>(x.c[ks], scale), codes_to_bf16<2>(x.c[ks], scale), codes_to_bf16<3>(x.c[ks], scale));
    }
    if (!has_keys) {
      const int valid = valid_of(i, mysub);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.vs[e] = qd * 4 + e < valid ? x.vs[e] : 0u;   // (see the other form)
      char* v = buf + 64 * D * 2 + ((mysub / 2) * NT * 64 + lane) * 16 + (mysub % 2) * 8;
#pragma unroll
      for (int g = 0; g < J; ++g) {
        uint2 lo, hi;
        value_operands(x.c[g], x.vs, g, lo, hi);
        *reinterpret_cast<uint2*>(v + (2 * g) * 1024) = lo;
        *reinterpret_cast<uint2*>(v + (2 * g + 1) * 1024) = hi;
      }
    }
  };

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
  const bool has_rows = row0 < M;   // (the others convert only)

  auto compute_stage = [&](int i, const char* buf, bool first) {
    f32x4_t sc[R][4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
#pragma unroll
      for (int mt = 0; mt < R; ++mt) sc[mt][s] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(buf + ((s * KS + ks) * 64 + lane) * 16);
#pragma unroll
        for (int mt = 0; mt < R; ++mt) sc[mt][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[mt][ks], sc[mt][s], 0, 0, 0);
      }
    }
    int nv[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) nv[s] = valid_of(i, s);
    if (!(nv[0] >= 16 && nv[1] >= 16 && nv[2] >= 16 && nv[3] >= 16)) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int mt = 0; mt < R; ++mt) sc[mt][s][e] = qd * 4 + e < nv[s] ? sc[mt][s][e] : -INFINITY;
    }
    float tm[R];
    bool any_up = false;
#pragma unroll
    for (int mt = 0; mt < R; ++mt) {
      tm[mt] = sc[mt][0][0];
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) tm[mt] = fmaxf(tm[mt], sc[mt][s][e]);
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
#pragma unroll
    for (int h = 0; h < 2; ++h) {   // a pair of subtiles at a time
      f16x8_t p_hi[R], p_lo[R];
#pragma unroll
      for (int mt = 0; mt < R; ++mt) l_run[mt] += numerators(sc[mt][2 * h], sc[mt][2 * h + 1], scale_log2e, -m_run[mt], p_hi[mt], p_lo[mt]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const f16x8_t vf = *reinterpret_cast<const f16x8_t*>(buf + 64 * D * 2 + ((h * NT + nt) * 64 + lane) * 16);
#pragma unroll
        for (int mt = 0; mt < R; ++mt) o[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p_hi[mt], o[mt][nt], 0, 0, 0);
#pragma unroll
        for (int mt = 0; mt < R; ++mt) o[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p_lo[mt], o[mt][nt], 0, 0, 0);
      }
    }
  };

  constexpr int SPF = TPR / 2;   // stages per fetch of page entries
  Raw raw[kAhead];
  for (int n0 = 0; n0 < stages; n0 += SPF) {
    const int ne = min(stages - n0, SPF);   // stages of this fetch, counted from its first
    fetch_pages(2 * n0);
    if (n0 > 0) __syncthreads();            // the buffers' last readers are done
#pragma unroll
    for (int k = 0; k < kAhead; ++k) load_stage(raw[k], k);
    convert_stage(raw[0], 0, lds);
    load_stage(raw[0], kAhead);
    __syncthreads();
    for (int i = 0; i < ne; i += 2) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // Stage i + k is in buffer k, the next one goes to the other.  (Whether there is one or not: loads behind a branch, or a use of theirs,
        // would be waited for where the branches join.)
        convert_stage(raw[(k + 1) % kAhead], i + k + 1, lds + (1 - k) * kStageBytes<D>);
        load_stage(raw[(k + 1) % kAhead], i + k + 1 + kAhead);
        if (has_rows && i + k < ne) compute_stage(i + k, lds + k * kStageBytes<D>, n0 + i + k == 0);
        __syncthreads();
      }
    }
  }

  float l_row[R];
#pragma unroll
  for (int mt = 0; mt < R; ++mt) l_row[mt] = over_lane_groups_sum(l_run[mt]);
#pragma unroll
  for (int mt = 0; mt < R; ++mt) {
    const int r = row0 + mt * 16 + l16;
    if (r >= M) continue;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) store_state<D>(sh, in, part, out, seg, r, nt * 16 + qd * 4, o[mt][nt], m_run[mt], l_row[mt]);
  }
}

#define LOSA_PACKED_ARGS KvView kv, Shape sh, AttnInputs in, PackedView pk, Partials part, PackedOut out, float scale_log2e, int heads, int workgroups, int least_tiles
// Rows that the host knows: blocks of SETS * R row tiles, one after the other.
template <int D, int GP, int R, int NQ, int SETS = 1>
__global__ __launch_bounds__(128 * kSlots) void packed_attn_kernel(LOSA_PACKED_ARGS) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  constexpr int kRows = SETS * R * 16;
  int* plan = reinterpret_cast<int*>(lds) + DealtLds<R, D, NQ, SETS>::kBytes / 4;
  for_each_segment<GP, kRows>(kv, sh, in, part, out, heads, workgroups, least_tiles, plan, [&](const Segment& s) {
    for (int row0 = 0; row0 < s.M; row0 += kRows) packed_attn_body<D, GP, R, NQ, SETS>(kv, sh, in, pk, s, row0, part, out, scale_log2e, lds);
  });
}
// ... blocks of 8 * R row tiles.
template <int D, int GP, int R>
__global__ __launch_bounds__(512) void packed_rows_kernel(LOSA_PACKED_ARGS) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  constexpr int kRows = 128 * R;
  int* plan = reinterpret_cast<int*>(lds) + 2 * kStageBytes<D> / 4;
  for_each_segment<GP, kRows>(kv, sh, in, part, out, heads, workgroups, least_tiles, plan, [&](const Segment& s) {
    for (int row0 = 0; row0 < s.M; row0 += kRows) packed_rows_body<D, GP, R>(kv, sh, in, pk, s, row0, part, out, scale_log2e, reinterpret_cast<char*>(lds));
  });
}
// Rows counted on the device: the form made for the rows a head has, block after block.
template <int NQ>
constexpr int kCountedRows = NQ == 1 ? 64 : 32;
template <int D, int NQ>
constexpr int kCountedBytes = NQ == 1 ? std::max(DealtLds<3, D, 1>::kBytes, DealtLds<2, D, 1, 2>::kBytes) : DealtLds<2, D, NQ>::kBytes;
template <int D, int GP, int NQ>
__global__ __launch_bounds__(128 * kSlots) void packed_attn_counted_kernel(LOSA_PACKED_ARGS) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  int* plan = reinterpret_cast<int*>(lds) + kCountedBytes<D, NQ> / 4;
  for_each_segment<GP, kCountedRows<NQ>>(kv, sh, in, part, out, heads, workgroups, least_tiles, plan, [&](const Segment& s) {
    for (int row0 = 0; row0 < s.M; row0 += kCountedRows<NQ>) {
      const int left = s.M - row0;
      if (left <= 16)
        packed_attn_body<D, GP, 1, NQ>(kv, sh, in, pk, s, row0, part, out, scale_log2e, lds);
      else if (left <= 32 || NQ > 1)
        packed_attn_body<D, GP, 2, NQ>(kv, sh, in, pk, s, row0, part, out, scale_log2e, lds);
      else if constexpr (NQ == 1) {
        if (left <= 48)
          packed_attn_body<D, GP, 3, NQ>(kv, sh, in, pk, s, row0, part, out, scale_log2e, lds);
        else
          packed_attn_body<D, GP, 2, NQ, 2>(kv, sh, in, pk, s, row0, part, out, scale_log2e, lds);
      }
    }
  });
}

// ---- joins a list's partials: a workgroup per row (of a few, in turn), 1024 / D lanes of items times D / 4 channel quads, eight items of a lane at
// once; sums in a fixed order.
template <int D>
__global__ __launch_bounds__(256) void packed_join_kernel(KvView kv, Shape sh, AttnInputs in, Partials part, PackedOut out) {
  constexpr int C4 = D / 4, CL = 256 / C4, KB = 8;
  __shared__ __attribute__((aligned(16))) float4 red[CL][C4];
  __shared__ float2 stats[CL];
  const int tid = threadIdx.x, cl = tid / C4, c4 = tid % C4, head = blockIdx.y, b = head / sh.Hkv, j = head - b * sh.Hkv;
  const int2 table = out.table[head];
  const int M = min(active_rows(in, kv, sh, b), min(sh.rows_max, part.rows));
  if (table.y == 1) return;   // finished already
  for (int r = blockIdx.x; r < M; r += gridDim.x) {
    const int a = row_token(sh, r), tok = in.active_idx ? in.active_idx[(size_t)b * sh.B + a] : a;
    float m = kNegBig, l = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = cl; i0 < table.y; i0 += CL * KB) {
      float mk[KB], lk[KB];
      f32x4_t x[KB];
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const uint32_t prow = (uint32_t)(table.x + min(i0 + CL * k, table.y - 1)) * part.rows + r;
        mk[k] = part.m[prow];
        lk[k] = part.l[prow];
        x[k] = reinterpret_cast<const f32x4_t*>(part.o + (size_t)prow * D)[c4];
      }
      float m_new = m;
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        if (i0 + CL * k >= table.y) mk[k] = kNegBig, lk[k] = 0.f, x[k] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
        m_new = fmaxf(m_new, mk[k]);
      }
      const float keep = __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= keep;
      acc *= keep;
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const float wgt = __builtin_amdgcn_exp2f(mk[k] - m);
        l = fmaf(lk[k], wgt, l);
        acc += x[k] * wgt;
      }
    }
    red[cl][c4] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (c4 == 0) stats[cl] = make_float2(m, l);
    __syncthreads();
    if (tid < C4 && (unsigned)tok < (unsigned)sh.B) {
      float m_all = kNegBig, l_all = 0.f;
      f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < CL; ++k) m_all = fmaxf(m_all, stats[k].x);
#pragma unroll
      for (int k = 0; k < CL; ++k) {
        const float wgt = __builtin_amdgcn_exp2f(stats[k].x - m_all);
        const float4 x = red[k][c4];
        l_all = fmaf(stats[k].y, wgt, l_all);
        o += (f32x4_t){x.x, x.y, x.z, x.w} * wgt;
      }
      Segment s;
      s.b = b;
      s.j = j;
      s.item = -1;
      store_state<D>(sh, in, part, out, s, r, c4 * 4, o, m_all, l_all);
    }
    __syncthreads();   // the LDS is the next row's
  }
}

typedef void (*PackedKernel)(LOSA_PACKED_ARGS);

template <int D, int GP>
static hipError_t launch_dg(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, const AttnInputs& in, const PackedView& pk, int heads, int workgroups,
                            int least_tiles, int rows, bool known, const Partials& part, const PackedOut& out) {
  auto go = [&](PackedKernel kern, int lds_bytes, bool& attr_set) {
    const int all = lds_bytes + (workgroups ? heads * 16 : 0);   // the plan behind the kernel's own
    if (!attr_set) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes + kPlannedHeads * 16);
      if (e != hipSuccess) return e;
      attr_set = true;
    }
    kern<<<workgroups ? workgroups : heads, 512, all, st>>>(kv, sh, in, pk, part, out, sh.sm_scale * 1.4426950408889634f, heads, workgroups, least_tiles);
    return hipGetLastError();
  };
  static bool set[10];   // per kernel
  if (dtype != LOSA_BF16) {
    if (rows <= 16) return go(packed_attn_kernel<D, GP, 1, 3>, DealtLds<1, D, 3>::kBytes, set[0]);
    return known ? go(packed_attn_kernel<D, GP, 2, 3>, DealtLds<2, D, 3>::kBytes, set[1]) : go(packed_attn_counted_kernel<D, GP, 3>, kCountedBytes<D, 3>, set[2]);
  }
  if (rows <= 16) return go(packed_attn_kernel<D, GP, 1, 1>, DealtLds<1, D, 1>::kBytes, set[3]);
  if (!known) return go(packed_attn_counted_kernel<D, GP, 1>, kCountedBytes<D, 1>, set[4]);
  if (rows <= 32) return go(packed_attn_kernel<D, GP, 2, 1>, DealtLds<2, D, 1>::kBytes, set[5]);
  if (rows <= 48) return go(packed_attn_kernel<D, GP, 3, 1>, DealtLds<3, D, 1>::kBytes, set[6]);
  if (rows <= 64) return go(packed_attn_kernel<D, GP, 2, 1, 2>, DealtLds<2, D, 1, 2>::kBytes, set[7]);
  return rows <= 128 ? go(packed_rows_kernel<D, GP, 1>, 2 * kStageBytes<D>, set[8]) : go(packed_rows_kernel<D, GP, 2>, 2 * kStageBytes<D>, set[9]);
}

hipError_t launch_packed_attn(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, int batch, const AttnInputs& in, const PackedView& pk, int workgroups,
                              int least_tiles, int rows, bool rows_known, const Partials& part, const PackedOut& out) {
  const int heads = batch * sh.Hkv;
  if (heads <= 0 || rows <= 0) return hipSuccess;
  auto launch = sh.d == 128 ? (sh.g == 16 ? launch_dg<128, 16> : launch_dg<128, 32>) : (sh.g == 16 ? launch_dg<64, 16> : launch_dg<64, 32>);
  return launch(st, dtype, kv, sh, in, pk, heads, workgroups, least_tiles, rows, rows_known, part, out);
}

hipError_t launch_packed_join(hipStream_t st, const KvView& kv, const Shape& sh, int batch, const AttnInputs& in, int rows, bool rows_known, const Partials& part,
                              const PackedOut& out) {
  const dim3 grid(rows_known ? rows : min(rows, 64), batch * sh.Hkv);   // (rows that only the device counts are mostly few)
  if (sh.d == 128)
    packed_join_kernel<128><<<grid, 256, 0, st>>>(kv, sh, in, part, out);
  else
    packed_join_kernel<64><<<grid, 256, 0, st>>>(kv, sh, in, part, out);
  return hipGetLastError();
}

}  // namespace losa
