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
// nearest and lo = p - hi rounded again (22 bits: error 2^-23 of p, against 2^-17 of a bfloat16 pair at the same cost), and so does their sum,
// in float.  Float mode splits a query into three bfloat16 terms, which hold its 24 bits.
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

template <int N>
__device__ __forceinline__ void lds_dwords(const char* p, uint32_t (&w)[N]) {
  if constexpr (N == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    w[0] = x.x, w[1] = x.y;
  }
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

// The power of two that byte g of a dword stands for, in one instruction (left to itself the compiler makes two of the shift and the mask).
__device__ __forceinline__ float power_of_byte(uint32_t w, int g) {
  uint32_t r;
  const uint32_t places = 23;
  if (g == 0)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(places), "v"(w));
  else if (g == 1)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(places), "v"(w));
  else if (g == 2)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(places), "v"(w));
  else
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(r) : "v"(places), "v"(w));
  return __uint_as_float(r);
}

// Group g's codes of four tokens under their scales: the halves of channel tiles 2 g (low codes) and 2 g + 1, tokens side by side.
__device__ __forceinline__ void value_operands(uint32_t codes, const uint32_t (&scales)[4], int g, uint2& lo, uint2& hi) {
  float f[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = power_of_byte(scales[e], g);
  const uint32_t n0 = codes_to_f16<0>(codes, f[0]), n1 = codes_to_f16<1>(codes, f[1]);
  const uint32_t n2 = codes_to_f16<2>(codes, f[2]), n3 = codes_to_f16<3>(codes, f[3]);
  lo.x = __builtin_amdgcn_perm(n1, n0, 0x05040100u);
  lo.y = __builtin_amdgcn_perm(n3, n2, 0x05040100u);
  hi.x = __builtin_amdgcn_perm(n1, n0, 0x07060302u);
  hi.y = __builtin_amdgcn_perm(n3, n2, 0x07060302u);
}

// p - hi, where hi is the low (HIGH: high) half of a dword, in one instruction.
template <bool HIGH>
__device__ __forceinline__ float remainder_of(float p, f16x2_t hi) {
  float r;
  const uint32_t bits = __builtin_bit_cast(uint32_t, hi);
  if constexpr (HIGH)
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(bits), "v"(p));
  else
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(bits), "v"(p));
  return r;
}

// Numerators of two neighbouring scores as pairs of halves, element e and the next of the operands; their sum.
__device__ __forceinline__ float numerator_pair(float s0, float s1, float scale_log2e, float neg_m, int e, f16x8_t& p_hi, f16x8_t& p_lo) {
  const f32x2_t p = {__builtin_amdgcn_exp2f(fmaf(s0, scale_log2e, neg_m)), __builtin_amdgcn_exp2f(fmaf(s1, scale_log2e, neg_m))};
  const f16x2_t hi = __builtin_convertvector(p, f16x2_t);
  const f32x2_t rest = {remainder_of<false>(p[0], hi), remainder_of<true>(p[1], hi)};
  const f16x2_t lo = __builtin_convertvector(rest, f16x2_t);
  p_hi[e] = hi[0];
  p_hi[e + 1] = hi[1];
  p_lo[e] = lo[0];
  p_lo[e + 1] = lo[1];
  return p[0] + p[1];
}
// ... of a lane's four tokens of two subtiles.
__device__ __forceinline__ void numerators(const f32x4_t& a, const f32x4_t& b, float scale_log2e, float neg_m, f16x8_t& p_hi, f16x8_t& p_lo) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const f32x4_t& s = e < 4 ? a : b;
    numerator_pair(s[e & 3], s[(e & 3) + 1], scale_log2e, neg_m, e, p_hi, p_lo);
  }
}
// One more row of values, all ones: its products with the numerators are their sums, on the matrix core, which has time for them where the vector
// units have not.
__device__ __forceinline__ f16x8_t ones() {
  f16x8_t x;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (_Float16)1.0f;
  return x;
}
__device__ __forceinline__ f32x4_t sum_of(const f16x8_t& p_hi, const f16x8_t& p_lo, f32x4_t l) {
  l = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones(), p_hi, l, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(ones(), p_lo, l, 0, 0, 0);
}

// ---- who does what.  The tiles of all (sequence, KV head) lists, one list behind the other and weighted with what a tile of so many query rows costs, are
// cut into equal shares, one per workgroup: lists of any lengths keep every compute unit busy to the end.  A share that ends inside a list leaves a
// partial, and the merge kernel joins a list's partials; a list that lies in one share is finished by its workgroup.
// Every workgroup works the cut out for itself from the counts (one memory round trip and a prefix sum): lists in the order of their
// heads, list h at [start, start + tiles * unit), and ahead of each the time that its start and its end take, as tiles (GAP: some 10 us where four
// wavefronts deal tiles out; without it a workgroup with the end of one list and the start of another took twice the others' time).  Tile t is workgroup (start + t * unit) / share's.  The partial of workgroup w for list h is item w + h.
// Beyond kPlannedHeads lists every one has a workgroup of its own.
struct Segment {
  int b, j, head, M;               // M: query rows
  int base, tokens, seq_pages;     // the sequence
  int pages, t0, t1;               // listed pages, and the tiles [t0, t1) of them that are this workgroup's
  int item;                        // partial; negative: the list is finished here
};
__device__ __forceinline__ int row_blocks(int M, int most) { return (M + most - 1) / most; }
// What a tile costs: converting it once per block of rows, and every 16 rows about as much as half of that.
__device__ __forceinline__ int unit_cost(int M, int block) { return M <= 0 ? 0 : 2 * row_blocks(M, block) + row_blocks(M, 16); }

// a / b for 0 <= a < 2^31 and a quotient below 2^20: the float's is off by one at most.
__device__ __forceinline__ int quotient(int a, int b) {
  int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b));
  const int r = a - q * b;
  q += r >= b ? 1 : 0;
  return q - (r < 0 ? 1 : 0);
}

// BLOCK: query rows that convert a tile once.  f(segment) for every list of this workgroup, in order.
template <int GP, int BLOCK, int GAP, typename F>
__device__ __forceinline__ void for_each_segment(const KvView& kv, const Shape& sh, const AttnInputs& in, const Partials& part, const PackedOut& out, int heads,
                                                 int workgroups, int least_tiles, int* plan, F f) {
  constexpr int PPT = 32 / GP;
  const int lane = threadIdx.x & 63;
  if (workgroups == 0) {   // a list each
    Segment s;
    s.head = blockIdx.x;
    s.b = s.head / sh.Hkv;
    s.j = s.head % sh.Hkv;
    s.M = min(active_rows(in, kv, sh, s.b), min(sh.rows_max, part.rows));
    const Sequence seq = sequence(kv, sh, s.b);
    s.base = seq.base;
    s.tokens = seq.tokens;
    s.seq_pages = seq.pages;
    s.pages = in.list ? max(0, min(min(in.sel_count[s.head], in.cap), sh.max_pages)) : seq.pages;
    s.t0 = 0;
    s.t1 = (s.pages + PPT - 1) / PPT;
    s.item = -1;
    if (s.M > 0) f(s);
    return;
  }
  // the plan in LDS, two int4 per head: every wavefront makes it, all of them the same
  int4* const heads_plan = reinterpret_cast<int4*>(plan);
  int total = 0, most_unit = 1;
  for (int h0 = 0; h0 < heads; h0 += 64) {
    const int h = min(h0 + lane, heads - 1), b = quotient(h, sh.Hkv);
    int n = (in.active_count ? in.active_count : kv.seq_lens)[b], listed = *(in.list ? in.sel_count + h : kv.seq_lens + b);
    const Sequence seq = sequence_of(kv, sh, b);
    n = (in.active_count ? min(n, sh.B) : sh.B) * sh.G;
    const int M = h0 + lane < heads ? min(n, min(sh.rows_max, part.rows)) : 0, pages = in.list ? max(0, min(min(listed, in.cap), sh.max_pages)) : seq.pages;
    const int unit = unit_cost(M, BLOCK), tiles = M > 0 ? (pages + PPT - 1) / PPT : 0, cost = tiles > 0 ? (GAP + tiles) * unit : 0;
    const int incl = wave_inclusive_scan(cost);
    if (h0 + lane < heads) {
      heads_plan[2 * h] = make_int4(total + incl - tiles * unit, tiles, unit, pages);
      heads_plan[2 * h + 1] = make_int4(M, seq.base, seq.tokens, seq.pages);
    }
    total += __builtin_amdgcn_readlane(incl, 63);
    most_unit = max(most_unit, (int)wave_max_u32((uint32_t)unit));
  }
  wave_lds_fence();
  const int w = blockIdx.x, share = max((int)((float)total * (1.000001f * __builtin_amdgcn_rcpf((float)workgroups))) + 1, least_tiles * most_unit);   // (at least total / workgroups)
  const int begin = w * share, end = begin + share;
  int first = heads, last = -1;   // the lists that reach into the share
  for (int h0 = 0; h0 < heads; h0 += 64) {
    const int h = h0 + lane;
    const int4 p = heads_plan[2 * min(h, heads - 1)];
    const unsigned long long in_it = __ballot(h < heads && p.x < end && p.x + p.y * p.z > begin);
    if (in_it) {
      first = min(first, h0 + __builtin_ctzll(in_it));
      last = h0 + 63 - __builtin_clzll(in_it);
    }
    if (w == 0 && threadIdx.x < 64 && h < heads) {
      const int from = quotient(p.x, share);
      out.table[h] = make_int2(from + h, p.y > 0 ? quotient(p.x + (p.y - 1) * p.z, share) - from + 1 : 0);
    }
  }
  for (int h = first; h <= last; ++h) {
    const int4 p = heads_plan[2 * h], more = heads_plan[2 * h + 1];
    const int start = __builtin_amdgcn_readfirstlane(p.x), tiles = __builtin_amdgcn_readfirstlane(p.y), unit = __builtin_amdgcn_readfirstlane(p.z);
    if (tiles == 0) continue;
    Segment s;   // (uniform, as the compiler does not see by itself)
    s.head = __builtin_amdgcn_readfirstlane(h);
    s.b = __builtin_amdgcn_readfirstlane(quotient(h, sh.Hkv));
    s.j = __builtin_amdgcn_readfirstlane(s.head - s.b * sh.Hkv);
    s.pages = __builtin_amdgcn_readfirstlane(p.w);
    s.M = __builtin_amdgcn_readfirstlane(more.x);
    s.base = __builtin_amdgcn_readfirstlane(more.y);
    s.tokens = __builtin_amdgcn_readfirstlane(more.z);
    s.seq_pages = __builtin_amdgcn_readfirstlane(more.w);
    s.t0 = begin <= start ? 0 : __builtin_amdgcn_readfirstlane(quotient(begin - start + unit - 1, unit));
    s.t1 = min(tiles, __builtin_amdgcn_readfirstlane(quotient(end - start + unit - 1, unit)));
    if (s.t0 >= s.t1) continue;
    s.item = s.t0 == 0 && s.t1 == tiles ? -1 : w + s.head;
    f(s);
  }
}

// The block token of row r of a sequence, and the output row that is (negative: none).
__device__ __forceinline__ int token_of(const Shape& sh, const AttnInputs& in, int b, int r) {
  const int a = row_token(sh, r);
  return in.active_idx ? in.active_idx[(size_t)b * sh.B + a] : a;
}
__device__ __forceinline__ long output_row(const Shape& sh, int b, int j, int r, int tok) {
  return (unsigned)tok < (unsigned)sh.B ? ((long)b * sh.B + tok) * sh.Hq + j * sh.G + (r - row_token(sh, r) * sh.G) : -1;
}
template <int D>
__device__ __forceinline__ void store_output(const PackedOut& out, long row, int channel, f32x4_t acc, float m, float l) {
  if (row < 0) return;
  const bool any = m > -1.0e29f || l != l;   // no valid token at all: the neutral element of a merge.  (Scores that are all NaN move no reference)
  *reinterpret_cast<f32x4_t*>(out.o_p + row * D + channel) = any ? acc / l : (f32x4_t){0.f, 0.f, 0.f, 0.f};
  if (channel == 0) out.lse_p[row] = any ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
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
  store_output<D>(out, output_row(sh, s.b, s.j, r, token_of(sh, in, s.b, r)), channel, acc, m, l);
}

// Sixteen bytes a lane from `base` + offset to LDS at `to` + 16 lane, without a register on the way.  The wavefront waits for them itself (landed()).
// (In assembly, as the compiler waits for all of them ahead of any LDS read; there is no output that it could take for written.  It keeps nothing
// in M0 from one instruction to another.)
__device__ __forceinline__ void start_to_lds(const uint8_t* base, uint32_t offset, uint32_t to) {
  const uint64_t at = (uint64_t)(uintptr_t)base;
  const uint64_t uniform = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(offset), "s"(uniform), "s"(to) : "memory");
}
// ... from an address of each lane's own: two pages are any distance apart, in either direction, and an offset is 32 bits without a sign.
__device__ __forceinline__ void start_to_lds(const uint8_t* lane_address, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(lane_address), "s"(to) : "memory");
}
// All but the last N of them are there.
template <int N>
__device__ __forceinline__ void landed() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Query rows row0 .. row0 + 16 R - 1 of a (sequence, KV head): what a workgroup of up to 64 rows does.  Its four wavefronts deal the share's tiles out.  Two
// workgroups fit a compute unit, so that one's way to its first tile and the joining of its wavefronts' states, some 10 us together, run beside the
// other's tiles.  That takes 256 registers a lane and 80 KiB of LDS at most:
//   tiles come into LDS, a ring of kRing per wavefront, all but two of them on their way;
//   the query fragments are read from LDS for every tile where there are more than two row tiles (or float queries).
// Four row tiles do not fit.  They are two sets of two (SETS): a wavefront of each set takes every tile, which reads its codes from
// the cache the second time and converts them twice, 128 of some 240 vector instructions a tile.
// One row of 7 queries against 131072 tokens of 4 heads: 24 us with the join, 71 MB (14 at a large copy's rate; the rest is the way to the first tile and the end).  35 rows a
// head, 16 sequences of 8191 to 32768 tokens, a third of the pages: 37 us with the join, of which the matrix core works some 20 (48 rows'
// products, those with probabilities twice); a workgroup's wavefronts sharing tiles through LDS took 65, eight wavefronts dealing them out 42.
constexpr int kWaves = 4, kDealtGap = 16;
template <int R, int D, int NQ, int SETS = 1>
struct DealtLds {
  static constexpr bool kQueries = R > 2 || NQ > 1;
  static constexpr int kState = R * (D / 16) * 256 + 2 * R * 16;                    // floats: O as [row tile][channel tile][lane] vectors, references, sums
  static constexpr int kQueryFloats = kQueries ? NQ * R * (D / 32) * 256 : 0;
  static constexpr int kTile = 32 * D + 64 * (D / 32);                              // bytes of a tile: keys, values, scales
  // two workgroups to a compute unit, with the plan of some 64 heads each
  static constexpr int kRoom = 80 * 1024 - 64 * 32 - kQueryFloats * 4;
  static constexpr int kRing = kRoom >= kWaves * 4 * kTile ? 4 : 3;                 // tiles
  // LDS images of the wavefronts' states: all of them, or where there is no room for that half (each wavefront of the second half hands its state
  // to one of the first, before those hand theirs to everybody)
  static constexpr bool kAll = kRoom >= kWaves * kState * 4;
  static constexpr int kSlots = (kAll ? kWaves : kWaves / 2) / SETS;                // of a set
  static constexpr int kRingBytes = kWaves * kRing * kTile, kStateBytes = SETS * kSlots * kState * 4;   // (one after the other in the same place)
  static constexpr int kBytes = kQueryFloats * 4 + (kRingBytes > kStateBytes ? kRingBytes : kStateBytes);
};
template <int D, int GP, int R, int NQ, int SETS = 1>
__device__ __forceinline__ void packed_attn_body(const KvView& kv, const Shape& sh, const AttnInputs& in, const PackedView& pk, const Segment& seg, int row_base,
                                                 const Partials& part, const PackedOut& out, float scale_log2e, float* lds) {
  constexpr int WAVES = kWaves / SETS;   // of a set
  constexpr int KS = D / 32, NT = D / 16, J = D / 32, W = D / 32;   // products per score, channel tiles, groups, dwords a lane has of a subtile
  constexpr int CPL = D / 4;                                        // channels of a token that a lane has
  constexpr int PPT = 32 / GP, TPR = 64 / PPT;                      // pages per tile, tiles per fetch of page entries
  constexpr int kPageBytes = GP * D / 2, kPageScales = 2 * GP * J;
  typedef DealtLds<R, D, NQ, SETS> Lds;
  static_assert(SETS == 1 || (!Lds::kQueries && Lds::kAll), "the sets' queries are not the same, and a wavefront hands its state to one of its set");
  constexpr int kRing = Lds::kRing;
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));   // (what derives from it is worked out per segment, not kept in registers over all of them)
  const int in_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = in_group % WAVES, set = in_group / WAVES;
  const int l16 = lane & 15, qd = lane >> 4;
  const int b = seg.b, j = seg.j, M = seg.M, row0 = row_base + set * (R * 16);
  // tiles are dealt round-robin to the wavefronts
  const int tfirst = seg.t0 + wave, ntw = tfirst < seg.t1 ? (seg.t1 - 1 - tfirst) / WAVES + 1 : 0;

  // ---- pages of this wavefront's next TPR tiles, one per lane: list entry, page table, decoded
  int pg_phys = 0, pg_valid = 0;
  auto listed = [&](int n0) {
    const int at = (tfirst + (n0 + lane / PPT) * WAVES) * PPT + lane % PPT;
    int logical = at < seg.pages ? at : -1;
    if (in.list && at < seg.pages) logical = in.list[(size_t)seg.head * in.cap + at];
    return logical;
  };
  auto entry = [&](int logical) { return (unsigned)logical < (unsigned)seg.seq_pages ? kv.page_indices[seg.base + logical] : -1; };
  auto decode = [&](int logical, int phys) {
    const bool ok = (unsigned)phys < (unsigned)kv.num_pages;
    pg_phys = ok ? phys : 0;
    pg_valid = ok ? min(GP, seg.tokens - logical * GP) : 0;
  };

  // ---- the way to the first tile: list entries and the query rows' tokens, then page table and query rows, each pair in one memory round trip
  constexpr int kFragments = R * KS, kOwn = Lds::kQueries ? (kFragments + WAVES - 1) / WAVES : kFragments;   // of queries; that this wavefront fetches
  const int logical = listed(0);
  int tok[Lds::kQueries ? kOwn : R];
#pragma unroll
  for (int i = 0; i < (Lds::kQueries ? kOwn : R); ++i) {
    const int mt = Lds::kQueries ? (wave + i * WAVES) / KS : i, a = row_token(sh, min(row0 + mt * 16 + l16, sh.rows_max - 1));
    tok[i] = in.active_idx ? in.active_idx[(size_t)b * sh.B + a] : a;
  }
  const int phys = entry(logical);
  uint4 q_raw[kOwn][NQ == 1 ? 1 : 2];
  bool q_keep[kOwn];
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const int f = Lds::kQueries ? wave + i * WAVES : i, mt = f / KS, ks = f % KS, t = tok[Lds::kQueries ? i : mt];
    const int r = row0 + mt * 16 + l16, rr = min(r, sh.rows_max - 1);
    q_keep[i] = r < M && (unsigned)t < (unsigned)sh.B;
    const size_t at = (((size_t)b * sh.B + (q_keep[i] ? t : 0)) * sh.Hq + j * sh.G + (rr - row_token(sh, rr) * sh.G)) * D + qd * CPL + ks * 8;
    if constexpr (NQ == 1) {
      q_raw[i][0] = *reinterpret_cast<const uint4*>((const bf16_t*)in.q + at);
    } else {
      q_raw[i][0] = *reinterpret_cast<const uint4*>((const float*)in.q + at);
      q_raw[i][1] = *reinterpret_cast<const uint4*>((const float*)in.q + at + 4);
    }
  }
  decode(logical, phys);

  // ---- the ring: keys of subtiles 0 and 1, values of both, scales as they lie
  constexpr int kLoads = D == 128 ? 5 : 3;   // loads per tile
  char* const ring = reinterpret_cast<char*>(lds + Lds::kQueryFloats) + in_group * (kRing * Lds::kTile);
  const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring;
  int nv[kRing][2];   // valid tokens of the subtiles of the tiles n, n + 1, ... (the first kRing - 1 of them before tile n + kRing - 1 is started)
  auto start_tile = [&](int n, int slot) {
    const int e0 = GP == 16 ? (2 * n) & 63 : n & 63, e1 = GP == 16 ? e0 + 1 : e0;
    int p0 = __builtin_amdgcn_readlane(pg_phys, e0), p1 = __builtin_amdgcn_readlane(pg_phys, e1);
    nv[kRing - 1][0] = __builtin_amdgcn_readlane(pg_valid, e0);
    nv[kRing - 1][1] = GP == 16 ? __builtin_amdgcn_readlane(pg_valid, e1) : nv[kRing - 1][0] - 16;
    // (a tile that does not exist: the pool's first page, so that the loads on their way are the same number always)
    p0 = n < ntw ? p0 : 0;
    p1 = n < ntw ? p1 : 0;
    const size_t t0 = (size_t)p0 * sh.Hkv + j, t1 = (size_t)p1 * sh.Hkv + j;
    const uint32_t to = ring_at + slot * Lds::kTile;
    if constexpr (D == 128) {
      const uint32_t key = l16 * 64 + qd * 16, value = lane * 16, second = GP == 16 ? 0 : 1024;
      start_to_lds(pk.k + t0 * kPageBytes, key, to);
      start_to_lds(pk.k + t1 * kPageBytes + second, key, to + 1024);
      start_to_lds(pk.v + t0 * kPageBytes, value, to + 2 * 1024);
      start_to_lds(pk.v + t1 * kPageBytes + second, value, to + 3 * 1024);
    } else {
      // two pages' 512 bytes are a load: lanes 32 .. 63 have the second's
      const size_t from = GP == 16 ? (lane < 32 ? t0 : t1) * kPageBytes + (lane & 31) * 16 : t0 * kPageBytes + lane * 16;
      start_to_lds(pk.k + from, to);
      start_to_lds(pk.v + from, to + 1024);
    }
    constexpr int kPieces = kPageScales / 16;   // of a page
    if (lane < kPieces * PPT)
      start_to_lds(pk.scales + (lane < kPieces ? t0 : t1) * kPageScales + lane % kPieces * 16, to + 32 * D);
  };
  auto start_first = [&](int n) {
    start_tile(n, n);
    nv[n][0] = nv[kRing - 1][0];
    nv[n][1] = nv[kRing - 1][1];
  };
  start_first(0);

  // ---- query rows, in the order the keys' channels are contracted in: fragment (row tile, product), its terms
  bf16x8_t qf[Lds::kQueries ? 1 : R][NQ][KS];
  const bf16x8_t* const q_lds = reinterpret_cast<const bf16x8_t*>(lds);
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    bf16x8_t term[NQ];
    if constexpr (NQ == 1) {
      uint4 x = q_raw[i][0];
      if (!q_keep[i]) x = make_uint4(0u, 0u, 0u, 0u);
      term[0] = __builtin_bit_cast(bf16x8_t, x);
    } else {
      const uint4 lo = q_raw[i][0], hi = q_raw[i][1];
      const uint32_t bits[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = q_keep[i] ? __uint_as_float(bits[e]) : 0.f;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          term[n][e] = (__bf16)x;
          x -= (float)term[n][e];
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      if constexpr (Lds::kQueries) {
        const int f = wave + i * WAVES;
        if (f < kFragments) reinterpret_cast<bf16x8_t*>(lds)[(f * NQ + n) * 64 + lane] = term[n];
      } else {
        qf[i / KS][n][i % KS] = term[n];
      }
    }
  }
#pragma unroll
  for (int n = 1; n < kRing - 1; ++n) start_first(n);
  if constexpr (Lds::kQueries) __syncthreads();

  float m_run[R], up_thr[R];
  const float inv_scale_log2e = 1.0f / scale_log2e;
  f32x4_t o[R][NT], l_sum[R];   // (a row's sum in all four components)
#pragma unroll
  for (int mt = 0; mt < R; ++mt) {
    m_run[mt] = kNegBig;
    up_thr[mt] = -INFINITY;
    l_sum[mt] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) o[mt][nt] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  }

  // Scores of the tile in ring slot `slot`.
  auto score = [&](int slot, f32x4_t (&sc)[R][2]) {
    const char* tile = ring + slot * Lds::kTile;
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(tile + 32 * D);
    bf16x8_t kf[2][KS];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint32_t c[W];
      lds_dwords<W>(tile + (D == 128 ? s * 1024 + lane * 16 : s * 512 + l16 * 32 + qd * 8), c);
      const float scale = power_of(scales[(GP == 16 ? s * kPageScales + l16 * J : (16 * s + l16) * J) + qd * CPL / 32]);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        kf[s][ks] = __builtin_bit_cast(bf16x8_t, make_uint4(codes_to_bf16<0>(c[ks], scale), codes_to_bf16<1>(c[ks], scale),
                                                            codes_to_bf16<2>(c[ks], scale), codes_to_bf16<3>(c[ks], scale)));
    }
#pragma unroll
    for (int mt = 0; mt < R; ++mt) {
      sc[mt][0] = sc[mt][1] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int t = NQ - 1; t >= 0; --t) {
          bf16x8_t q;
          if constexpr (Lds::kQueries)
            q = q_lds[((mt * KS + ks) * NQ + t) * 64 + lane];
          else
            q = qf[mt][t][ks];
          sc[mt][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[0][ks], q, sc[mt][0], 0, 0, 0);
          sc[mt][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[1][ks], q, sc[mt][1], 0, 0, 0);
        }
    }
  };
  // A tile's scores are made beside the numerators and value products of the one before it: the matrix core works on the ones while the vector units
  // work on the others.
  f32x4_t sc[R][2];
  landed<kLoads * (kRing - 2)>();
  score(0, sc);
  int slot_now = 0, slot_start = kRing - 1;
  for (int n = 0; n < ntw; ++n) {
    if ((n + kRing - 1) % TPR == 0) {   // (the entries are decoded behind the branch, so nothing waits where it joins)
      const int next = listed(n + kRing - 1);
      decode(next, entry(next));
    }
    start_tile(n + kRing - 1, slot_start);
    const char* tile = ring + slot_now * Lds::kTile;
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(tile + 32 * D);
    uint32_t vc[2][W], vs[2][4];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      lds_dwords<W>(tile + 16 * D + (D == 128 ? s * 1024 + lane * 16 : s * 512 + lane * 8), vc[s]);
      load_scales<J>(scales + (GP == 16 ? s * kPageScales + GP * J + qd * 4 * J : GP * J + (16 * s + qd * 4) * J), vs[s]);
    }
    if (!(nv[0][0] >= 16 && nv[0][1] >= 16)) {   // slots behind the sequence's end may hold anything
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool there = qd * 4 + e < nv[0][s];
          vs[s][e] = there ? vs[s][e] : 0u;   // (the smallest scale: nothing, in half precision)
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
      tm[mt] = fmaxf(fmaxf(fmaxf(fmaxf(a[0], a[1]), a[2]), fmaxf(fmaxf(a[3], c[0]), c[1])), fmaxf(c[2], c[3]));
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
        l_sum[mt] *= alpha;
        if (n > 0) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) o[mt][nt] *= alpha;
        }
      }
    }
    landed<kLoads * (kRing - 2)>();   // the next tile
    slot_start = slot_now;
    slot_now = slot_now == kRing - 1 ? 0 : slot_now + 1;
    f32x4_t next_sc[R][2];
    score(slot_now, next_sc);         // (behind the last tile: of the pool's first page, for nothing)
    f16x8_t p_hi[R], p_lo[R];
#pragma unroll
    for (int mt = 0; mt < R; ++mt) {
      numerators(sc[mt][0], sc[mt][1], scale_log2e, -m_run[mt], p_hi[mt], p_lo[mt]);
      l_sum[mt] = sum_of(p_hi[mt], p_lo[mt], l_sum[mt]);
    }
#pragma unroll
    for (int g = 0; g < J; ++g) {
      uint2 lo[2], hi[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) value_operands(vc[s][g], vs[s], g, lo[s], hi[s]);
      const f16x8_t va = __builtin_bit_cast(f16x8_t, make_uint4(lo[0].x, lo[0].y, lo[1].x, lo[1].y));
      const f16x8_t vb = __builtin_bit_cast(f16x8_t, make_uint4(hi[0].x, hi[0].y, hi[1].x, hi[1].y));
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
    // one matrix instruction, a few vector ones, in turn (and a query fragment from LDS just ahead of its product, not all of them)
#pragma unroll
    for (int i = 0; i < R * (2 * KS * NQ + 2 * NT + 2); ++i) {
      if (Lds::kQueries && i < R * 2 * KS * NQ && i % 2 == 0) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
    }
#pragma unroll
    for (int mt = 0; mt < R; ++mt) {
      sc[mt][0] = next_sc[mt][0];
      sc[mt][1] = next_sc[mt][1];
    }
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) {
      nv[i][0] = nv[i + 1][0];
      nv[i][1] = nv[i + 1][1];
    }
  }

  // ---- the wavefronts' states become one partial, in a fixed order, each wavefront making some of its vectors
  landed<0>();
  __syncthreads();   // the rings' place is the states' now
  float l_run[R];
#pragma unroll
  for (int mt = 0; mt < R; ++mt) l_run[mt] = l_sum[mt][0];
  float* const states = lds + Lds::kQueryFloats;
  constexpr int kSlots = Lds::kSlots;
  float* const slot = states + (Lds::kAll ? in_group : wave % kSlots) * Lds::kState;
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
  if constexpr (!Lds::kAll) {
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
// them once for all rows and leaves them in LDS as the matrix core's operands, 16 bytes a lane, in lane order.  A barrier per stage, two LDS buffers of
// keys and three of values (see compute_stage); the codes of the next kAhead stages are on their way in registers.
//
// Bound by the matrix core: three products per useful two, the values' being with pairs of halves.  64 tokens' queries against four prefixes of 65536 (256 rows, 8 KV heads) take
// 323 us, 1.28 PFLOP/s executed, which is what a large bfloat16 product of the library's reaches here.  Reading each operand, waiting for it and using it took
// 413 us; scores, numerators and products one after the other, each for all of a stage, 371.
template <int D>
constexpr int kKeyBytes = 64 * D * 2;   // of a stage, and as many of values
template <int D>
constexpr int kStagedBytes = 5 * kKeyBytes<D>;
constexpr int kAhead = 2;

// use(n, operand) for operands 0 .. N-1, 16 bytes a lane and 1024 bytes apart in LDS, each read kReadsAhead uses before its own.  (Left to its own order,
// the compiler reads one, waits for it and uses it.)
constexpr int kReadsAhead = 2;
template <typename V, int N, typename F>
__device__ __forceinline__ void with_operands(const char* from, F&& use) {
  V x[kReadsAhead + 1];
#pragma unroll
  for (int n = 0; n < kReadsAhead; ++n) x[n] = *reinterpret_cast<const V*>(from + n * 1024);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if (n + kReadsAhead < N) x[(n + kReadsAhead) % (kReadsAhead + 1)] = *reinterpret_cast<const V*>(from + (n + kReadsAhead) * 1024);
    __builtin_amdgcn_sched_barrier(0);
    use(n, x[n % (kReadsAhead + 1)]);
  }
  __builtin_amdgcn_sched_barrier(0);
}

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
    if ((unsigned)logical < (unsigned)seg.seq_pages) phys = kv.page_indices[seg.base + logical];
    const bool ok = (unsigned)phys < (unsigned)kv.num_pages;
    pg_phys = ok ? phys : 0;
    pg_valid = ok ? min(GP, seg.tokens - logical * GP) : 0;
  };
  // valid tokens of subtile s of stage i (of the TPR tiles at hand)
  auto valid_of = [&](int i, int s) {
    const int at = (2 * i + s / 2) * PPT;
    return GP == 16 ? __builtin_amdgcn_readlane(pg_valid, (at + s % 2) & 63) : __builtin_amdgcn_readlane(pg_valid, at & 63) - 16 * (s % 2);
  };

  struct Raw {
    uint32_t c[W], vs[4], ks;   // codes of keys or of values
  };
  // Of two wavefronts on a SIMD the older one has the way free, so the younger ones (4 .. 7) get the shorter conversions, and precedence: without
  // either they were at work for 5400 cycles a stage, the others for 4000, of 5650.
  const bool has_keys = wave >= 4;
  if (has_keys) __builtin_amdgcn_s_setprio(1);
  const int mysub = wave & 3;
  const uint32_t code_at = has_keys ? l16 * (D / 2) + qd * (CPL / 2) : (qd * 16 + l16) * (J * 4);   // (a tile's first 16 tokens)
  const uint32_t key_scale_at = l16 * J + qd * CPL / 32, scales_at = GP * J + qd * 4 * J;
  auto load_stage = [&](Raw& x, int i) {   // (past the end: the pool's first page, as nothing depends on it)
    const int at = ((2 * i + mysub / 2) * PPT + (GP == 16 ? mysub % 2 : 0)) & 63;
    const size_t tile = (size_t)__builtin_amdgcn_readlane(pg_phys, at) * sh.Hkv + j;
    const int row = GP == 16 ? 0 : 16 * (mysub % 2);
    const uint8_t* sc = pk.scales + tile * (2 * GP * J) + row * J;
    load_dwords<W>((has_keys ? pk.k : pk.v) + tile * kTileBytes + row * (D / 2) + code_at, x.c);   // (16 tokens are as many bytes in either order)
    x.ks = sc[key_scale_at];   // (one of the two in vain: no branch around a load)
    load_scales<J>(sc + scales_at, x.vs);
  };
  auto convert_stage = [&](Raw& x, int i, char* keys, char* values) {
    if (has_keys) {
      const float scale = power_of(x.ks);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        *reinterpret_cast<uint4*>(keys + ((mysub * KS + ks) * 64 + lane) * 16) =
            make_uint4(codes_to_bf16<0>(x.c[ks], scale), codes_to_bf16<1>(x.c[ks], scale), codes_to_bf16<2>(x.c[ks], scale), codes_to_bf16<3>(x.c[ks], scale));
    }
    if (!has_keys) {
      const int valid = valid_of(i, mysub);
#pragma unroll
      for (int e = 0; e < 4; ++e) x.vs[e] = qd * 4 + e < valid ? x.vs[e] : 0u;   // (see the other form)
      char* v = values + ((mysub / 2) * NT * 64 + lane) * 16 + (mysub % 2) * 8;
#pragma unroll
      for (int g = 0; g < J; ++g) {
        uint2 lo, hi;
        value_operands(x.c[g], x.vs, g, lo, hi);
        *reinterpret_cast<uint2*>(v + (2 * g) * 1024) = lo;
        *reinterpret_cast<uint2*>(v + (2 * g + 1) * 1024) = hi;
      }
    }
  };

  float m_run[R], up_thr[R], l_run[R];   // l_run: of this lane's tokens
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

  // A stage: scores and their maxima, then for its two pairs of subtiles numerators and their products with the values.  The matrix core works on a pair's
  // products while the vector units make the next pair's numerators, so the second pair's products come with the next stage's first numerators.
  f32x4_t sc[R][4];
  f16x8_t p_hi[2][R], p_lo[2][R];
#pragma unroll
  for (int mt = 0; mt < R; ++mt)
#pragma unroll
    for (int e = 0; e < 8; ++e) p_hi[1][mt][e] = p_lo[1][mt][e] = (_Float16)0.f;   // (ahead of the first stage: nothing, times that stage's values)
  char* values[3] = {lds + 2 * kKeyBytes<D>, lds + 3 * kKeyBytes<D>, lds + 4 * kKeyBytes<D>};   // the last stage's, this one's, the next one's
  auto numerators_of = [&](int pair, int i) {   // scores 2 i' and 2 i' + 1, i' = i % 4, of row tile i / 4
    const int mt = i / 4, e = 2 * (i % 4);
    const f32x4_t& s = sc[mt][2 * pair + e / 4];
    l_run[mt] += numerator_pair(s[e & 3], s[(e & 3) + 1], scale_log2e, -m_run[mt], e, p_hi[pair][mt], p_lo[pair][mt]);
  };
  auto products_of = [&](int pair, const char* from, auto&& beside) {   // beside(n) goes with channels 16 n and the next 15
    with_operands<f16x8_t, NT>(from + (pair * NT * 64 + lane) * 16, [&](int n, const f16x8_t& vf) {
#pragma unroll
      for (int mt = 0; mt < R; ++mt) o[mt][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p_hi[pair][mt], o[mt][n], 0, 0, 0);
#pragma unroll
      for (int mt = 0; mt < R; ++mt) o[mt][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, p_lo[pair][mt], o[mt][n], 0, 0, 0);
      beside(n);
    });
  };
  auto numerators_beside = [&](int pair) {
    return [&, pair](int n) {
#pragma unroll
      for (int i = n * 4 * R / NT; i < (n + 1) * 4 * R / NT; ++i) numerators_of(pair, i);
    };
  };
  auto compute_stage = [&](int i, const char* keys, const char* last_values) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int mt = 0; mt < R; ++mt) sc[mt][s] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    with_operands<bf16x8_t, 4 * KS>(keys + lane * 16, [&](int n, const bf16x8_t& kf) {   // subtile n / KS, channels n % KS
#pragma unroll
      for (int mt = 0; mt < R; ++mt) sc[mt][n / KS] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[mt][n % KS], sc[mt][n / KS], 0, 0, 0);
    });
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
    float alpha[R];
    const bool rescale = __any(any_up);
    if (rescale) {
#pragma unroll
      for (int mt = 0; mt < R; ++mt) {
        const float cand = over_lane_groups_max(tm[mt]) * scale_log2e - kHeadroom;
        const bool up = cand > m_run[mt] + kLag;
        alpha[mt] = up ? __builtin_amdgcn_exp2f(m_run[mt] - cand) : 1.0f;
        m_run[mt] = up ? cand : m_run[mt];
        up_thr[mt] = (m_run[mt] + kHeadroom + kLag) * inv_scale_log2e;
        l_run[mt] *= alpha[mt];
      }
    }
    products_of(1, last_values, numerators_beside(0));
    if (rescale) {   // (what was owed was against the old reference)
#pragma unroll
      for (int mt = 0; mt < R; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[mt][nt] *= alpha[mt];
    }
    products_of(0, values[1], numerators_beside(1));
  };

  constexpr int SPF = TPR / 2;   // stages per fetch of page entries
  Raw raw[kAhead];
  for (int n0 = 0; n0 < stages; n0 += SPF) {
    const int ne = min(stages - n0, SPF);   // stages of this fetch, counted from its first
    fetch_pages(2 * n0);
    if (n0 > 0) __syncthreads();            // the buffers' last readers are done
#pragma unroll
    for (int k = 0; k < kAhead; ++k) load_stage(raw[k], k);
    convert_stage(raw[0], 0, lds, values[1]);
    load_stage(raw[0], kAhead);
    __syncthreads();
    for (int i = 0; i < ne; i += 2) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // Stage i + k's keys are in buffer k, the next one's go to the other.  (Whether there is one or not: loads behind a branch, or a use of theirs,
        // would be waited for where the branches join.)
        convert_stage(raw[(k + 1) % kAhead], i + k + 1, lds + (1 - k) * kKeyBytes<D>, values[2]);
        load_stage(raw[(k + 1) % kAhead], i + k + 1 + kAhead);
        if (i + k == ne) break;   // (the last fetch's last: values[0] is still the last stage's)
        if (has_rows) compute_stage(i + k, lds + k * kKeyBytes<D>, values[n0 + i + k == 0 ? 1 : 0]);
        __syncthreads();
        char* const free = values[0];
        values[0] = values[1];
        values[1] = values[2];
        values[2] = free;
      }
    }
  }
  if (has_rows && stages > 0) products_of(1, values[0], [](int) {});
  __syncthreads();   // the LDS is the next segment's

#pragma unroll
  for (int mt = 0; mt < R; ++mt) {
    const int r = row0 + mt * 16 + l16;
    const float l = over_lane_groups_sum(l_run[mt]);
    if (r >= M) continue;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) store_state<D>(sh, in, part, out, seg, r, nt * 16 + qd * 4, o[mt][nt], m_run[mt], l);
  }
}

#define LOSA_PACKED_ARGS KvView kv, Shape sh, AttnInputs in, PackedView pk, Partials part, PackedOut out, float scale_log2e, int heads, int workgroups, int least_tiles
// Rows that the host knows: blocks of SETS * R row tiles, one after the other.
template <int D, int GP, int R, int NQ, int SETS = 1>
__global__ __launch_bounds__(64 * kWaves) void packed_attn_kernel(LOSA_PACKED_ARGS) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  constexpr int kRows = SETS * R * 16;
  int* plan = reinterpret_cast<int*>(lds) + DealtLds<R, D, NQ, SETS>::kBytes / 4;
  for_each_segment<GP, kRows, kDealtGap>(kv, sh, in, part, out, heads, workgroups, least_tiles, plan, [&](const Segment& s) {
    for (int row0 = 0; row0 < s.M; row0 += kRows) packed_attn_body<D, GP, R, NQ, SETS>(kv, sh, in, pk, s, row0, part, out, scale_log2e, lds);
  });
}
// ... blocks of 8 * R row tiles.
template <int D, int GP, int R>
__global__ __launch_bounds__(512) void packed_rows_kernel(LOSA_PACKED_ARGS) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  constexpr int kRows = 128 * R;
  int* plan = reinterpret_cast<int*>(lds) + kStagedBytes<D> / 4;
  for_each_segment<GP, kRows, 4>(kv, sh, in, part, out, heads, workgroups, least_tiles, plan, [&](const Segment& s) {
    for (int row0 = 0; row0 < s.M; row0 += kRows) packed_rows_body<D, GP, R>(kv, sh, in, pk, s, row0, part, out, scale_log2e, reinterpret_cast<char*>(lds));
  });
}
// Rows counted on the device: the form made for the rows a head has, block after block.
template <int NQ>
constexpr int kCountedRows = NQ == 1 ? 64 : 32;
template <int D, int NQ>
constexpr int kCountedBytes = NQ == 1 ? std::max(DealtLds<3, D, 1>::kBytes, DealtLds<2, D, 1, 2>::kBytes) : DealtLds<2, D, NQ>::kBytes;
template <int D, int GP, int NQ>
__global__ __launch_bounds__(64 * kWaves) void packed_attn_counted_kernel(LOSA_PACKED_ARGS) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  int* plan = reinterpret_cast<int*>(lds) + kCountedBytes<D, NQ> / 4;
  for_each_segment<GP, kCountedRows<NQ>, kDealtGap>(kv, sh, in, part, out, heads, workgroups, least_tiles, plan, [&](const Segment& s) {
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

// ---- joins a list's partials, in the order of the items.  D / 4 threads have a row's channels, four each.  Up to kFewItems items: those threads take all of them
// one after the other, eight requested at once, and a workgroup has 1024 / D rows.  More: a workgroup has a row, 1024 / D lanes of items.
constexpr int kFewItems = 16;
template <int D>
__global__ __launch_bounds__(256) void packed_join_kernel(KvView kv, Shape sh, AttnInputs in, Partials part, PackedOut out) {
  constexpr int C4 = D / 4, CL = 256 / C4, KB = 8;
  __shared__ __attribute__((aligned(16))) float4 red[CL][C4];
  __shared__ float2 stats[CL];
  const int tid = threadIdx.x, cl = tid / C4, c4 = tid % C4, head = blockIdx.y, b = head / sh.Hkv;
  const int j = head - b * sh.Hkv;
  // asked for with the counts: the token of a thread's first row, of which it has one only as a rule
  const int first_r = min((int)blockIdx.x * CL + cl, sh.rows_max - 1), first_tok = token_of(sh, in, b, first_r);
  int n = __builtin_amdgcn_readfirstlane((in.active_count ? in.active_count : kv.seq_lens)[b]);
  int first = __builtin_amdgcn_readfirstlane(out.table[head].x), items = __builtin_amdgcn_readfirstlane(out.table[head].y);
  asm("" : "+s"(n), "+s"(first), "+s"(items) : "s"(sh.B), "s"(sh.G), "s"(sh.rows_max), "s"(part.rows), "s"(part.m), "s"(part.l), "s"(part.o));   // (one round trip; see Sequence)
  if (items == 1) return;   // finished already
  const int M = min((in.active_count ? min(n, sh.B) : sh.B) * sh.G, min(sh.rows_max, part.rows));
  const bool few = items <= kFewItems;
  // items lane, lane + step, ... of row r
  auto gather = [&](int r, int lane, int step, float& m, float& l, f32x4_t& acc) {
    m = kNegBig;
    l = 0.f;
    acc = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    for (int i0 = lane; i0 < items; i0 += step * KB) {
      float mk[KB], lk[KB];
      f32x4_t x[KB];
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const uint32_t prow = (uint32_t)(first + min(i0 + step * k, items - 1)) * part.rows + r;
        mk[k] = part.m[prow];
        lk[k] = part.l[prow];
        x[k] = reinterpret_cast<const f32x4_t*>(part.o + (size_t)prow * D)[c4];
      }
      float m_new = m;
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        if (i0 + step * k >= items) mk[k] = kNegBig, lk[k] = 0.f, x[k] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
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
  };
  if (few) {
    for (int r = blockIdx.x * CL + cl; r < M; r += gridDim.x * CL) {
      float m, l;
      f32x4_t acc;
      gather(r, 0, 1, m, l, acc);
      const int tok = r == first_r ? first_tok : token_of(sh, in, b, r);
      store_output<D>(out, output_row(sh, b, j, r, tok), c4 * 4, acc, m, l);
    }
    return;
  }
  for (int r = blockIdx.x; r < M; r += gridDim.x) {
    float m, l;
    f32x4_t acc;
    gather(r, cl, CL, m, l, acc);
    red[cl][c4] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (c4 == 0) stats[cl] = make_float2(m, l);
    __syncthreads();
    if (tid < C4) {
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
      store_output<D>(out, output_row(sh, b, j, r, token_of(sh, in, b, r)), c4 * 4, o, m_all, l_all);
    }
    __syncthreads();   // the LDS is the next row's
  }
}

typedef void (*PackedKernel)(LOSA_PACKED_ARGS);

template <int D, int GP>
static hipError_t launch_dg(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, const AttnInputs& in, const PackedView& pk, int heads, int workgroups,
                            int least_tiles, int rows, bool known, const Partials& part, const PackedOut& out) {
  auto go = [&](PackedKernel kern, int lds_bytes, bool& attr_set, int waves = kWaves) {
    const int all = lds_bytes + (workgroups ? heads * 32 : 0);   // the plan behind the kernel's own
    if (!attr_set) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes + kPlannedHeads * 32);
      if (e != hipSuccess) return e;
      attr_set = true;
    }
    kern<<<workgroups ? workgroups : heads, 64 * waves, all, st>>>(kv, sh, in, pk, part, out, sh.sm_scale * 1.4426950408889634f, heads, workgroups, least_tiles);
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
  return rows <= 128 ? go(packed_rows_kernel<D, GP, 1>, kStagedBytes<D>, set[8], 8) : go(packed_rows_kernel<D, GP, 2>, kStagedBytes<D>, set[9], 8);
}

hipError_t launch_packed_attn(hipStream_t st, int dtype, const KvView& kv, const Shape& sh, int batch, const AttnInputs& in, const PackedView& pk, int workgroups,
                              int least_tiles, int rows, bool rows_known, const Partials& part, const PackedOut& out) {
  const int heads = batch * sh.Hkv;
  if (heads <= 0 || rows <= 0) return hipSuccess;
  auto launch = sh.d == 128 ? (sh.g == 16 ? launch_dg<128, 16> : launch_dg<128, 32>) : (sh.g == 16 ? launch_dg<64, 16> : launch_dg<64, 32>);
  return launch(st, dtype, kv, sh, in, pk, heads, workgroups, least_tiles, rows, rows_known, part, out);
}

hipError_t launch_packed_join(hipStream_t st, const KvView& kv, const Shape& sh, int batch, const AttnInputs& in, int workgroups, int rows, bool rows_known,
                              const Partials& part, const PackedOut& out) {
  const int heads = batch * sh.Hkv, per_group = 1024 / sh.d, likely = rows_known ? rows : min(rows, 64);   // (rows that only the device counts are mostly few)
  // (how many items a list has is the device's to know; on average no more than these)
  const dim3 grid(workgroups / heads + 2 <= kFewItems ? (likely + per_group - 1) / per_group : likely, heads);
  if (sh.d == 128)
    packed_join_kernel<128><<<grid, 256, 0, st>>>(kv, sh, in, part, out);
  else
    packed_join_kernel<64><<<grid, 256, 0, st>>>(kv, sh, in, part, out);
  return hipGetLastError();
}

}  // namespace losa
