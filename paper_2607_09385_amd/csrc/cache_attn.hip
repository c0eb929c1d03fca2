// Attention of new queries over the paged 4-bit cache.
//
//   o_r = sum_j p_rj v_j,  p_rj = 2^(c q_r . k_j - m_r) / l_r,  c = scale log2 e
// over the keys j that row r sees, with the online softmax (running maximum m,
// running sum l in fp32) over pages of 64 tokens.
//
// Scores.  S^T = K Q^T on bf16 MFMAs, K's codes and their scale turned into bf16 two at a time,
// exactly.  The scaled MFMAs would take K as it is stored (and Q as two E4M3 parts), but they add
// the products of a lane group on a grid of 2^-13 of the largest one: where channels differ
// much in size a score was off by up to 2^-16 of the sum of its magnitudes, against 2^-23 here.
// They were as fast for tokens (64 ragged sequences 65.1 us against 67.1, 4 of 8000 tokens
// 18.1 both) and up to 6% faster for chunks (1000 queries against 12000 keys 227 against 241).
//
// A query row is a column of every result and its m, l and rescaling stay in the lanes
// l % 16 = row (32 in the kernel for chunks).  Any order of the channels will do for K as
// long as Q has the same, so lane (n = l % 16, q = l / 16) takes D / 4 consecutive channels of
// token n: one 16-byte load of codes (D = 128) straight into registers, with one scale byte.
//
// O^T += V^T P^T on bf16 MFMAs.  The scores arrive with tokens 4 q .. 4 q + 3 of each 16 in a
// lane, which is what the P^T operand takes when the tokens of a page are numbered in that
// order; V goes through LDS, where a transposing read of 4-bit elements gives each lane 16
// tokens of one channel in the same order.  V's scales differ from token to token, along the
// sum, so they go into the weights: p_rj 2^e_jg is formed once per group of 32 channels (an
// addition to the exponents: exact), and the codes alone are turned into bf16.  Weights are
// rounded to bf16, the precision of the MFMA's operands (off by 2^-8 of each weight at most, in
// either direction), as in this library's dense calls; l adds them before that rounding.  A
// second bf16 part of each weight would take the error of a bf16 output from 0.0020-0.0023 of it to
// the 0.0017 of its own rounding, for 8 to 18% of the time of tokens (16 x 32768 112 us to 121, 64 x
// 3000 42 to 48, 32 rows 53 to 74) and 20% of chunks (226 to 278).
//
// A page id outside the pool is a page without visible keys; keys behind the
// sequence's length are never visible, whatever their bytes.
#include "cache_common.h"

namespace steel {

namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// Rows r0 .. r1 - 1 of (b, g): their positions and the pages that any of them sees,
// [0, a_len) and [b0, b0 + count - a_len).  Positions are below 2^31 and, since a
// negative length counts as 0, not below -S_q.
struct Span {
  int keys;        // keys that exist
  int first;       // position of query 0
  int n;           // queries of the sequence
  int pmin, pmax;  // positions of the rows
  int a_len, b0, count;
};

__device__ __forceinline__ Span make_span(const CacheArgs& a, int b, int r0, int r1) {
  Span s;
  const int len = max(a.lens[b], 0);
  s.n = a.fresh == nullptr ? a.S_q : min(max(a.fresh[b], 0), a.S_q);
  s.keys = min(len, a.M * kBlk);
  s.first = len - s.n;
  s.pmin = s.first + r0 / a.G;
  s.pmax = s.first + min((r1 - 1) / a.G, s.n - 1);
  s.a_len = s.b0 = s.count = 0;
  if (s.pmax < s.pmin || s.pmax < 0) return s;
  int kend = (s.keys + kBlk - 1) / kBlk;
  if (a.causal) kend = min(kend, s.pmax / kBlk + 1);
  s.a_len = s.count = kend;
  if (a.win > 0) {
    s.a_len = min(a.sink, kend);
    s.b0 = max(s.a_len, max(s.pmin, 0) / kBlk - a.win + 1);
    s.count = s.a_len + max(min(kend, s.pmax / kBlk + 1) - s.b0, 0);
  }
  return s;
}

__device__ __forceinline__ int span_page(const Span& s, int i) {
  return i < s.a_len ? i : s.b0 + (i - s.a_len);
}

// Whether every row of the span sees every key of page kb.
__device__ __forceinline__ bool page_full(const CacheArgs& a, const Span& s, int kb) {
  const int end = (kb + 1) * kBlk;
  bool full = s.pmin >= 0 && end <= s.keys;
  if (a.causal) full = full && end - 1 <= s.pmin;
  if (a.win > 0 && kb >= a.sink) full = full && kb <= s.pmin / kBlk && kb > s.pmax / kBlk - a.win;
  return full;
}

// Last key of page kb (0 .. 63, or negative: none) that the query at position pos sees.
__device__ __forceinline__ int row_limit(const CacheArgs& a, const Span& s, int pos, int kb) {
  int last = s.keys - 1;
  if (a.causal) last = min(last, pos);
  if (a.win > 0 && kb >= a.sink && (kb > pos / kBlk || kb <= pos / kBlk - a.win)) last = -1;
  if (pos < 0) last = -1;
  return min(last - kb * kBlk, 63);
}

// Maximum and sum over the lanes l % 16 (the four lane groups of a row), added in the
// same order on all of them.
__device__ __forceinline__ float row_max(float x) {
  const unsigned u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return other_half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float row_sum(float x) {
  const unsigned u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return half_pair_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// Inclusive sum over the wave's lanes in order; maximum of x >= 0 over them in lane 63.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // the lanes 1, 2, 4, 8 before, in rows of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 of the row before, to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31, to rows 2 and 3
  return x;
}
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }
__device__ __forceinline__ int wave_top(int x) {
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return __builtin_amdgcn_readlane(x, 63);
}

// Whether a row that sees the keys 0 .. last of a page (last < 0: none) sees one of the set.
__device__ __forceinline__ bool sees_any(uint64_t set, int last) {
  return last >= 0 && (set & ((2ull << last) - 1)) != 0;
}

// A running maximum to subtract: 0 before the first key.
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }

// Two numbers rounded to bf16, in one register.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// 8 codes and their scale as 8 bf16 values.
__device__ __forceinline__ bf16x8 decode8(uint32_t w, float sc) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The thread number, computed where it stands: what follows from it at a list's end then
// holds no register over the pages.
__device__ __forceinline__ int thread_here() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

constexpr int kWaves = 4;
// Workgroups of k_cache_token per CU (one wave on each SIMD).
constexpr int waves_per_simd(int D, int NT) { return NT == 1 ? 3 : 2; }
constexpr float kTau = 8.f;  // see the running maximum below

// One page's K codes and scales of a wave, on their way to registers.
template <int D>
struct PageRegs {
  typedef unsigned Codes __attribute__((ext_vector_type(D / 32)));
  Codes k0, k1, k2, k3;
  uint32_t ks0, ks1, ks2, ks3;  // scales of the lane's K codes
  uint32_t vs;                  // V scales of token `lane` (D / 32 bytes)
};

// Q of a lane's row as the B operand of K Q^T: channels D / 4 q4 .., what the lane has of K.
template <int D>
struct QueryRows {
  bf16x8 x[D / 32];
};
template <int D>
__device__ __forceinline__ QueryRows<D> load_query(const __bf16* q, bool real, int q4) {
  QueryRows<D> r{};
  if (real) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) r.x[i] = *(const bf16x8*)(q + D / 4 * q4 + 8 * i);
  }
  return r;
}

// A number that is not finite makes its row NaN: infinities become NaN, or a row whose scores are
// all -inf would pass for one that sees nothing.
template <int N>
__device__ __forceinline__ void nan_query(bf16x8 (&x)[N]) {
  u16x2 top = {0, 0};
#pragma unroll
  for (int i = 0; i < 4 * N; ++i) {
    const uint32_t w = __builtin_bit_cast(u32x4, x[i / 4])[i % 4] & 0x7fff7fffu;
    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, w));
  }
  if (max((uint32_t)top[0], (uint32_t)top[1]) >= 0x7f80u) x[0][0] = (__bf16)__builtin_nanf("");
}

// S^T of tokens 16 i ..: K, a lane's D / 4 codes and their scale, times Q.
template <int D, int NT>
__device__ __forceinline__ void scores(const typename PageRegs<D>::Codes& k, uint32_t ks,
                                       const QueryRows<D> (&q)[NT], f32x4 (&s)[NT][4], int i) {
  const float sc = __uint_as_float(ks << 23);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    const bf16x8 x = decode8(k[c], sc);
#pragma unroll
    for (int t = 0; t < NT; ++t)
      s[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[t].x[c], c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[t][i], 0, 0, 0);
  }
}

// How the live pages of a call are dealt to the workgroups: all lists one after
// another in the order (sequence, key/value head, page), and workgroup w takes units
// [w U, (w + 1) U) of them.  A list that lies in more than one workgroup is joined
// from partial results; a workgroup leaves at most two of them, slot 2 w for the
// first list it touches and 2 w + 1 for the last.
//
// Few lists (a quarter of the workgroups at most) of few pages (32 a workgroup): U is a
// multiple of the waves and every list is filled up to a multiple of U, so a workgroup has
// one list only.  64 lists of 51 pages: 22.4 us against 25.5 as below, 8 of 512: 24.7 against
// 29.3; but 128 of 512: 124 against 117, for the workgroups left without a unit.
// Lists of nearly one length (the longest up to 9/8 of the mean) of which two or three a CU
// fill all but a quarter of the CUs' last places (448 .. 512, 704 .. 768): a workgroup each, nothing
// is joined.  456 of 32 pages: 36.6 us against 41.5, 512 40.9 against 46.0, 704 51.5 against 55.8;
// of 128 pages 456 105 against 114, 512 115.8 against 124.4; but 384 of 128 pages: 104 against 98,
// 576 of 128 with D = 64: 72 against 65.
// Else a list counts `cost` units beyond its pages for what it takes besides (page
// numbers, Q, the first page's latency, the joined states): up to 10, but no more than a
// quarter of what a workgroup gets (64 ragged sequences 82.6 us, with 8 85.2, with 12 83.5).
// Left out, the workgroups with the shortest of 64 ragged sequences' lists took 238,000
// cycles where the mean was 123,000.
struct SplitArgs {
  int groups;     // workgroups of the attention kernel
  // With a page mask: the live pages of every list, found ahead by k_cache_lists, as {place
  // in the sequence, page number} [B * Hkv][M] and their count, or nullptr
  const int2* list;
  const int* counts;
  float* part;    // O [2 groups][rows][D], or nullptr: one workgroup per list, nothing is split
  float* ml;      // {m, l} [2 groups][rows]
  int2* where;    // [B * Hkv] first and last slot of a list's partial results (equal: none)
};

// Where the units of a call lie, fewer than 2^31: computed by every workgroup from the
// lengths.  All of it is the same for the whole workgroup and kept in scalar registers.
struct Deal {
  int total;   // units of the call
  int unit;    // units per workgroup
  int cost;    // units of a list beyond its pages, or
  int fill;    //   the unit that lists are filled up to (else 1)
  int set;     // set of lists of this workgroup's first unit
  int before;  // units before it
  int pages;   // pages of each of its lists
  bool empty;  // some list has no page
};

// Units of a list; a list's pages follow its `cost` first ones.
__device__ __forceinline__ int list_units(int pages, int cost, int fill) {
  return pages > 0 ? (pages + cost + fill - 1) / fill * fill : 0;
}

// The deal goes over sets of lists: a sequence's (every head has the same pages), or with a
// page mask a list each.
__device__ __forceinline__ int deal_sets(const CacheArgs& a, const SplitArgs& sa) {
  return sa.counts != nullptr ? a.B * a.Hkv : a.B;
}
// Pages of each list of set i.
__device__ __forceinline__ int set_pages(const CacheArgs& a, const SplitArgs& sa, int i, int rows) {
  return sa.counts != nullptr ? sa.counts[i] : make_span(a, i, 0, rows).count;
}

// Every wave finds it by itself, lane by lane 64 sets at a time: no exchange, and where there
// are no more sets than that one load.  More are read three times over, a latency each: calls
// of one-page lists take 8.8 us with 64 sequences, 37 with 512 and 151 with 4096 (18 and 62
// where each list is a workgroup's), under a page mask 17 us with 512 lists, 47 with 2048, 167 with 8192.
__device__ __forceinline__ Deal make_deal(const CacheArgs& a, const SplitArgs& sa, int rows) {
  const int lane = threadIdx.x & 63, sets = deal_sets(a, sa), heads = sa.counts != nullptr ? 1 : a.Hkv;
  const int n0 = lane < sets ? set_pages(a, sa, lane, rows) : 0;
  auto pages_at = [&](int i) { return i < 64 ? n0 : i < sets ? set_pages(a, sa, i, rows) : 0; };
  int pages = 0, lists = 0, longest = 0, present = 0;
  for (int i = lane; i - lane < sets; i += 64) {
    const int n = pages_at(i);
    pages += n * heads;
    lists += n > 0 ? heads : 0;
    present += n > 0 ? 1 : 0;
    longest = max(longest, n);
  }
  const int tp = wave_total(pages), tl = wave_total(lists), top = wave_top(longest);
  Deal d;
  d.empty = wave_total(present) < sets;
  if (4 * tl <= sa.groups && tp < 32 * sa.groups) {
    const int u = (tp + sa.groups - tl - 1) / (sa.groups - tl);  // the lists' last units fill at most tl more
    d.cost = 0;
    d.unit = d.fill = max((u + kWaves - 1) / kWaves * kWaves, kWaves);
  } else if (tl > 256 && tl <= sa.groups && (tl + 64) / 256 * 256 >= tl && (long long)top * tl <= (long long)tp + tp / 8) {
    d.cost = 0;
    d.unit = d.fill = top;
  } else {
    d.cost = min(tp / sa.groups / 4, 10);
    d.fill = 1;
    d.unit = max((tp + d.cost * tl + sa.groups - 1) / sa.groups, kWaves);
  }
  int units = 0;
  for (int i = lane; i - lane < sets; i += 64) units += list_units(pages_at(i), d.cost, d.fill) * heads;
  d.total = wave_total(units);
  d.set = d.before = d.pages = 0;
  const long long want = (long long)blockIdx.x * d.unit;
  if (want >= d.total) return d;
  for (int i0 = 0, before = 0; i0 < sets; i0 += 64) {
    const int n = pages_at(i0 + lane), u = list_units(n, d.cost, d.fill) * heads, upto = before + wave_scan(u);
    const uint64_t behind = __builtin_amdgcn_ballot_w64(upto > want);
    if (behind != 0) {
      const int l = __builtin_ctzll(behind);
      d.set = i0 + l;
      d.before = __builtin_amdgcn_readlane(upto - u, l);
      d.pages = __builtin_amdgcn_readlane(n, l);
      break;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return d;
}

// Row r of (b, g) whose sums are O / l with l the sum of the weights: out and lse.
template <int EPT>
__device__ __forceinline__ void store_row(const CacheArgs& a, const Span& sp, int D, int b, int g,
                                          int r, int d0, const float* acc, float top, float den) {
  const int qi = r / a.G, h = g * a.G + r % a.G;
  const bool dead = qi >= sp.n || sp.first + qi < 0 || den == 0.f;
  const float inv = dead ? 0.f : 1.f / den;
  const size_t row = ((size_t)b * a.Hq + h) * a.S_q + qi;
  if (a.out_bf16) {
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
      bf16x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (__bf16)(dead ? 0.f : acc[e + i] * inv);
      *(bf16x4*)((__bf16*)a.out + row * D + d0 + e) = v;
    }
  } else {
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = dead ? 0.f : acc[e + i] * inv;
      *(f32x4*)((float*)a.out + row * D + d0 + e) = v;
    }
  }
  if (d0 == 0 && a.lse != nullptr)
    a.lse[row] = dead ? -INFINITY : (top + __builtin_amdgcn_logf(den)) * 0.6931471805599453f;
}

}  // namespace

// Few rows per key/value head (S_q G <= 16 NT): every row in one tile.  A workgroup's
// waves take every fourth page of a list, each with a state of its own, joined at
// the list's (or the workgroup's) end.
//
// Bound by memory where there is much of it: the next page's V (to LDS) and K (to registers)
// are on their way while a wave computes, 12 waves a CU, 104 KB.  16 sequences of 32768
// tokens, 8 heads of 128 (570 MB): 115 us, 5.0 TB/s; a kernel that only reads these records in
// this order reaches 5.8.  64 ragged sequences of up to 32768 (374 MB): 83 us, 4.5 TB/s, for
// the lists that begin and end inside workgroups.  4 sequences of 8000 (35 MB): 14 us cold, bound by
// a chain of latencies: lengths, page numbers, 2 pages a wave, the joined states.  A third
// wave per SIMD is worth more than registers: 2 waves, 73 us against 68 for 64 sequences of
// 4000 on average; 4 waves spill (150 us and more).  With NT = 2 two waves fit.
template <int D, int NT>
__global__ __launch_bounds__(64 * kWaves, waves_per_simd(D, NT)) void k_cache_token(CacheArgs a, SplitArgs sa) {
  using R = Record<D>;
  constexpr int GR = D / 32;        // scale groups
  constexpr int CT = D / 16;        // channel tiles of the output
  constexpr int VROW = D / 2;       // bytes of a token's V codes
  constexpr int OP = D + 4;         // padded output row in LDS
  constexpr int kVBytes = 64 * VROW;
  constexpr int kWaveBytes = 2 * kVBytes + 64 * GR * 2;
  constexpr int kJoinBytes = kWaves * 16 * (OP + 2) * 4;
  constexpr int kLds = kWaves * kWaveBytes > kJoinBytes ? kWaves * kWaveBytes : kJoinBytes;
  __shared__ __attribute__((aligned(16))) char lds[kLds];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, q4 = lane >> 4;
  const int rows = a.S_q * a.G;

  int left;              // units of this workgroup
  int b, g, off;         // list and unit of it of the next one
  int cost = 0, fill = 1;
  const bool split = sa.part != nullptr, listed = sa.counts != nullptr;
  if (!split) {
    b = blockIdx.x / a.Hkv;
    g = blockIdx.x % a.Hkv;
    off = 0;
    left = 1;  // one list, whatever its length
  } else {
    const Deal d = make_deal(a, sa, rows);
    const long long lo = (long long)blockIdx.x * d.unit;
    left = (int)max(min((long long)d.unit, d.total - lo), 0ll);
    cost = d.cost;
    fill = d.fill;
    b = g = off = 0;
    if (left > 0) {
      const int n = list_units(d.pages, cost, fill), at = (int)lo - d.before;
      const int i = at / n;  // list of the set
      b = __builtin_amdgcn_readfirstlane(listed ? d.set / a.Hkv : d.set);
      g = __builtin_amdgcn_readfirstlane(listed ? d.set % a.Hkv : i);
      off = __builtin_amdgcn_readfirstlane(at - i * n);
    }
    // lists without a page: their rows are zero
    const int sets = deal_sets(a, sa), heads = listed ? 1 : a.Hkv;
    for (int z = d.empty ? (int)blockIdx.x : sets; z < sets; z += sa.groups) {
      if (set_pages(a, sa, z, rows) > 0) continue;
      const int zb = listed ? z / a.Hkv : z, zg = listed ? z % a.Hkv : 0;
      const Span sp = make_span(a, zb, 0, rows);
      const float zero[4] = {0.f, 0.f, 0.f, 0.f};
      constexpr int C = D / 4;  // threads of a row; heads * rows alone is below 2^31
      for (int i = threadIdx.x / C; i < heads * rows; i += 64 * kWaves / C)
        store_row<4>(a, sp, D, zb, zg + i / rows, i % rows, threadIdx.x % C * 4, zero, 0.f, 0.f);
    }
  }

  char* wv = lds + wave * kWaveBytes;  // V codes of two pages, 16-byte chunks swizzled in their rows
  unsigned short* wvs = (unsigned short*)(wv + 2 * kVBytes);  // V scales [group][token] as bf16
  const uint32_t wv_lds = lds_addr(wv);

  bool first = true;
  for (; left > 0; first = false) {
    const Span sp = make_span(a, b, 0, rows);
    const int count = __builtin_amdgcn_readfirstlane(listed ? sa.counts[b * a.Hkv + g] : sp.count);
    const int units = list_units(count, cost, fill), last = split ? min(units, off + left) : units;
    const int begin = max(off - cost, 0), end = min(max(last - cost, 0), count);

    // this wave's next 64 pages, one per lane: number (-1: no key of it is visible) and place
    int ids = -1, places = 0, base = begin + wave;
    auto load_ids = [&](int from) {
      const int i = from + kWaves * (thread_here() & 63);
      if (i >= end) return;
      if (listed) {
        const int2 e = sa.list[(size_t)(b * a.Hkv + g) * a.M + i];
        places = e.x;
        ids = e.y;
        return;
      }
      places = span_page(sp, i);
      ids = a.table[(size_t)b * a.M + places];
      if (ids >= a.n_pages) ids = -1;
      if (a.mask != nullptr && a.mask[((size_t)b * a.Hkv + g) * a.M + places] == 0) ids = -1;
    };
    auto record = [&](int id) { return a.pages + ((size_t)id * a.Hkv + g) * R::kBytes; };
    // a lane's places in a record
    const uint32_t k_at = n * R::kRow + q4 * (D / 8), ks_at = R::kKs + n * GR + (GR == 4 ? q4 : q4 >> 1);
    const uint32_t vs_at = R::kVs + GR * lane;
    PageRegs<D> x;
    typedef typename PageRegs<D>::Codes Codes;
    auto load_k = [&](const uint8_t* rec) {
      x.k0 = *(const Codes*)(rec + k_at);
      x.k1 = *(const Codes*)(rec + 16 * R::kRow + k_at);
      x.k2 = *(const Codes*)(rec + 32 * R::kRow + k_at);
      x.k3 = *(const Codes*)(rec + 48 * R::kRow + k_at);
      x.ks0 = (rec + ks_at)[0];
      x.ks1 = (rec + 16 * GR + ks_at)[0];
      x.ks2 = (rec + 32 * GR + ks_at)[0];
      x.ks3 = (rec + 48 * GR + ks_at)[0];
      if constexpr (GR == 4) x.vs = *(const uint32_t*)(rec + vs_at);
      else x.vs = *(const unsigned short*)(rec + vs_at);
    };
    // V codes straight to LDS: chunk c of token row r at slot c ^ (r / 4) % 4 (D = 128, 4
    // chunks a row) or c ^ (r / 8) % 2 (D = 64, 2 chunks)
    constexpr int CPR = VROW / 16, RPC = 64 / CPR;  // chunks per row, rows per copy
    const uint32_t v_chunk = (lane % CPR) ^ (D == 128 ? (lane >> 4) & 3 : (lane >> 4) & 1);
    const uint32_t v_at = R::kV + lane / CPR * VROW + v_chunk * 16;
    auto copy_v = [&](const uint8_t* rec, int buf) {
#pragma unroll
      for (int j = 0; j < 64 / RPC; ++j)
        copy16_to_lds(rec + j * 1024, v_at, wv_lds + buf * kVBytes + j * 1024);
    };

    // page numbers and query rows asked for together, then the first page, then Q is split
    int id = -1, buf = 0, kb_next = 0;
    if (base < end) load_ids(base);
    QueryRows<D> qf[NT];
    int pos[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int row = 16 * t + n, qi = row / a.G;
      const bool real = row < rows && qi < sp.n;
      pos[t] = real ? sp.first + qi : -1;
      qf[t] = load_query<D>(a.q + b * a.q_sb + (g * a.G + row % a.G) * a.q_sh + qi * a.q_ss, real, q4);
    }
    if (base < end) {
      id = __builtin_amdgcn_readfirstlane(ids);
      kb_next = __builtin_amdgcn_readfirstlane(places);
      copy_v(record(max(id, 0)), 0);
      load_k(record(max(id, 0)));
    }
    f32x4 o[NT][CT];
    float m[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      nan_query(qf[t].x);
#pragma unroll
      for (int c = 0; c < CT; ++c) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[t] = -INFINITY;
      l[t] = 0.f;
    }
    for (int i = base; i < end; i += kWaves, buf ^= 1) {
      const bool there = id >= 0;  // else page 0 stands in, none of its keys visible
      const int kb = kb_next;
      // S^T: 4 tiles of 16 tokens
      f32x4 sc[NT][4];
      scores<D, NT>(x.k0, x.ks0, qf, sc, 0);
      scores<D, NT>(x.k1, x.ks1, qf, sc, 1);
      scores<D, NT>(x.k2, x.ks2, qf, sc, 2);
      scores<D, NT>(x.k3, x.ks3, qf, sc, 3);
      // tokens whose values stand for NaN (all scale bytes 255, or none), and whether any value is
      // above 2^64; bytes behind the sequence count as 0
      uint32_t vs = kb * kBlk + lane < sp.keys ? x.vs : 0u;
      const uint64_t v_nan = __builtin_amdgcn_ballot_w64((vs & 0xff) == kScaleNan);
      const bool v_large = __builtin_amdgcn_ballot_w64((vs & (vs << 1) & 0x80808080u) != 0) != 0;
      vs = (vs & 0xff) == kScaleNan ? 0x7f7f7f7fu : vs;
#pragma unroll
      for (int gr = 0; gr < GR; ++gr)
        wvs[64 * gr + lane] = (unsigned short)((vs >> (8 * gr) & 0xff) << 7);
      wait_vm<0>();  // this page's V is in LDS (and its K was used)
      // the next page on its way
      if (i + kWaves < end) {
        const int k = (i + kWaves - base) / kWaves;
        if (k % 64 == 0) load_ids(i + kWaves);
        id = __builtin_amdgcn_readlane(ids, k % 64);
        kb_next = __builtin_amdgcn_readlane(places, k % 64);
        copy_v(record(max(id, 0)), buf ^ 1);
        load_k(record(max(id, 0)));
      }
      const bool full = there && page_full(a, sp, kb);
      if (!full) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int lim = there ? row_limit(a, sp, pos[nt], kb) - 4 * q4 : -1;
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) sc[nt][t][r] = 16 * t + r > lim ? -INFINITY : sc[nt][t][r];
        }
      }
      // The running maximum moves only where a row's scores exceed it by 2^kTau: m
      // cancels in O / l, and weights up to 2^8 lose nothing in bf16.  With values above 2^64
      // it moves at once, so that no weight times a value leaves the range of fp32.
      const float tau = v_large ? 0.f : kTau;
      bool grow = false;
      float mx[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        mx[nt] = sc[nt][0][0];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) mx[nt] = fmaxf(mx[nt], sc[nt][t][r]);
        grow |= mx[nt] * a.c > m[nt] + tau;
      }
      if (__builtin_amdgcn_ballot_w64(grow)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float mnew = fmaxf(m[nt], row_max(mx[nt]) * a.c);
          const float alpha = __builtin_amdgcn_exp2f(m[nt] - finite_max(mnew));  // 0 before the first key
          m[nt] = mnew;
          l[nt] *= alpha;
#pragma unroll
          for (int c = 0; c < CT; ++c) o[nt][c] *= alpha;
        }
      }
      // P = 2^(S c - m) in bf16, two to a register
      uint32_t pk[NT][8];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float ms = finite_max(m[nt]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nt][e / 2][e % 2 * 2], a.c, -ms));
          const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nt][e / 2][e % 2 * 2 + 1], a.c, -ms));
          l[nt] += p0;
          l[nt] += p1;
          pk[nt][e] = pack_bf16(p0, p1);
        }
      }
      // O^T += V^T P^T, 32 channels (one scale per token) at a time.  The scaling of P is an
      // addition to both exponents of a pair: P + (e - 127) in units of 2^7, not below 0.  A
      // weight under 2^-126 then ends as up to 2^(e - 254), 2^-127 of what the token's values
      // can be, which is nothing where the row sees the token; where it may not, and where
      // e > 191 might carry into the sign, zero weights stay 0 and the sum is kept below it.
      const bool special = !full || v_large;
      const char* wvb = wv + buf * kVBytes;
      const int tok = 16 * (n >> 2) + 4 * q4 + (n & 3);
      auto read_v = [&](int ct) {
        const int slot = ((ct >> 1) ^ (D == 128 ? q4 : q4 >> 1)) * 16 + (ct & 1) * 8;
        return __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2*)(wvb + tok * VROW + slot));
      };
#pragma unroll
      for (int gr = 0; gr < GR; ++gr) {
        __builtin_amdgcn_sched_barrier(0);  // else all groups' operands are held at one time
        u32x2 sv[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sv[t] = *(const u32x2*)(wvs + 64 * gr + 16 * t + 4 * q4);
        const i32x2 w[2] = {read_v(2 * gr), read_v(2 * gr + 1)};
        u32x4 u[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t se = sv[e / 2][e % 2];
            const u16x2 y = __builtin_bit_cast(u16x2, pk[nt][e]) + __builtin_bit_cast(u16x2, se);
            u[nt][e / 4][e % 4] = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(y, u16x2{0x3f80, 0x3f80}));
          }
        if (special) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t ue = u[nt][e / 4][e % 4];
              const u16x2 some = __builtin_elementwise_min(__builtin_bit_cast(u16x2, pk[nt][e]), u16x2{1, 1});
              const u16x2 y = __builtin_elementwise_min(__builtin_bit_cast(u16x2, ue), u16x2{0x7fc0, 0x7fc0});
              u[nt][e / 4][e % 4] = __builtin_bit_cast(uint32_t, some * y);
            }
        }
#pragma unroll
        for (int c2 = 0; c2 < 2; ++c2) {
          const int ct = 2 * gr + c2;
          const bf16x8 v0 = decode8((uint32_t)w[c2][0], 1.f), v1 = decode8((uint32_t)w[c2][1], 1.f);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            o[nt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, __builtin_bit_cast(bf16x8, u[nt][0]), o[nt][ct], 0, 0, 0);
            o[nt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, __builtin_bit_cast(bf16x8, u[nt][1]), o[nt][ct], 0, 0, 0);
          }
        }
      }
      if (v_nan != 0) {  // values that stand for NaN (as numbers above), where the row sees them
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          if (there && sees_any(v_nan, row_limit(a, sp, pos[nt], kb))) {
#pragma unroll
            for (int c = 0; c < CT; ++c) o[nt][c] = f32x4{} + __builtin_nanf("");
          }
      }
    }

    // the waves' states of a row joined, then the rows or a partial result stored
    const bool whole = off == 0 && last == units;
    const int slot = 2 * (int)blockIdx.x + (first ? 0 : 1);
    if (split && threadIdx.x == 0) {
      if (off == 0) sa.where[b * a.Hkv + g].x = slot;
      if (last == units) sa.where[b * a.Hkv + g].y = slot;
    }
    const int tid = thread_here(), en = tid & 15, eq4 = tid >> 4 & 3, ew = tid >> 6;
    float* jo = (float*)lds;              // [wave][16][OP]
    float* jml = jo + kWaves * 16 * OP;   // [wave][16][2]
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      __syncthreads();
      const float ls = row_sum(l[nt]);
#pragma unroll
      for (int c = 0; c < CT; ++c) *(f32x4*)(jo + (ew * 16 + en) * OP + 16 * c + 4 * eq4) = o[nt][c];
      if (eq4 == 0) {
        jml[(ew * 16 + en) * 2] = m[nt];
        jml[(ew * 16 + en) * 2 + 1] = ls;
      }
      __syncthreads();
      constexpr int TPR = 64 * kWaves / 16;     // threads per row
      constexpr int EPT = D / TPR;              // elements per thread
      const int jr = tid / TPR, d0 = tid % TPR * EPT, r = 16 * nt + jr;
      if (r < rows) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, jml[(w * 16 + jr) * 2]);
        const float ts = top == -INFINITY ? 0.f : top;
        float den = 0.f, acc[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) acc[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(jml[(w * 16 + jr) * 2] - ts);
          den += f * jml[(w * 16 + jr) * 2 + 1];
#pragma unroll
          for (int e = 0; e < EPT; ++e) acc[e] += f * jo[(w * 16 + jr) * OP + d0 + e];
        }
        if (whole) {
          store_row<EPT>(a, sp, D, b, g, r, d0, acc, ts, den);
        } else {
#pragma unroll
          for (int e = 0; e < EPT; e += 4)
            *(f32x4*)(sa.part + ((size_t)slot * rows + r) * D + d0 + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
          if (d0 == 0) {
            sa.ml[((size_t)slot * rows + r) * 2] = top;
            sa.ml[((size_t)slot * rows + r) * 2 + 1] = den;
          }
        }
      }
    }
    __syncthreads();

    left = split ? left - (last - off) : 0;
    if (left == 0) break;
    // the next list that has a page
    off = 0;
    if (listed) {
      do {
        if (++g == a.Hkv) {
          g = 0;
          ++b;
        }
      } while (b < a.B && sa.counts[b * a.Hkv + g] == 0);
    } else if (++g == a.Hkv) {
      g = 0;
      do ++b;
      while (b < a.B && make_span(a, b, 0, rows).count == 0);
    }
    if (b >= a.B) break;
  }
}

// Lists that lie in more than one workgroup of k_cache_token: their partial results
// joined.  One workgroup per list and row; 8 (D = 128) or 16 threads of a column of 4
// channels share the parts, each in one pass with a running maximum.  Latency bound (slots,
// then parts, then the exchange): 4.8 us, 3 us of a step's time behind the kernel above.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void k_cache_join(CacheArgs a, SplitArgs sa) {
  constexpr int C = D / 4, PG = 64 * kWaves / C;
  __shared__ __attribute__((aligned(16))) f32x4 lds[PG][C];
  __shared__ float ldsl[PG], ldsm[PG];
  const int rows = a.S_q * a.G, b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, r = blockIdx.y;
  const int2 at = sa.where[blockIdx.x];  // asked for before it is known to be written
  const Span sp = make_span(a, b, 0, rows);
  const int count = sa.counts != nullptr ? sa.counts[blockIdx.x] : sp.count;
  if (count == 0) return;  // uniform over the workgroup
  const int first = at.x, w0 = at.x / 2, w1 = at.y / 2;
  if (w0 == w1) return;  // stored by its workgroup
  const int c = threadIdx.x % C, pg = threadIdx.x / C;
  const int parts = w1 - w0 + 1;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  for (int i = pg; i < parts; i += PG) {
    const size_t s = (size_t)(i == 0 ? first : 2 * (w0 + i)) * rows + r;
    const float ms = sa.ml[s * 2], ls = sa.ml[s * 2 + 1];
    const f32x4 os = *(const f32x4*)(sa.part + s * D + 4 * c);
    const float mnew = fmaxf(m, ms), f0 = __builtin_amdgcn_exp2f(m - finite_max(mnew)),
                f1 = __builtin_amdgcn_exp2f(ms - finite_max(mnew));
    l = l * f0 + f1 * ls;
    acc = acc * f0 + f1 * os;
    m = mnew;
  }
  lds[pg][c] = acc;
  if (c == 0) {
    ldsm[pg] = m;
    ldsl[pg] = l;
  }
  __syncthreads();
  if (pg != 0) return;
#pragma unroll
  for (int i = 1; i < PG; ++i) m = fmaxf(m, ldsm[i]);
  const float ms = finite_max(m);
  acc = f32x4{0.f, 0.f, 0.f, 0.f};
  l = 0.f;
#pragma unroll
  for (int i = 0; i < PG; ++i) {
    const float f = __builtin_amdgcn_exp2f(ldsm[i] - ms);
    l += f * ldsl[i];
    acc += f * lds[i][c];
  }
  const float out[4] = {acc[0], acc[1], acc[2], acc[3]};
  store_row<4>(a, sp, D, b, g, r, 4 * c, out, ms, l);
}

// Many rows per key/value head (chunks of prompts): tiles of 128 rows, 4 waves of 32.
//
// S^T = K Q^T and O^T = V^T P^T on 32x32 MFMAs, a row in the lanes l % 32.  A page's K codes go
// to LDS as they are and every wave turns them into bf16 (once for the workgroup, with bf16
// keys in LDS: 254 us against 241); its V is turned into bf16 by the whole
// workgroup (16 conversions and four 16-byte LDS writes a thread) and read
// transposed, as the dense kernels do.  Both are one page ahead: K by copies, V's codes in
// registers until the present page is done.
//
// Bound by the MFMAs and the exponentials between them: 1000 queries of 32 heads against 12000
// keys of 8 heads of 128 (188 GFLOP) 213 us with the join, 880 TFLOP/s; a large bf16 matrix
// product reaches 1256 on the same card.  MFMAs take 39% of the cycles, VALU 53%, and the two
// hardly overlap.  Two workgroups per CU.
// Segments (below) fill the chip where the tiles are few: 239 us against 283 without here (random
// codes), 64 queries against 16000 keys 55 against 355.
// Waves of 64 rows were no faster (D = 64: 152 against 157 us, but 159 against 130 with 12 heads) or
// spilled (D = 128: 596).
struct ChunkArgs {
  int tiles, ns;  // tiles of a (sequence, key/value head), segments of a tile's list at most
  int least;      // pages of a segment at least
  float* part;    // O [unit][tile][ns][128][D] when ns > 1
  float* ml;      // {m, l}
};

constexpr int kTile = 128;

// Segments of a tile with `count` pages.
__device__ __forceinline__ int tile_segments(const ChunkArgs& ca, int count) {
  return min(ca.ns, max(count / ca.least, 1));
}

// Workgroup -> (unit, tile, segment).  With a multiple of 8 units each keeps to one XCD,
// whose L2 then holds its keys and values (2048 queries of 32 heads, 4096 keys: 143 us against
// 161; 512 queries, 16384 keys 177 against 179); a unit's heaviest tiles come first.
__device__ __forceinline__ void chunk_item(const CacheArgs& a, const ChunkArgs& ca, int* unit, int* tile,
                                           int* seg) {
  const int per = ca.tiles * ca.ns, units = a.B * a.Hkv, i = blockIdx.x;
  int at = i;
  if (units % 8 == 0) {
    const int x = i & 7, j = i >> 3;
    *unit = j / per * 8 + x;
    at = j % per;
  } else {
    *unit = i / per;
    at = i % per;
  }
  *tile = ca.tiles - 1 - at / ca.ns;
  *seg = at % ca.ns;
}

template <int D>
__global__ __launch_bounds__(256, 2) void k_cache_chunk(CacheArgs a, ChunkArgs ca) {
  using R = Record<D>;
  constexpr int KS = D / 64;        // K steps of 64 channels
  constexpr int GR = D / 32, DT = D / 32;
  constexpr int VROW = D / 2;       // bytes of a token's codes
  constexpr int RB = 2 * D;         // bytes of a token's values in bf16
  constexpr int VB = 64 * RB, KB = 64 * VROW;
  constexpr int CPR = VROW / 16;    // 16-byte chunks of a token's codes
  __shared__ __attribute__((aligned(1024))) char lds[2 * VB + 2 * KB];

  int unit, tile, seg;
  chunk_item(a, ca, &unit, &tile, &seg);
  const int g = unit % a.Hkv, b = unit / a.Hkv, rows = a.S_q * a.G;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, hf = lane >> 5;
  const int r0 = tile * kTile, r1 = min(r0 + kTile, rows);
  const Span sp = make_span(a, b, r0, r1);
  const int ns = tile_segments(ca, sp.count);
  if (seg >= ns) return;
  const int p0 = (int)((long long)sp.count * seg / ns), p1 = (int)((long long)sp.count * (seg + 1) / ns);

  // this lane's row
  const int row = r0 + 32 * wave + n, qi = row / a.G;
  const bool real = row < r1 && qi < sp.n;
  const int pos = real ? sp.first + qi : -1;
  bf16x8 q[4 * KS];  // channels 64 s + 32 hf + 8 i .. at 4 s + i
#pragma unroll
  for (int i = 0; i < 4 * KS; ++i) q[i] = bf16x8{};
  if (real) {
    const __bf16* at = a.q + b * a.q_sb + (g * a.G + row % a.G) * a.q_sh + qi * a.q_ss + 32 * hf;
#pragma unroll
    for (int i = 0; i < 4 * KS; ++i) q[i] = *(const bf16x8*)(at + i / 4 * 64 + i % 4 * 8);
  }
  nan_query(q);

  // pages: the numbers of 64 list entries, one per lane, and the set of those still to come;
  // pages that do not exist or are masked are never visited
  int ids = -1, from = p0 - 64;
  uint64_t todo = 0;
  auto next_page = [&](int* kb) {  // the next page's number, or -1; kb: its place in the sequence
    while (todo == 0) {
      from += 64;
      if (from >= p1) return -1;
      const int i = from + lane;
      ids = -1;
      if (i < p1) {
        const int k = span_page(sp, i);
        ids = a.table[(size_t)b * a.M + k];
        if (ids >= a.n_pages) ids = -1;
        if (a.mask != nullptr && a.mask[((size_t)b * a.Hkv + g) * a.M + k] == 0) ids = -1;
      }
      todo = __builtin_amdgcn_ballot_w64(ids >= 0);
    }
    const int j = __builtin_ctzll(todo);
    todo &= todo - 1;
    *kb = span_page(sp, from + j);
    return __builtin_amdgcn_readlane(ids, j);
  };
  auto record = [&](int id) { return a.pages + ((size_t)id * a.Hkv + g) * R::kBytes; };

  // K: wave w copies a quarter (D = 64: the first two waves a half) of the codes; chunk c of
  // token row r stands at slot c ^ (r / 4) % 4 (D = 64: c ^ (r / 8) % 2)
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(lds));
  const uint32_t kc_at = lane / CPR * VROW + ((lane % CPR) ^ (D == 128 ? (lane >> 4) & 3 : (lane >> 4) & 1)) * 16;
  auto copy_k = [&](const uint8_t* rec, int buf) {
    if (D == 128 || wave < 2)
      copy16_to_lds(rec + wave * 1024, kc_at, lds0 + 2 * VB + buf * KB + wave * 1024);
  };
  // V: thread t turns a quarter of token t / 4's codes into bf16
  typedef unsigned Codes __attribute__((ext_vector_type(D / 32)));
  const int vt = tid >> 2, vq = tid & 3;
  const uint32_t vc_at = R::kV + vt * VROW + vq * (VROW / 4);
  const uint32_t vs_at = R::kVs + vt * GR + (D == 128 ? vq : vq >> 1);
  struct Next {
    Codes v;
    uint32_t vs, vt, ks[2];  // V scale of the thread's codes, scales of token `lane`; K scales of tokens n, 32 + n
  } x;
  auto load_next = [&](const uint8_t* rec) {
    x.v = *(const Codes*)(rec + vc_at);
    x.vs = (rec + vs_at)[0];
    if constexpr (D == 128) x.vt = *(const uint32_t*)(rec + R::kVs + GR * lane);
    else x.vt = *(const unsigned short*)(rec + R::kVs + GR * lane);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if constexpr (D == 128) x.ks[t] = *(const uint32_t*)(rec + R::kKs + (32 * t + n) * GR);
      else x.ks[t] = *(const unsigned short*)(rec + R::kKs + (32 * t + n) * GR);
    }
  };
  auto store_v = [&](int buf, int kb) {
    // bytes behind the sequence, and of tokens that stand for NaN, become 0
    const float sc = kb * kBlk + vt < sp.keys && x.vs != kScaleNan ? __uint_as_float(x.vs << 23) : 0.f;
    const bool zero = sc == 0.f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const bf16x8 v = decode8(zero ? 0u : x.v[c], zero ? 1.f : sc);
      *(bf16x8*)(lds + buf * VB + tile_elem<D>(vt, vq * (D / 32) + c) * 2) = v;
    }
  };
  const uint32_t kr_at = lds0 + 2 * VB + n * VROW;
  const int ksw = D == 128 ? (n >> 2) & 3 : (n >> 3) & 1;
  const int tg = lane >> 4, tr = (lane >> 2) & 3, tq = lane & 3;
  const uint32_t vr_at = lds0 + (uint32_t)(tile_elem<D>(4 * (tg >> 1) + tr, 2 * (tg & 1) + (tq >> 1)) + 4 * (tq & 1)) * 2;
  typedef const __attribute__((address_space(3))) char* lds_cp;
  typedef const __attribute__((address_space(3))) u32x4* lds_u32x4;

  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x16{};
  float m = -INFINITY, l = 0.f;

  int kb = 0, buf = 0, kb_next = 0;
  int id = next_page(&kb);
  if (id >= 0) {
    copy_k(record(id), 0);
    load_next(record(id));
    store_v(0, kb);
  }
  uint32_t ks[2] = {x.ks[0], x.ks[1]};
  // tokens whose values stand for NaN (all scale bytes 255, or none), and whether any value is
  // above 2^64; bytes behind the sequence count as 0
  uint64_t v_nan = 0;
  bool v_large = false;
  auto look_at_v = [&](int kb) {
    const uint32_t vt = kb * kBlk + lane < sp.keys ? x.vt : 0u;
    v_nan = __builtin_amdgcn_ballot_w64((vt & 0xff) == kScaleNan);
    v_large = __builtin_amdgcn_ballot_w64((vt & (vt << 1) & 0x80808080u) != 0) != 0;
  };
  look_at_v(kb);
  wait_vm<0>();
  __syncthreads();
  while (id >= 0) {
    const int id_next = next_page(&kb_next);
    if (id_next >= 0) {
      copy_k(record(id_next), buf ^ 1);
      load_next(record(id_next));
    }
    // S^T: 2 tiles of 32 tokens
    f32x16 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) sc[t] = f32x16{};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 k[2];
      float kse[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        k[t] = *(lds_u32x4)(lds_cp)(kr_at + buf * KB + 32 * t * VROW + (((2 * s + hf) ^ ksw) * 16));
        kse[t] = __uint_as_float((ks[t] >> (8 * hf + 16 * s) & 0xff) << 23);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode8(k[t][i], kse[t]), q[4 * s + i], sc[t], 0, 0, 0);
    }
    if (!page_full(a, sp, kb)) {
      const int lim = row_limit(a, sp, pos, kb) - 4 * hf;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[t][r] = 32 * t + 8 * (r >> 2) + (r & 3) > lim ? -INFINITY : sc[t][r];
    }
    // the running maximum, as in k_cache_token
    float mx = fmaxf(sc[0][0], sc[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(fmaxf(mx, sc[0][r]), sc[1][r]);
    if (__builtin_amdgcn_ballot_w64(mx * a.c > m + (v_large ? 0.f : kTau))) {
      const float mnew = fmaxf(m, other_half_max(mx) * a.c);
      const float alpha = __builtin_amdgcn_exp2f(m - finite_max(mnew));
      m = mnew;
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= alpha;
    }
    const float ms = finite_max(m);
    const uint32_t vb = vr_at + buf * VB;
    // Weights of 16 tokens, then their products: the next 16's exponentials run beside these
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u32x4 u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][8 * c + 2 * e], a.c, -ms));
          const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][8 * c + 2 * e + 1], a.c, -ms));
          l += w0;
          l += w1;
          u[e] = pack_bf16(w0, w1);
        }
        const bf16x8 pa = __builtin_bit_cast(bf16x8, u);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_s16x4*)(lds_cp)((vb ^ (uint32_t)(d << 6)) + (32 * t + 16 * c) * RB));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (lds_s16x4*)(lds_cp)((vb ^ (uint32_t)((d << 6) | 32)) + (32 * t + 16 * c + 8) * RB));
          const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pa, o[d], 0, 0, 0);
        }
      }
    if (v_nan != 0 && sees_any(v_nan, row_limit(a, sp, pos, kb))) {  // values that stand for NaN (as 0 above)
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] = f32x16{} + __builtin_nanf("");
    }
    if (id_next >= 0) {
      store_v(buf ^ 1, kb_next);
      ks[0] = x.ks[0];
      ks[1] = x.ks[1];
      look_at_v(kb_next);
    }
    wait_vm<0>();
    __syncthreads();
    id = id_next;
    kb = kb_next;
    buf ^= 1;
  }

  // this lane's row: channels 32 d + 8 i + 4 hf ..
  const float ls = half_pair_sum(l);
  if (row >= r1) return;
  if (ns > 1) {
    const size_t at = (((size_t)unit * ca.tiles + tile) * ca.ns + seg) * kTile + 32 * wave + n;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(ca.part + at * D + 32 * d + 8 * i + 4 * hf) =
            f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    if (hf == 0) {
      ca.ml[at * 2] = m;
      ca.ml[at * 2 + 1] = ls;
    }
    return;
  }
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v[4] = {o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
      store_row<4>(a, sp, D, b, g, row, 32 * d + 8 * i + 4 * hf, v, finite_max(m), ls);
    }
}

// The segments of a tile's rows joined: a thread per row and 4 channels.  Memory bound: 2 segments
// of 32000 rows of 128 (41 MB with the bf16 output) 11 us, 3.8 TB/s.
template <int D>
__global__ __launch_bounds__(256) void k_cache_chunk_join(CacheArgs a, ChunkArgs ca) {
  constexpr int C = D / 4, RPW = 256 / C;  // rows of a workgroup
  const int rows = a.S_q * a.G;
  const long long i = (long long)blockIdx.x * RPW + threadIdx.x / C;
  const int d0 = threadIdx.x % C * 4, unit = (int)(i / rows), r = (int)(i % rows);
  if (unit >= a.B * a.Hkv) return;
  const int b = unit / a.Hkv, g = unit % a.Hkv, tile = r / kTile;
  const Span sp = make_span(a, b, tile * kTile, min((tile + 1) * kTile, rows));
  const int ns = tile_segments(ca, sp.count);
  if (ns == 1) return;  // stored by its workgroup
  const size_t at = ((size_t)unit * ca.tiles + tile) * ca.ns * kTile + r % kTile;
  float top = -INFINITY;
  for (int s = 0; s < ns; ++s) top = fmaxf(top, ca.ml[(at + (size_t)s * kTile) * 2]);
  const float ts = top == -INFINITY ? 0.f : top;
  float den = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < ns; ++s) {
    const size_t p = at + (size_t)s * kTile;
    const float f = __builtin_amdgcn_exp2f(ca.ml[p * 2] - ts);
    den += f * ca.ml[p * 2 + 1];
    acc += f * *(const f32x4*)(ca.part + p * D + d0);
  }
  const float v[4] = {acc[0], acc[1], acc[2], acc[3]};
  store_row<4>(a, sp, D, b, g, r, d0, v, ts, den);
}

struct ChunkPlan {
  int tiles, ns, least, grid;
  size_t part, total;
};

ChunkPlan chunk_plan(int B, int Hkv, int rows, int D, int pages) {
  ChunkPlan p{};
  p.tiles = (rows + kTile - 1) / kTile;
  const long long items = (long long)B * Hkv * p.tiles;
  long long ns = (512 + items - 1) / items;  // two workgroups per CU
  // A segment saves its share of a tile's pages and costs 64 KB or 128 KB written and read back, the
  // more the more tiles do so: 8 pages at least, 27 with 384 tiles.  With 8 always, 376 tiles of up
  // to 36 pages take 88 us (67), 436 of up to 32 54 us (48); 32 of 188 the same.
  p.least = 8 + (int)(items < 512 ? items / 20 : 0);
  const long long most = pages / p.least > 1 ? pages / p.least : 1;
  p.ns = (int)(ns < most ? ns : most);
  p.grid = (int)(items * p.ns);
  const size_t slots = (size_t)p.grid * kTile;
  p.part = (slots * 2 * sizeof(float) + 255) & ~(size_t)255;
  p.total = p.ns > 1 ? p.part + slots * D * sizeof(float) : 0;
  return p;
}

template <int D>
void launch_chunk(const CacheArgs& a, const ChunkPlan& p, void* ws, hipStream_t s) {
  ChunkArgs ca{p.tiles, p.ns, p.least, (float*)((char*)ws + p.part), (float*)ws};
  hipLaunchKernelGGL(k_cache_chunk<D>, dim3(p.grid), dim3(256), 0, s, a, ca);
  if (p.ns > 1) {
    const long long rows = (long long)a.B * a.Hkv * a.S_q * a.G;
    hipLaunchKernelGGL(k_cache_chunk_join<D>, dim3((unsigned)((rows + 1024 / D - 1) / (1024 / D))), dim3(256), 0, s, a, ca);
  }
}

// The live pages of every list, one workgroup each: the pages of the span that exist and
// whose mask byte is set, in order.  A tenth of 64 lists of 512: 5.0 us, latency bound, and the
// attention 13.9; where k_cache_token skipped the others itself it took 49.
__global__ __launch_bounds__(256) void k_cache_lists(CacheArgs a, int rows, int2* list, int* counts) {
  __shared__ int found[2][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x, b = i / a.Hkv;
  const Span sp = make_span(a, b, 0, rows);
  int n = 0;
  for (int from = 0, k = 0; from < sp.count; from += 256, k ^= 1) {
    const int j = from + threadIdx.x;
    int kb = 0, id = -1;
    if (j < sp.count) {
      kb = span_page(sp, j);
      const uint8_t live = a.mask[(size_t)i * a.M + kb];
      id = a.table[(size_t)b * a.M + kb];
      if (live == 0 || id >= a.n_pages) id = -1;
    }
    const uint64_t set = __builtin_amdgcn_ballot_w64(id >= 0);
    if (lane == 0) found[k][wave] = __builtin_popcountll(set);
    __syncthreads();
    int at = n + __builtin_popcountll(set & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      at += w < wave ? found[k][w] : 0;
      n += found[k][w];
    }
    if (id >= 0) list[(size_t)i * a.M + at] = int2{kb, id};
  }
  if (threadIdx.x == 0) counts[i] = n;
}

// What a call's sizes make of it.
struct TokenPlan {
  int groups;  // workgroups
  bool split;
  size_t part, where, list, counts, total;  // workspace offsets and size in bytes; {m, l} stand first
};

// pages: what a list can have at most.  Up to 24 a list is one workgroup's: nothing to join and
// no second launch.  One token at 4 / 16 / 24 / 32 pages, whole against split: 8 heads of 128
// 6.8 / 10.9 / 13.6 / 16.4 us against 11.3 / 13.7 / 13.7 / 13.7, 64 sequences of 8 heads
// 10.4 / 19.5 / 27.2 / 32.9 us against 15.6 / 30.1 / 37.9 / 43.2.
TokenPlan token_plan(int B, int Hkv, int rows, int D, int M, int pages, bool masked) {
  TokenPlan p{};
  const long long lists = (long long)B * Hkv;
  const long long want = (lists * pages + 3) / 4;
  const int most_groups = 256 * waves_per_simd(D, rows <= 16 ? 1 : 2);
  p.groups = (int)(want < most_groups ? want : most_groups);
  p.split = pages > 24;
  if (!p.split) p.groups = (int)lists;
  const size_t slots = 2 * (size_t)p.groups * rows;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  p.part = up(slots * 2 * sizeof(float));
  p.where = p.part + up(slots * D * sizeof(float));
  p.list = p.where + up((size_t)lists * sizeof(int2));
  p.counts = p.list + up((size_t)lists * M * sizeof(int2));
  p.total = !p.split ? 0 : masked ? p.counts + (size_t)lists * sizeof(int) : p.list;
  return p;
}

template <int D>
void launch_token(const CacheArgs& a, const TokenPlan& p, char* ws, int rows, hipStream_t s) {
  SplitArgs sa{};
  sa.groups = p.groups;
  if (p.split) {
    sa.ml = (float*)ws;
    sa.part = (float*)(ws + p.part);
    sa.where = (int2*)(ws + p.where);
    if (a.mask != nullptr) {
      sa.list = (const int2*)(ws + p.list);
      sa.counts = (const int*)(ws + p.counts);
      hipLaunchKernelGGL(k_cache_lists, dim3(a.B * a.Hkv), dim3(256), 0, s, a, rows,
                         (int2*)(ws + p.list), (int*)(ws + p.counts));
    }
  }
  const dim3 grid(p.groups), wg(64 * kWaves);
  if (rows <= 16) hipLaunchKernelGGL((k_cache_token<D, 1>), grid, wg, 0, s, a, sa);
  else hipLaunchKernelGGL((k_cache_token<D, 2>), grid, wg, 0, s, a, sa);
  if (p.split) hipLaunchKernelGGL(k_cache_join<D>, dim3(a.B * a.Hkv, rows), wg, 0, s, a, sa);
}

// Up to 32 rows of a key/value head go to k_cache_token, which streams pages past the rows; more to
// k_cache_chunk, whose tiles of 128 share them.  32 rows, 8 heads of 128: 8 sequences of 16384 tokens
// 52 us against 89, one of 32768 29 against 62, 64 of 200 to 8100 114 against 236 (D = 64: 83
// against 169).  More than 32 rows would take a
// third tile of accumulators, which do not fit into registers beside two.
constexpr int kTokenRows = 32;

size_t cache_attn_ws(int B, int Hq, int Hkv, int S_q, int D, int M, bool masked) {
  const int rows = S_q * (Hq / Hkv);
  return rows <= kTokenRows ? token_plan(B, Hkv, rows, D, M, M, masked).total
                            : chunk_plan(B, Hkv, rows, D, M).total;
}

// Pages that `queries` of a sequence next to each other can see: with a window its own, the
// sinks', and more where the queries lie in several pages.
int most_pages(const CacheArgs& a, int queries) {
  const long long n = a.win > 0 ? (long long)a.sink + a.win + (queries + 62) / kBlk : a.M;
  return (int)(n < a.M ? n : a.M);
}

hipError_t launch_cache_attn(const CacheArgs& a, int D, void* ws, hipStream_t s) {
  const int rows = a.S_q * a.G;
  if (rows <= kTokenRows) {
    const TokenPlan p = token_plan(a.B, a.Hkv, rows, D, a.M, most_pages(a, a.S_q), a.mask != nullptr);
    if (D == 64) launch_token<64>(a, p, (char*)ws, rows, s);
    else launch_token<128>(a, p, (char*)ws, rows, s);
  } else {
    const ChunkPlan p = chunk_plan(a.B, a.Hkv, rows, D, most_pages(a, (kTile - 1) / a.G + 2));
    if (D == 64) launch_chunk<64>(a, p, ws, s);
    else launch_chunk<128>(a, p, ws, s);
  }
  return hipGetLastError();
}

}  // namespace steel
