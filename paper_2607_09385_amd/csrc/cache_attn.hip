// Attention of new queries over the paged 4-bit cache.
//
//   o_r = sum_j p_rj v_j,  p_rj = 2^(c q_r . k_j - m_r) / l_r,  c = scale log2 e
// over the keys j that row r sees, with the online softmax (running maximum m,
// running sum l in fp32) over pages of 64 tokens.
//
// Operands.  S^T = K Q^T and O^T = V^T P^T on 16x16x32 bf16 MFMAs, so a query
// row is a column of every result and its m, l and rescaling stay in the lanes
// l % 16 = row.  Lane (n = l % 16, q = l / 16) of the K operand takes D / 4
// consecutive channels of token n: one 16-byte (D = 128) load of codes straight
// into registers, with one scale byte, since any order of the channels will do as
// long as Q has the same.  Two codes and the scale become two bf16 values in one
// instruction, without rounding.  The scores arrive with tokens 4 q .. 4 q + 3 of
// each 16 in a lane, which is what the P^T operand takes when the tokens of a
// page are numbered in that order; V goes through LDS, where a transposing read
// of 4-bit elements gives each lane 16 tokens of one channel in the same order.
// V's scales differ from token to token, along the sum, so they go into the
// weights: p_rj 2^e_jg is formed once per group of 32 channels (a power of two:
// exact) and rounded to bf16, the precision of the MFMA's operands (2^-9 of each
// weight, averaged over the keys); l adds the weights before that rounding.
//
// A page id outside the pool is a page without visible keys; keys behind the
// sequence's length are never visible, whatever their bytes.
#include "cache_common.h"

namespace steel {

namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// Rows r0 .. r1 - 1 of (b, g): their positions and the pages that any of them sees,
// [0, a_len) and [b0, b0 + count - a_len).
struct Span {
  int keys;              // keys that exist
  long long first;       // position of query 0
  int n;                 // queries of the sequence
  long long pmin, pmax;  // positions of the rows
  int a_len, b0, count;
};

__device__ __forceinline__ Span make_span(const CacheArgs& a, int b, int r0, int r1) {
  Span s;
  const int len = a.lens[b];
  s.n = a.fresh == nullptr ? a.S_q : min(max(a.fresh[b], 0), a.S_q);
  s.keys = (int)min((long long)max(len, 0), (long long)a.M * kBlk);
  s.first = (long long)len - s.n;
  s.pmin = s.first + r0 / a.G;
  s.pmax = s.first + min((r1 - 1) / a.G, s.n - 1);
  s.a_len = s.b0 = s.count = 0;
  if (s.pmax < s.pmin || s.pmax < 0) return s;
  int kend = (s.keys + kBlk - 1) / kBlk;
  if (a.causal) kend = (int)min((long long)kend, s.pmax / kBlk + 1);
  s.a_len = s.count = kend;
  if (a.win > 0) {
    s.a_len = min(a.sink, kend);
    s.b0 = (int)max((long long)s.a_len, max(s.pmin, 0ll) / kBlk - a.win + 1);
    s.count = s.a_len + max((int)min((long long)kend, s.pmax / kBlk + 1) - s.b0, 0);
  }
  return s;
}

__device__ __forceinline__ int span_page(const Span& s, int i) {
  return i < s.a_len ? i : s.b0 + (i - s.a_len);
}

// Whether every row of the span sees every key of page kb.
__device__ __forceinline__ bool page_full(const CacheArgs& a, const Span& s, int kb) {
  bool full = s.pmin >= 0 && (kb + 1) * (long long)kBlk <= s.keys;
  if (a.causal) full = full && (kb + 1) * (long long)kBlk - 1 <= s.pmin;
  if (a.win > 0 && kb >= a.sink) full = full && kb <= s.pmin / kBlk && kb > s.pmax / kBlk - a.win;
  return full;
}

// Last key of page kb (0 .. 63, or -1) that the query at position pos sees.
__device__ __forceinline__ int row_limit(const CacheArgs& a, const Span& s, long long pos, int kb) {
  if (pos < 0) return -1;
  if (a.win > 0 && kb >= a.sink && (kb > pos / kBlk || kb <= pos / kBlk - a.win)) return -1;
  long long last = s.keys - 1;
  if (a.causal) last = min(last, pos);
  return (int)max(min(last - (long long)kb * kBlk, 63ll), -1ll);
}

// Maximum or sum over the lanes l % 16 (the four lane groups of a row).
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ uint32_t bf16_bits(__bf16 x) {
  return (uint32_t)__builtin_bit_cast(unsigned short, x);
}

// 8 codes and their scale as 8 bf16 values.
__device__ __forceinline__ bf16x8 decode8(uint32_t w, float sc) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

constexpr int kWaves = 4;
constexpr int kRows = 16;

// One page's codes and scales of a wave, on their way to registers.
template <int D>
struct PageRegs {
  static constexpr int KW = D / 32;  // dwords of K codes per lane and 16 tokens
  uint32_t k[4][KW];
  uint32_t v[4][KW];
  uint32_t ks, vs;  // scales of token `lane` (D / 32 bytes)
};

}  // namespace

// One workgroup per (sequence, key/value head, 16 rows); its waves take every
// fourth live page, each with a state of its own, joined at the end.
template <int D>
__global__ __launch_bounds__(64 * kWaves) void k_cache_attn(CacheArgs a, int tiles) {
  using R = Record<D>;
  using Regs = PageRegs<D>;
  constexpr int KW = Regs::KW;      // also: K steps of 32 channels
  constexpr int GR = D / 32;        // scale groups
  constexpr int CT = D / 16;        // channel tiles of the output
  constexpr int VROW = D / 2;       // bytes of a token's V codes
  constexpr int OP = D + 4;         // padded output row in LDS
  constexpr int kWaveBytes = 64 * VROW + 64 * GR * 2;
  constexpr int kJoinBytes = kWaves * kRows * (OP + 2) * 4;
  constexpr int kLds = kWaves * kWaveBytes > kJoinBytes ? kWaves * kWaveBytes : kJoinBytes;
  __shared__ __attribute__((aligned(16))) char lds[kLds];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, q4 = lane >> 4;
  const int tile = blockIdx.x % tiles, bg = blockIdx.x / tiles;
  const int g = bg % a.Hkv, b = bg / a.Hkv;
  const int r0 = tile * kRows, r1 = min(r0 + kRows, a.S_q * a.G);
  const Span sp = make_span(a, b, r0, r1);

  // this lane's query row, and its part of Q as the B operand
  const int row = r0 + n, qi = row / a.G, h = g * a.G + row % a.G;
  const bool real = row < r1 && qi < sp.n;
  const long long pos = real ? sp.first + qi : -1;
  bf16x8 qf[KW];
#pragma unroll
  for (int s = 0; s < KW; ++s) qf[s] = bf16x8{};
  if (real) {
    const __bf16* qp = a.q + b * a.q_sb + h * a.q_sh + qi * a.q_ss + q4 * (D / 4);
#pragma unroll
    for (int s = 0; s < KW; ++s) qf[s] = *(const bf16x8*)(qp + 8 * s);
  }

  char* wv = lds + wave * kWaveBytes;        // V codes, then K scales, V scales
  char* wks = wv + 64 * VROW;
  char* wvs = wks + 64 * GR;

  f32x4 o[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  for (int i = wave; i < sp.count; i += kWaves) {
    const int kb = span_page(sp, i);
    const int id = a.table[(size_t)b * a.M + kb];
    if (id < 0 || id >= a.n_pages) continue;
    if (a.mask != nullptr && a.mask[((size_t)b * a.Hkv + g) * a.M + kb] == 0) continue;
    const uint8_t* rec = a.pages + ((size_t)id * a.Hkv + g) * R::kBytes;
    Regs x;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      __builtin_memcpy(x.k[t], rec + (16 * t + n) * R::kRow + q4 * 4 * KW, 4 * KW);
      __builtin_memcpy(x.v[t], rec + R::kV + (16 * t + n) * R::kRow + q4 * 4 * KW, 4 * KW);
    }
    if constexpr (GR == 4) {
      x.ks = *(const uint32_t*)(rec + R::kKs + 4 * lane);
      x.vs = *(const uint32_t*)(rec + R::kVs + 4 * lane);
      *(uint32_t*)(wks + 4 * lane) = x.ks;
      *(uint32_t*)(wvs + 4 * lane) = x.vs;
    } else {
      x.ks = *(const unsigned short*)(rec + R::kKs + 2 * lane);
      x.vs = *(const unsigned short*)(rec + R::kVs + 2 * lane);
      *(unsigned short*)(wks + 2 * lane) = (unsigned short)x.ks;
      *(unsigned short*)(wvs + 2 * lane) = (unsigned short)x.vs;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
      __builtin_memcpy(wv + (16 * t + n) * VROW + q4 * 4 * KW, x.v[t], 4 * KW);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");

    // S^T: 4 tiles of 16 tokens
    f32x4 sc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t e = (uint8_t)wks[(16 * t + n) * GR + q4 * GR / 4];
      const float ksc = __uint_as_float(e << 23);
      sc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KW; ++s) {
        bf16x8 kf = decode8(x.k[t][s], ksc);
        if (__builtin_amdgcn_ballot_w64(e == kScaleNan)) {
          const __bf16 nan = __builtin_bit_cast(__bf16, (unsigned short)0x7fc0);
          if (e == kScaleNan) kf = bf16x8{nan, nan, nan, nan, nan, nan, nan, nan};
        }
        sc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[s], sc[t], 0, 0, 0);
      }
    }
    const bool full = page_full(a, sp, kb);
    if (!full) {
      const int lim = row_limit(a, sp, pos, kb) - 4 * q4;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[t][r] = 16 * t + r > lim ? -INFINITY : sc[t][r];
    }
    float mx = sc[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sc[t][r]);
    const float mnew = fmaxf(m, row_max(mx) * a.c);
    const float alpha = mnew == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mnew);
    const float ms = mnew == -INFINITY ? 0.f : mnew;
    m = mnew;
    l *= alpha;
#pragma unroll
    for (int c = 0; c < CT; ++c) o[c] *= alpha;
    float p[16];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[4 * t + r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][r], a.c, -ms));
        l += p[4 * t + r];
      }
    // V scales of this lane's tokens 16 t + 4 q4 + r
    uint32_t ve[16];
    bool nan_seen = false;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const char* at = wvs + (16 * t + 4 * q4 + r) * GR;
        ve[4 * t + r] = GR == 4 ? *(const uint32_t*)at : *(const unsigned short*)at;
        nan_seen |= (ve[4 * t + r] & 0xff) == kScaleNan;  // all of a vector's bytes or none
      }
    const bool any_nan = __builtin_amdgcn_ballot_w64(nan_seen) != 0;
#pragma unroll
    for (int gr = 0; gr < GR; ++gr) {
      bf16x8 pf[2];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float w = p[e] * __uint_as_float(((ve[e] >> (8 * gr)) & 0xff) << 23);
        if (any_nan && ((ve[e] >> (8 * gr)) & 0xff) == kScaleNan)
          w = sc[e / 4][e % 4] == -INFINITY ? 0.f : NAN;
        pf[e / 8][e % 8] = (__bf16)w;
      }
#pragma unroll
      for (int c2 = 0; c2 < 2; ++c2) {
        const int ct = 2 * gr + c2;
        const int tok = 16 * (n >> 2) + 4 * q4 + (n & 3);
        const i32x2 w = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2*)(wv + tok * VROW + 8 * ct));
        o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8((uint32_t)w[0], 1.f), pf[0], o[ct], 0, 0, 0);
        o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8((uint32_t)w[1], 1.f), pf[1], o[ct], 0, 0, 0);
      }
    }
  }
  l = row_sum(l);

  // the waves' states of a row joined
  __syncthreads();
  float* jo = (float*)lds;                       // [wave][row][OP]
  float* jml = jo + kWaves * kRows * OP;         // [wave][row][2]
#pragma unroll
  for (int c = 0; c < CT; ++c)
    *(f32x4*)(jo + (wave * kRows + n) * OP + 16 * c + 4 * q4) = o[c];
  if (q4 == 0) {
    jml[(wave * kRows + n) * 2] = m;
    jml[(wave * kRows + n) * 2 + 1] = l;
  }
  __syncthreads();
  constexpr int TPR = 64 * kWaves / kRows;  // threads per row
  constexpr int EPT = D / TPR;              // elements per thread
  const int jr = threadIdx.x / TPR, d0 = threadIdx.x % TPR * EPT;
  if (r0 + jr >= r1) return;
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, jml[(w * kRows + jr) * 2]);
  const float ts = top == -INFINITY ? 0.f : top;
  float den = 0.f, acc[EPT];
#pragma unroll
  for (int e = 0; e < EPT; ++e) acc[e] = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float f = __builtin_amdgcn_exp2f(jml[(w * kRows + jr) * 2] - ts);
    den += f * jml[(w * kRows + jr) * 2 + 1];
#pragma unroll
    for (int e = 0; e < EPT; ++e) acc[e] += f * jo[(w * kRows + jr) * OP + d0 + e];
  }
  const int jq = (r0 + jr) / a.G, jh = g * a.G + (r0 + jr) % a.G;
  const bool dead = jq >= sp.n || sp.first + jq < 0 || den == 0.f;
  const float inv = dead ? 0.f : 1.f / den;
  const size_t orow = ((size_t)b * a.Hq + jh) * a.S_q + jq;
#pragma unroll
  for (int e = 0; e < EPT; ++e) {
    const float v = dead ? 0.f : acc[e] * inv;
    if (a.out_bf16) ((__bf16*)a.out)[orow * D + d0 + e] = (__bf16)v;
    else ((float*)a.out)[orow * D + d0 + e] = v;
  }
  if (d0 == 0 && a.lse != nullptr)
    a.lse[orow] = dead ? -INFINITY : (ts + __builtin_amdgcn_logf(den)) * 0.6931471805599453f;
}

size_t cache_attn_ws(int B, int Hq, int Hkv, int S_q, int D, int M) { return 256; }

hipError_t launch_cache_attn(const CacheArgs& a, int D, void* ws, hipStream_t s) {
  const int tiles = (a.S_q * a.G + kRows - 1) / kRows;
  const dim3 grid((unsigned)(a.B * a.Hkv * tiles));
  if (D == 64)
    hipLaunchKernelGGL(k_cache_attn<64>, grid, dim3(64 * kWaves), 0, s, a, tiles);
  else
    hipLaunchKernelGGL(k_cache_attn<128>, grid, dim3(64 * kWaves), 0, s, a, tiles);
  return hipGetLastError();
}

}  // namespace steel
