// Keys and values into the paged 4-bit cache, and back out of it as bf16.
//
// Quantisation of a token's vector x (D channels in bf16), per 32 channels:
//   2^e = the smallest power of two with max |x| <= 6 * 2^e, e in [-125, 125]
//   code = x / 2^e rounded to the nearest E2M1 number, ties to the even code
// so a value is off by at most half a step of its own size and none saturates
// below 6 * 2^125.  A vector with a non-finite element gets scale bytes of 255.
// All of it is integer work on the bf16 bits and one conversion per pair:
// |x| as 15 bits orders like the value, E - 2 (+ 1 where the mantissa is above
// 1.5) is the scale byte.
//
// Memory bound: a lane takes 8 channels (16 bytes of bf16, 4 of codes), the
// lanes of a vector are neighbours and so are the tokens of a head, so a wave
// reads 1 KiB and writes 256 bytes of codes contiguously per tensor.  Prompts of 8,586 tokens in
// all (8 heads of 128) out of a cold cache: written in 15.2 us, read back into 4 x 8192 padded rows
// in 20.4; 160 MB together at 4.5 TB/s, where a plain copy of as many bytes takes 27 us.
// One token of 64 sequences: 4.8 us, a launch and two dependent loads.
#include "cache_common.h"

namespace steel {

namespace {

typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Packed maximum of |x| (bf16 bits) over 8 channels, then over the lanes l ^ 1, l ^ 2.
__device__ __forceinline__ uint32_t group_amax(u32x4 x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = x[i] & 0x7fff7fffu;
    m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m),
                                                               __builtin_bit_cast(u16x2, w)));
  }
  m = max(m & 0xffffu, m >> 16);
  m = max(m, (uint32_t)__shfl_xor((int)m, 1));
  return max(m, (uint32_t)__shfl_xor((int)m, 2));
}

// 8 channels of one vector into the record; the D / 8 lanes of a vector are
// neighbours, sub is the lane's place among them.
template <int D>
__device__ __forceinline__ void store8(u32x4 x, uint8_t* codes, uint8_t* scales, int sub) {
  constexpr int L = D / 8;
  const uint32_t m = group_amax(x);
  uint32_t all = m;  // the vector's maximum: is any element non-finite?
#pragma unroll
  for (int o = 4; o < L; o *= 2) all = max(all, (uint32_t)__shfl_xor((int)all, o));
  const bool bad = all >= 0x7f80u;
  int e = (int)(m >> 7) - 2 + ((m & 0x7fu) > 0x40u ? 1 : 0);
  e = min(max(e, kScaleMin), kScaleMax);
  const float sc = __uint_as_float((uint32_t)e << 23);
  uint32_t w = 0;
  const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x0), sc, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x1), sc, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x2), sc, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x3), sc, 3);
  *(uint32_t*)(codes + 4 * sub) = bad ? 0u : w;
  if ((sub & 3) == 0) scales[sub >> 2] = (uint8_t)(bad ? kScaleNan : e);
}

// 8 channels of one stored vector in bf16.
__device__ __forceinline__ u32x4 load8(uint32_t w, uint32_t e) {
  const float sc = __uint_as_float(e << 23);
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, sc, 3));
  if (e == (uint32_t)kScaleNan) r = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
  return r;
}

// The record of a token's page, or nullptr where the token has none.
template <int D, typename T>
__device__ __forceinline__ T* token_record(T* pages, const int32_t* table, int M, int n_pages,
                                           int Hkv, int b, int g, long long pos) {
  if (pos < 0 || pos >= (long long)M * kBlk) return nullptr;
  const int id = table[(size_t)b * M + (int)(pos / kBlk)];
  if (id < 0 || id >= n_pages) return nullptr;
  return pages + ((size_t)id * Hkv + g) * Record<D>::kBytes;
}

}  // namespace

template <int D>
__global__ __launch_bounds__(256) void k_cache_append(StoreArgs a) {
  constexpr int L = D / 8;
  const long long vec = ((long long)blockIdx.x * 256 + threadIdx.x) / L;
  const int sub = threadIdx.x % L;
  if (vec >= (long long)a.B * a.Hkv * a.S) return;  // whole vectors: their lanes leave together
  const int i = (int)(vec % a.S), bg = (int)(vec / a.S), g = bg % a.Hkv, b = bg / a.Hkv;
  const int n = a.fresh == nullptr ? a.S : min(max(a.fresh[b], 0), a.S);
  if (i >= n) return;
  const long long pos = (long long)a.lens[b] - n + i;
  uint8_t* rec = token_record<D>(a.pages, a.table, a.M, a.n_pages, a.Hkv, b, g, pos);
  if (rec == nullptr) return;
  const int t = (int)(pos % kBlk);
  const u32x4 xk = *(const u32x4*)(a.k + b * a.k_sb + g * a.k_sh + i * a.k_ss + 8 * sub);
  const u32x4 xv = *(const u32x4*)(a.v + b * a.v_sb + g * a.v_sh + i * a.v_ss + 8 * sub);
  using R = Record<D>;
  store8<D>(xk, rec + t * R::kRow, rec + R::kKs + t * R::kGroups, sub);
  store8<D>(xv, rec + R::kV + t * R::kRow, rec + R::kVs + t * R::kGroups, sub);
}

template <int D>
__global__ __launch_bounds__(256) void k_cache_load(LoadArgs a) {
  constexpr int L = D / 8;
  const long long vec = ((long long)blockIdx.x * 256 + threadIdx.x) / L;
  const int sub = threadIdx.x % L;
  if (vec >= (long long)a.B * a.Hkv * a.S) return;
  const int i = (int)(vec % a.S), bg = (int)(vec / a.S), g = bg % a.Hkv, b = bg / a.Hkv;
  const long long pos = (a.start == nullptr ? 0ll : (long long)a.start[b]) + i;
  const uint8_t* rec = pos >= a.lens[b] ? nullptr
                                        : token_record<D>(a.pages, a.table, a.M, a.n_pages, a.Hkv, b, g, pos);
  u32x4 xk = {0u, 0u, 0u, 0u}, xv = xk;
  if (rec != nullptr) {
    using R = Record<D>;
    const int t = (int)(pos % kBlk);
    const uint32_t wk = *(const uint32_t*)(rec + t * R::kRow + 4 * sub);
    const uint32_t wv = *(const uint32_t*)(rec + R::kV + t * R::kRow + 4 * sub);
    xk = load8(wk, rec[R::kKs + t * R::kGroups + (sub >> 2)]);
    xv = load8(wv, rec[R::kVs + t * R::kGroups + (sub >> 2)]);
  }
  *(u32x4*)(a.k + vec * D + 8 * sub) = xk;
  *(u32x4*)(a.v + vec * D + 8 * sub) = xv;
}

hipError_t launch_cache_append(const StoreArgs& a, int D, hipStream_t s) {
  const long long threads = (long long)a.B * a.Hkv * a.S * (D / 8);
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (D == 64)
    hipLaunchKernelGGL(k_cache_append<64>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(k_cache_append<128>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_cache_load(const LoadArgs& a, int D, hipStream_t s) {
  const long long threads = (long long)a.B * a.Hkv * a.S * (D / 8);
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (D == 64)
    hipLaunchKernelGGL(k_cache_load<64>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(k_cache_load<128>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace steel
