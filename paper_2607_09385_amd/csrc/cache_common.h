// The paged 4-bit key/value cache: record layout, arguments and launches.
//
// A page holds 64 tokens (the mask block edge, so a page is one key tile).  The
// record of a page and a key/value head is 68 D contiguous bytes,
//   key codes    [64][D/2]   low nibble: even channel
//   value codes  [64][D/2]
//   key scales   [64][D/32]
//   value scales [64][D/32]
// A code is an E2M1 number (0 .5 1 1.5 2 3 4 6 and a sign) and a scale byte b
// stands for 2^(b - 127), shared by 32 channels of one token: the operands of
// gfx950's scaled conversions, which turn two codes and a scale into two bf16
// values without rounding.  Scale bytes of stored vectors are 2 .. 252 (every
// value they give is a normal bf16 number); 255 stands for NaN.
#pragma once

#include "attn_common.h"

namespace steel {

constexpr int kScaleMin = 2, kScaleMax = 252, kScaleNan = 255;

template <int D>
struct Record {
  static constexpr int kRow = D / 2, kGroups = D / 32;  // bytes of codes, scales per token
  static constexpr int kV = 32 * D, kKs = 64 * D, kVs = 66 * D, kBytes = 68 * D;
};

// Rows of a call are taken query by query with the G heads of a key/value head
// next to each other: row r is query r / G and head g * G + r % G, so a tile of
// rows covers few positions and all heads that share keys.
struct CacheArgs {
  const __bf16* q;
  long long q_sb, q_sh, q_ss;  // strides of q in elements (batch, head, query)
  const uint8_t* pages;
  const int32_t* table;  // [B][M]
  const int32_t* lens;   // [B]
  const int32_t* fresh;  // [B] queries of each sequence, or nullptr: S_q
  const uint8_t* mask;   // [B][Hkv][M], or nullptr
  void* out;
  float* lse;
  int out_bf16, B, Hq, Hkv, G, S_q, M, n_pages, causal, win, sink;
  float c;  // scale * log2(e)
};

struct StoreArgs {
  const __bf16* k;
  const __bf16* v;
  long long k_sb, k_sh, k_ss, v_sb, v_sh, v_ss;  // strides in elements
  uint8_t* pages;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* fresh;  // [B] tokens of each sequence, or nullptr: S
  int B, Hkv, S, M, n_pages;
};

struct LoadArgs {
  const uint8_t* pages;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* start;  // [B] first token, or nullptr: 0
  __bf16* k;
  __bf16* v;
  int B, Hkv, S, M, n_pages;
};

hipError_t launch_cache_append(const StoreArgs& a, int D, hipStream_t s);
hipError_t launch_cache_load(const LoadArgs& a, int D, hipStream_t s);

// Workspace bytes of the attention for these sizes, with a page mask or without (0: none is used).
size_t cache_attn_ws(int B, int Hq, int Hkv, int S_q, int D, int M, bool masked);
hipError_t launch_cache_attn(const CacheArgs& a, int D, void* ws, hipStream_t s);

// Page bookkeeping (cache_pages.hip).  Pages are counted in chunks of kPageChunk.
constexpr int kPageChunk = 4096;
constexpr int kMaxPages = kPageChunk * 1024;

hipError_t launch_pages_fork(const int32_t* table, const int32_t* lens, int32_t* refs,
                             const int32_t* parent, int32_t* table_out, int32_t* lens_out, int B_in,
                             int B_out, int M, int n_pages, hipStream_t s);

// Up to 1024 rows and 2^16 pages one thread takes a row and LDS holds all that a growth needs.
inline bool pages_few(int n_pages, int B) { return B <= 1024 && n_pages <= 65536; }

// Workspace of pages_grow: {writers, last writer} per page, the free pages by
// rank, the first rank of each sequence; none where pages_few.  took: may be nullptr.
hipError_t launch_pages_grow(int32_t* table, int32_t* lens, int32_t* refs, const int32_t* fresh,
                             int32_t* src, int32_t* dst, int32_t* left, int32_t* took, int B, int M,
                             int n_pages, int32_t* ws, hipStream_t s);

hipError_t launch_pages_copy(uint8_t* pages, long long layer_bytes, long long page_bytes, int layers,
                             const int32_t* src, const int32_t* dst, int n, int n_pages, hipStream_t s);

// Workspace of pages_compact: live pages per chunk, {live, moves}, holes and
// moved pages by rank, the rank of each moved page.  to: may be nullptr.
hipError_t launch_pages_compact(uint8_t* pages, long long layer_bytes, long long page_bytes,
                                int layers, int32_t* table, const int32_t* lens, int32_t* refs,
                                int32_t* live, int32_t* to, int B, int M, int n_pages, int32_t* ws,
                                hipStream_t s);

inline size_t pages_ws_ints(int n_pages, int B) {
  return 3 * (size_t)n_pages + (size_t)B + kMaxPages / kPageChunk + 64;
}

}  // namespace steel
