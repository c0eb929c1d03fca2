// Page bookkeeping of the paged cache: rows forked, reordered and freed, pages
// taken for new tokens, copied on write, and live pages moved together.
//
// The page table, the lengths and the reference counts stay on the device and
// no call waits for the host; every result is fixed by the arguments alone
// (free pages are taken in increasing order, moved pages keep their order, and
// the atomics only add integers), so two runs give the same tables.
#include "cache_common.h"

namespace steel {

namespace {

__device__ __forceinline__ int pages_of(long long n) {
  return n <= 0 ? 0 : (int)((n + kBlk - 1) / kBlk);
}
// Entries of a row that its length holds.
__device__ __forceinline__ int held_pages(int len, int M) { return min(pages_of(len), M); }

// Exclusive sum of x over the workgroup's threads in order; total: the sum.
template <int WAVES>
__device__ __forceinline__ int block_scan(int x, int* lds, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int y = __shfl_up(inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();  // the previous scan's sums are read
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const int s = lds[w];
    before += w < wave ? s : 0;
    all += s;
  }
  *total = all;
  return before + inc - x;
}

// The last i < n with x[i] <= r, x increasing from x[0] <= r.
__device__ __forceinline__ int last_upto(const int* x, int n, int r) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (x[mid] <= r) lo = mid; else hi = mid;
  }
  return lo;
}

// Place of the k-th set bit.
__device__ __forceinline__ int select_bit(unsigned long long x, int k) {
  int at = 0;
#pragma unroll
  for (int w = 32; w > 0; w >>= 1) {
    const int n = (int)__popcll(x & ((1ull << w) - 1));
    if (k >= n) {
      k -= n;
      at += w;
      x >>= w;
    }
  }
  return at;
}

}  // namespace

// One workgroup per row: the new row's entries and holds, the old row's releases.
// A row that stays where it is changes no count.  Latency bound: 4.6 us for 4 rows of 9 and 64 of
// 66 pages alike.
__global__ __launch_bounds__(256) void k_pages_fork(const int32_t* __restrict__ table,
                                                    const int32_t* __restrict__ lens,
                                                    int32_t* __restrict__ refs,
                                                    const int32_t* __restrict__ parent,
                                                    int32_t* __restrict__ table_out,
                                                    int32_t* __restrict__ lens_out, int B_in, int B_out,
                                                    int M, int n_pages) {
  const int b = blockIdx.x;
  int p = b < B_out ? parent[b] : -1;
  if (p < 0 || p >= B_in) p = -1;
  if (b < B_out) {
    const int len = p < 0 ? 0 : max(lens[p], 0), n = held_pages(len, M);
    for (int j = threadIdx.x; j < M; j += 256) {
      const int id = j < n ? table[(size_t)p * M + j] : -1;
      table_out[(size_t)b * M + j] = id;
      if (p != b && id >= 0 && id < n_pages) atomicAdd(refs + id, 1);
    }
    if (threadIdx.x == 0) lens_out[b] = len;
  }
  if (b < B_in && p != b) {
    const int n = held_pages(lens[b], M);
    for (int j = threadIdx.x; j < n; j += 256) {
      const int id = table[(size_t)b * M + j];
      if (id >= 0 && id < n_pages) atomicAdd(refs + id, -1);
    }
  }
}

hipError_t launch_pages_fork(const int32_t* table, const int32_t* lens, int32_t* refs,
                             const int32_t* parent, int32_t* table_out, int32_t* lens_out, int B_in,
                             int B_out, int M, int n_pages, hipStream_t s) {
  hipLaunchKernelGGL(k_pages_fork, dim3(B_in > B_out ? B_in : B_out), dim3(256), 0, s, table, lens,
                     refs, parent, table_out, lens_out, B_in, B_out, M, n_pages);
  return hipGetLastError();
}

// One workgroup.  The pages that a sequence takes are ranks off[b] .. off[b + 1] - 1
// of the free pages in increasing order, the copy of its shared last page first.
// Of the sequences that write into a shared page all copy it, but for the last
// one where every holder writes: the others then let go of the page.  Bound by the latency of one
// workgroup's passes over the counts, two with a growth: 64 rows and 70,000 pages 24 us, 2^18 55, 2^20
// 198, 2^22 1320 (17 MB of counts); 20,000 rows and 2^20 pages 386.
__global__ __launch_bounds__(1024) void k_pages_grow(int32_t* __restrict__ table,
                                                     int32_t* __restrict__ lens,
                                                     int32_t* __restrict__ refs,
                                                     const int32_t* __restrict__ fresh,
                                                     int32_t* __restrict__ src,
                                                     int32_t* __restrict__ dst,
                                                     int32_t* __restrict__ left,
                                                     int32_t* __restrict__ took, int B, int M,
                                                     int n_pages, int32_t* ws) {
  constexpr int T = 1024;
  int32_t* writers = ws;
  int32_t* last = writers + n_pages;
  int32_t* free_at = last + n_pages;
  int32_t* off = free_at + n_pages;  // [B + 1]
  __shared__ int sums[T / 64];
  __shared__ int chunk_free[kMaxPages / kPageChunk];
  __shared__ int narrow;  // a row of the table is too short
  const int tid = threadIdx.x;
  const int chunks = (n_pages + kPageChunk - 1) / kPageChunk;
  if (tid == 0) narrow = 0;
  for (int c = tid; c < chunks; c += T) chunk_free[c] = 0;

  // the page that sequence b writes into besides fresh ones, if others hold it too
  auto shared_page = [&](int b) {
    const int len = lens[b];
    if (fresh[b] <= 0 || len <= 0 || len % kBlk == 0 || pages_of(len) > M) return -1;
    const int id = table[(size_t)b * M + pages_of(len) - 1];
    return id >= 0 && id < n_pages && refs[id] > 1 ? id : -1;
  };
  for (int b = tid; b < B; b += T) {
    const int id = shared_page(b);
    if (id >= 0) {
      atomicExch(writers + id, 0);
      atomicExch(last + id, -1);
    }
  }
  __threadfence();
  __syncthreads();
  for (int b = tid; b < B; b += T) {
    const int id = shared_page(b);
    if (id >= 0) {
      atomicAdd(writers + id, 1);
      atomicMax(last + id, b);
    }
  }
  __threadfence();
  __syncthreads();
  int demand = 0;
  for (int b0 = 0; b0 < B; b0 += T) {
    const int b = b0 + tid;
    int need = 0;
    if (b < B) {
      const long long len = max(lens[b], 0), to = len + max(fresh[b], 0);
      if (to > (long long)M * kBlk) narrow = 1;
      const int id = shared_page(b);
      const bool copy = id >= 0 && !(atomicAdd(writers + id, 0) == refs[id] && atomicMax(last + id, -1) == b);
      need = to > (long long)M * kBlk ? 0 : pages_of(to) - pages_of(len) + (copy ? 1 : 0);
      src[b] = copy ? id : -1;
      dst[b] = -1;
    }
    int all;
    const int at = demand + block_scan<T / 64>(need, sums, &all);
    if (b < B) off[b] = at;
    demand += all;
  }
  if (tid == 0) off[B] = demand;

  // free pages of every chunk
  for (int c = 0; c < chunks; ++c) {
    int n = 0;
#pragma unroll
    for (int u = 0; u < kPageChunk / T; ++u) {
      const int p = c * kPageChunk + u * T + tid;
      n += (int)__popcll(__ballot(p < n_pages && refs[p < n_pages ? p : 0] == 0));
    }
    if ((tid & 63) == 0) atomicAdd(&chunk_free[c], n);
  }
  __syncthreads();
  int total = 0;
  for (int c = 0; c < chunks; ++c) total += chunk_free[c];
  const bool fits = !narrow && total >= demand;
  if (tid == 0) left[0] = narrow ? INT_MIN : total - demand;
  if (!fits) {
    for (int b = tid; b < B; b += T) {
      src[b] = -1;
      if (took != nullptr) took[b] = 0;
    }
    return;
  }
  // the first `demand` of them in order
  for (int c = 0, base = 0; c < chunks && base < demand; base += chunk_free[c], ++c) {
    if (chunk_free[c] == 0) continue;
    constexpr int U = kPageChunk / T;
    const int p0 = c * kPageChunk + U * tid;
    bool f[U];
    int n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      f[u] = p0 + u < n_pages && refs[p0 + u < n_pages ? p0 + u : 0] == 0;
      n += f[u] ? 1 : 0;
    }
    int all, r = base + block_scan<T / 64>(n, sums, &all);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (f[u] && r < demand) free_at[r++] = p0 + u;
  }
  __threadfence();
  __syncthreads();
  for (int r = tid; r < demand; r += T) {
    const int b = last_upto(off, B, r), id = free_at[r], have = pages_of(lens[b]), old = src[b];
    const int k = r - off[b];
    refs[id] = 1;
    if (old >= 0 && k == 0) {
      table[(size_t)b * M + have - 1] = id;
      dst[b] = id;
      atomicAdd(refs + old, -1);
    } else {
      table[(size_t)b * M + have + k - (old >= 0 ? 1 : 0)] = id;
    }
  }
  __syncthreads();
  for (int b = tid; b < B; b += T) {
    const int more = max(fresh[b], 0);
    lens[b] = max(lens[b], 0) + more;
    if (took != nullptr) took[b] = more;
  }
}

// The same for up to 1024 sequences and 2^16 pages, with one sequence per thread: what a
// thread has loaded stays in registers, the free pages are a set of bits in LDS that is read
// once, and each free page finds the sequence that takes it.  Latency bound (four dependent loads, two
// scans): 64 rows and 2,600 pages 7.0 us, 19.5 with the kernel above; 4 rows 5.4.
__global__ __launch_bounds__(1024) void k_pages_grow_few(int32_t* __restrict__ table,
                                                         int32_t* __restrict__ lens,
                                                         int32_t* __restrict__ refs,
                                                         const int32_t* __restrict__ fresh,
                                                         int32_t* __restrict__ src,
                                                         int32_t* __restrict__ dst,
                                                         int32_t* __restrict__ left,
                                                         int32_t* __restrict__ took, int B, int M,
                                                         int n_pages) {
  constexpr int T = 1024;
  __shared__ unsigned long long free_set[T];  // bit i of word w: page 64 w + i is free
  __shared__ __attribute__((aligned(16))) int shared_id[T];
  __shared__ int off[T], have[T], free_before[T];
  __shared__ int sums[T / 64];
  __shared__ int narrow;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) narrow = 0;
  const int len = tid < B ? max(lens[tid], 0) : 0, more = tid < B ? max(fresh[tid], 0) : 0;
  const long long to = (long long)len + more;
  for (int p0 = 0; p0 < n_pages; p0 += T) {
    const int p = p0 + tid;
    const unsigned long long f = __ballot(p < n_pages && refs[p < n_pages ? p : 0] == 0);
    if (lane == 0) free_set[p0 / 64 + wave] = f;
  }
  int id = -1, holders = 0;
  if (more > 0 && len % kBlk != 0 && pages_of(len) <= M) {
    id = table[(size_t)tid * M + pages_of(len) - 1];
    if (id >= 0 && id < n_pages) holders = refs[id];
    if (holders <= 1) id = -1;
  }
  shared_id[tid] = id;
  __syncthreads();
  if (to > (long long)M * kBlk) narrow = 1;
  bool copy = false;
  if (id >= 0) {  // all writers copy but the last one where every holder writes
    int writers = 0, last = -1;
#pragma unroll 4
    for (int b = 0; b < B; b += 4) {  // entries past B are -1
      const int4 x = *(const int4*)(shared_id + b);
      const int y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        writers += y[u] == id ? 1 : 0;
        last = y[u] == id ? b + u : last;
      }
    }
    copy = !(writers == holders && last == tid);
  }
  const int need = to > (long long)M * kBlk ? 0 : pages_of(to) - pages_of(len) + (copy ? 1 : 0);
  int demand, total;
  const int at = block_scan<T / 64>(need, sums, &demand);
  off[tid] = at;
  have[tid] = pages_of(len) | (copy ? 1 << 30 : 0);
  const int words = (n_pages + T - 1) / T * (T / 64);
  free_before[tid] = block_scan<T / 64>(tid < words ? (int)__popcll(free_set[tid]) : 0, sums, &total);
  __syncthreads();
  const bool fits = !narrow && total >= demand;  // the scans' barriers are behind both
  if (tid == 0) left[0] = narrow ? INT_MIN : total - demand;
  if (tid < B) {
    src[tid] = fits && copy ? id : -1;
    if (!(fits && copy)) dst[tid] = -1;
    if (took != nullptr) took[tid] = fits ? more : 0;
    if (fits) lens[tid] = (int)to;
    if (fits && copy) atomicAdd(refs + id, -1);
  }
  if (!fits) return;
  for (int r = tid; r < demand; r += T) {
    const int w = last_upto(free_before, words, r);
    const int page = 64 * w + select_bit(free_set[w], r - free_before[w]);
    const int b = last_upto(off, B, r);
    const int k = r - off[b], held = have[b] & ~(1 << 30);
    const bool c = (have[b] >> 30) & 1;
    refs[page] = 1;
    if (c && k == 0) dst[b] = page;
    table[(size_t)b * M + held + k - (c ? 1 : 0)] = page;
  }
}

hipError_t launch_pages_grow(int32_t* table, int32_t* lens, int32_t* refs, const int32_t* fresh,
                             int32_t* src, int32_t* dst, int32_t* left, int32_t* took, int B, int M,
                             int n_pages, int32_t* ws, hipStream_t s) {
  if (pages_few(n_pages, B))
    hipLaunchKernelGGL(k_pages_grow_few, dim3(1), dim3(1024), 0, s, table, lens, refs, fresh, src, dst,
                       left, took, B, M, n_pages);
  else
    hipLaunchKernelGGL(k_pages_grow, dim3(1), dim3(1024), 0, s, table, lens, refs, fresh, src, dst,
                       left, took, B, M, n_pages, ws);
  return hipGetLastError();
}

// Piece of a page that a workgroup copies: 4 loads of 16 bytes in flight per thread.
constexpr int kCopyPiece = 4 * 256 * 16;

__device__ __forceinline__ void copy_piece(uint8_t* pages, long long layer_bytes,
                                           long long page_bytes, int layer, int from, int to,
                                           int piece) {
  const long long o0 = (long long)piece * kCopyPiece + 16 * threadIdx.x;
  const uint8_t* s = pages + layer * layer_bytes + from * page_bytes;
  uint8_t* d = pages + layer * layer_bytes + to * page_bytes;
  u32x4 x[4];
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (o0 + u * 4096 < page_bytes) x[u] = *(const u32x4*)(s + o0 + u * 4096);
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (o0 + u * 4096 < page_bytes) *(u32x4*)(d + o0 + u * 4096) = x[u];
}

// A workgroup per piece and layer.  Latency bound: 11 pages of 70 KB in two layers, 3 MB read and
// written, 5.2 us; one page 4.7.
__global__ __launch_bounds__(256) void k_pages_copy(uint8_t* pages, long long layer_bytes,
                                                    long long page_bytes, int pieces,
                                                    const int32_t* __restrict__ src,
                                                    const int32_t* __restrict__ dst, int n_pages) {
  const int i = blockIdx.x / pieces, piece = blockIdx.x % pieces;
  const int from = src[i], to = dst[i];
  if (from < 0 || from >= n_pages || to < 0 || to >= n_pages || from == to) return;
  copy_piece(pages, layer_bytes, page_bytes, blockIdx.y, from, to, piece);
}

hipError_t launch_pages_copy(uint8_t* pages, long long layer_bytes, long long page_bytes, int layers,
                             const int32_t* src, const int32_t* dst, int n, int n_pages,
                             hipStream_t s) {
  const int pieces = (int)((page_bytes + kCopyPiece - 1) / kCopyPiece);
  hipLaunchKernelGGL(k_pages_copy, dim3((unsigned)(n * pieces), layers), dim3(256), 0, s, pages,
                     layer_bytes, page_bytes, pieces, src, dst, n_pages);
  return hipGetLastError();
}

// Compaction.  With n live pages, the live ones at n or behind (in order) move
// to the free ones before n (in order): no page is read after it was written.
__global__ __launch_bounds__(256) void k_pages_count(const int32_t* __restrict__ refs, int n_pages,
                                                     int32_t* __restrict__ chunk_live) {
  __shared__ int sums[4];
  int n = 0;
#pragma unroll
  for (int u = 0; u < kPageChunk / 256; ++u) {
    const int p = blockIdx.x * kPageChunk + u * 256 + threadIdx.x;
    n += p < n_pages && refs[p < n_pages ? p : 0] > 0 ? 1 : 0;
  }
  int all;
  (void)block_scan<4>(n, sums, &all);
  if (threadIdx.x == 0) chunk_live[blockIdx.x] = all;
}

// head: {live, moves}; hole[r], mover[r]: the r-th move; rank[p]: the move of page p; to[p] (may
// be nullptr): p, or -1 for a free page (k_pages_move changes those that move)
__global__ __launch_bounds__(256) void k_pages_rank(const int32_t* __restrict__ refs, int n_pages,
                                                    const int32_t* __restrict__ chunk_live,
                                                    int32_t* __restrict__ head,
                                                    int32_t* __restrict__ hole,
                                                    int32_t* __restrict__ mover,
                                                    int32_t* __restrict__ rank,
                                                    int32_t* __restrict__ to,
                                                    int32_t* __restrict__ live_out) {
  constexpr int U = kPageChunk / 256;
  __shared__ int sums[4];
  const int chunks = gridDim.x, c = blockIdx.x;
  auto is_live = [&](int p) { return p < n_pages && refs[p < n_pages ? p : 0] > 0; };
  auto live_of = [&](int from, int to) {  // live pages of chunks [from, to)
    int n = 0, all;
    for (int i = from + threadIdx.x; i < to; i += 256) n += chunk_live[i];
    (void)block_scan<4>(n, sums, &all);
    return all;
  };
  const int live = live_of(0, chunks);
  // live pages before page number `live`
  const int cl = min(live / kPageChunk, chunks - 1);
  int stay = 0, all;
  for (int u = 0; u < U; ++u) {
    const int p = cl * kPageChunk + u * 256 + threadIdx.x;
    stay += p < live && is_live(p) ? 1 : 0;
  }
  (void)block_scan<4>(stay, sums, &all);
  stay = all + live_of(0, cl);
  // this chunk's pages, 16 in a row per thread
  int before = live_of(0, c), n = 0;
  uint32_t f = 0;
  const int p0 = c * kPageChunk + U * threadIdx.x;
#pragma unroll
  for (int u = 0; u < U; ++u) f |= is_live(p0 + u) ? 1u << u : 0u;
  n = __popc(f);
  before += block_scan<4>(n, sums, &all);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int p = p0 + u;
    const bool l = (f >> u) & 1;
    if (to != nullptr && p < n_pages) to[p] = l ? p : -1;
    if (l && p >= live) {
      mover[before - stay] = p;
      rank[p] = before - stay;
    } else if (!l && p < live) {
      hole[p - before] = p;
    }
    before += l ? 1 : 0;
  }
  if (c == 0 && threadIdx.x == 0) {
    head[0] = live;
    head[1] = live - stay;
    live_out[0] = live;
  }
}

// Both for up to 2^16 pages: one workgroup with the live pages as a set of bits in LDS, a word of
// 64 pages per thread.  Latency bound: 70 pages 5.0 us against 4.8 + 6.8, 1,728 pages 6.7.
__global__ __launch_bounds__(1024) void k_pages_rank_few(const int32_t* __restrict__ refs, int n_pages,
                                                         int32_t* __restrict__ head,
                                                         int32_t* __restrict__ hole,
                                                         int32_t* __restrict__ mover,
                                                         int32_t* __restrict__ rank,
                                                         int32_t* __restrict__ to,
                                                         int32_t* __restrict__ live_out) {
  constexpr int T = 1024;
  __shared__ unsigned long long live_set[T];
  __shared__ int sums[T / 64];
  __shared__ int kept;  // live pages before page number `live`
  const int tid = threadIdx.x;
  for (int p0 = 0; p0 < n_pages; p0 += T) {
    const int p = p0 + tid;
    const bool l = p < n_pages && refs[p < n_pages ? p : 0] > 0;
    if (to != nullptr && p < n_pages) to[p] = l ? p : -1;
    const unsigned long long f = __ballot(l);
    if ((tid & 63) == 0) live_set[p0 / 64 + (tid >> 6)] = f;
  }
  if (tid == 0) kept = 0;
  __syncthreads();
  const unsigned long long mine = tid < (n_pages + T - 1) / T * (T / 64) ? live_set[tid] : 0;
  int live;
  int before = block_scan<T / 64>((int)__popcll(mine), sums, &live);
  if (live / 64 == tid) kept = before + (int)__popcll(mine & ((1ull << (live % 64)) - 1));
  if (live == 64 * T && tid == 0) kept = live;
  __syncthreads();
  const int stay = kept;
  const int p0 = 64 * tid, p1 = min(p0 + 64, n_pages);
  if (p0 < live) {  // free pages below `live`
    unsigned long long f = ~mine;
    if (min(live, p1) - p0 < 64) f &= (1ull << (min(live, p1) - p0)) - 1;
    for (int r = p0 - before; f != 0; f &= f - 1, ++r) hole[r] = p0 + __builtin_ctzll(f);
  }
  if (p1 > live) {  // live pages from there on
    unsigned long long f = mine;
    int r = before - stay;
    if (live > p0) {
      f &= ~((1ull << (live - p0)) - 1);
      r = 0;
    }
    for (; f != 0; f &= f - 1, ++r) {
      const int p = p0 + __builtin_ctzll(f);
      mover[r] = p;
      rank[p] = r;
    }
  }
  if (tid == 0) {
    head[0] = live;
    head[1] = live - stay;
    live_out[0] = live;
  }
}

// The first `rows` workgroups rewrite the page table (one row each) and the first
// of them the counts; the others copy the moved pages.  Memory bound: 79 MB read and written in 16.5 us
// out of a cold cache, where a plain copy of that size takes 14.5; 2048 copying workgroups at
// most, since only the device knows how many pages move.
__global__ __launch_bounds__(256) void k_pages_move(uint8_t* pages, long long layer_bytes,
                                                    long long page_bytes, int layers, int pieces,
                                                    int32_t* __restrict__ table,
                                                    const int32_t* __restrict__ lens,
                                                    int32_t* __restrict__ refs, int rows, int M,
                                                    int n_pages, const int32_t* __restrict__ head,
                                                    const int32_t* __restrict__ hole,
                                                    const int32_t* __restrict__ mover,
                                                    const int32_t* __restrict__ rank,
                                                    int32_t* __restrict__ to) {
  const int live = head[0], moves = head[1];
  if ((int)blockIdx.x < rows) {
    const int b = blockIdx.x, n = held_pages(lens[b], M);
    for (int j = threadIdx.x; j < n; j += 256) {
      const int id = table[(size_t)b * M + j];
      if (id < live || id >= n_pages) continue;
      const int r = rank[id];  // not written for a page that no row holds
      if (r >= 0 && r < moves && mover[r] == id) table[(size_t)b * M + j] = hole[r];
    }
    if (b == 0)
      for (int r = threadIdx.x; r < moves; r += 256) {
        refs[hole[r]] = refs[mover[r]];
        refs[mover[r]] = 0;
        if (to != nullptr) to[mover[r]] = hole[r];
      }
    return;
  }
  const long long units = (long long)moves * layers * pieces;
  for (long long u = blockIdx.x - rows; u < units; u += gridDim.x - rows) {
    const int piece = (int)(u % pieces), layer = (int)(u / pieces % layers);
    const int r = (int)(u / pieces / layers);
    copy_piece(pages, layer_bytes, page_bytes, layer, mover[r], hole[r], piece);
  }
}

hipError_t launch_pages_compact(uint8_t* pages, long long layer_bytes, long long page_bytes,
                                int layers, int32_t* table, const int32_t* lens, int32_t* refs,
                                int32_t* live, int32_t* to, int B, int M, int n_pages, int32_t* ws,
                                hipStream_t s) {
  const int chunks = (n_pages + kPageChunk - 1) / kPageChunk;
  int32_t* hole = ws;
  int32_t* mover = hole + n_pages;
  int32_t* rank = mover + n_pages;
  int32_t* chunk_live = rank + n_pages;
  int32_t* head = chunk_live + chunks;
  const int pieces = (int)((page_bytes + kCopyPiece - 1) / kCopyPiece);
  const long long most = (long long)(n_pages / 2) * layers * pieces;  // moves <= n_pages / 2
  const int copiers = (int)(most < 2048 ? (most > 0 ? most : 1) : 2048);
  if (n_pages <= 65536) {
    hipLaunchKernelGGL(k_pages_rank_few, dim3(1), dim3(1024), 0, s, refs, n_pages, head, hole, mover,
                       rank, to, live);
  } else {
    hipLaunchKernelGGL(k_pages_count, dim3(chunks), dim3(256), 0, s, refs, n_pages, chunk_live);
    hipLaunchKernelGGL(k_pages_rank, dim3(chunks), dim3(256), 0, s, refs, n_pages, chunk_live, head,
                       hole, mover, rank, to, live);
  }
  hipLaunchKernelGGL(k_pages_move, dim3(B + copiers), dim3(256), 0, s, pages, layer_bytes, page_bytes,
                     layers, pieces, table, lens, refs, B, M, n_pages, head, hole, mover, rank, to);
  return hipGetLastError();
}

}  // namespace steel
