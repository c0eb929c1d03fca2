/*
 * libsteel -- sparsity-aware fused attention forward for AMD Instinct MI355X
 * (gfx950).  C ABI: plain pointers and sizes, no C++ or framework types.
 *
 * What it computes (Section II-A, Eq. 1 of the STEEL paper, with the masking
 * of Section IV-A):  for every batch b and query head h, with key/value head
 * g = h / (Hq / Hkv),
 *
 *     O[b,h,i,:] = sum_j softmax_j( scale * Q[b,h,i,:] . K[b,g,j,:] + M[b,h,i,j] ) V[b,g,j,:]
 *
 * where M is 0 where element (i, j) is visible and -inf elsewhere.  (i, j) is
 * visible iff its 64x64 block (i/64, j/64) is live in ``block_mask`` and, when
 * ``causal`` is nonzero, j <= i + (S_k - S_q) (bottom-right aligned causal
 * structure; plain lower-triangular when S_q == S_k).  A query row with no
 * visible key has output 0.
 *
 * The pass is fused (Section II-A; Algorithm 1): scores, the running row
 * maximum and row sum, and the rescaled accumulation of P.V stay on chip; only
 * Q, K, V, the mask and O touch device memory.  Key blocks that are dead
 * (mask byte 0, or entirely above the causal diagonal) are never loaded;
 * partially masked blocks get the element mask from their coordinates;
 * unmasked blocks run without it (the three tile cases of Section IV-A).
 *
 * All calls are asynchronous on the given HIP stream (a hipStream_t passed as
 * ``void*``; NULL means the default stream) and return once the work is
 * enqueued.  Argument checks run before any HIP call; on a non-OK status
 * nothing has been enqueued and no output has been written.  Kernel faults
 * surface at the caller's next synchronisation, as usual for HIP.
 *
 * Thread safety: calls may be made concurrently from several threads and on
 * several streams.  The fused calls keep their index in a scratch buffer
 * that belongs to the calling stream (one per device and stream, allocated on
 * the stream's first call, grown when a call needs more, kept until the
 * process ends): calls on one stream reuse it in stream order, and calls on
 * different streams use different buffers, so they never wait for each
 * other.  Two threads enqueueing on the same stream take turns while they
 * enqueue (a short host lock per stream).  Besides these buffers the only
 * process-wide state is the thread-local error text and the fixed array of
 * steel_attn_fwd_noalloc.
 */
#ifndef STEEL_H
#define STEEL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum steel_status {
  STEEL_OK = 0,
  STEEL_ERR_INVALID_ARGUMENT = 1, /* bad pointer, shape, alignment or scale    */
  STEEL_ERR_UNSUPPORTED = 2,      /* valid but not built: D not 64/128, blk != 64 */
  STEEL_ERR_HIP = 3               /* HIP runtime error; see steel_last_error()  */
} steel_status;

/*
 * Fused attention forward (Section II-A Eq. 1; Algorithm 1; Section IV-A).
 *
 *   q          bf16 [B][Hq][S_q][D], device memory, row-major, 16-byte aligned
 *   k, v       bf16 [B][Hkv][S_k][D], device memory, row-major, 16-byte aligned
 *   block_mask uint8 [B][Hq][ceil(S_q/blk)][ceil(S_k/blk)], device memory,
 *              nonzero = live block; NULL = every block live
 *   out        fp32 [B][Hq][S_q][D], device memory, 16-byte aligned; every
 *              element is written
 *   B, Hq, Hkv, S_q, S_k >= 1;  Hq % Hkv == 0
 *   D          head dimension: 64 or 128 (others: STEEL_ERR_UNSUPPORTED)
 *   blk        block edge of the mask: 64 (others: STEEL_ERR_UNSUPPORTED)
 *   scale      multiplies Q.K^T; finite and > 0 (1/sqrt(D) in the paper)
 *   causal     0 or 1
 *   stream     hipStream_t as void*, or NULL
 *
 * Inputs and output are owned by the caller; the library keeps no pointer to
 * them after it returns.  Internal workspace (the compressed live-block list
 * and the work order) lives in the calling stream's scratch buffer, which the
 * library allocates on the stream's first call and grows (hipMalloc,
 * synchronous; the stream's earlier calls are waited for) when a call needs
 * more than it holds; it is kept until the process ends.  Results are
 * bitwise reproducible run to run.
 *
 * Without a mask tensor nothing is indexed and, unless the lists are split,
 * no scratch is used.  The result is bit for bit that of the same mask given
 * as a tensor, but for two kinds of calls without a mask tensor, which take
 * the same sums in another order (differences of the rounding of the softmax
 * weights and, for packs of heads, of the scaled queries to bf16: up to 3e-3 of
 * the output's norm):
 *   split lists   query blocks too few to fill the GPU (decoding, a few
 *                 queries against many keys; only where S_k > 960) run every
 *                 live list in segments and add the partial results in fp32
 *   shared tiles  with one query block (S_q <= 64) and several query heads per
 *                 key/value head, heads of a group whose rows fit 64 rows
 *                 together run as one item
 * steel_attn_fwd_ex (without the fp8 flags), steel_attn_fwd_window and
 * steel_attn_fwd_noalloc treat such calls as this one does, so without a mask
 * tensor these calls agree with each other bit for bit; mask tensors and plans
 * are never split and share no tiles.
 */
int steel_attn_fwd(const void* q, const void* k, const void* v,
                   const uint8_t* block_mask, void* out,
                   int B, int Hq, int Hkv, int S_q, int S_k, int D, int blk,
                   float scale, int causal, void* stream);

/*
 * Live-block index (Section IV-A tile classes, as a compressed list; Section
 * IV-C balance, as a work order).  Rows are r = (b*Hq + h)*nQB + qb with
 * nQB = ceil(S_q/blk), nKB = ceil(S_k/blk).
 *
 *   A block (qb, kb) is dead if its mask byte is 0, or if causal and
 *   kb*blk > min((qb+1)*blk, S_q) - 1 + (S_k - S_q).  A live block is partial
 *   if causal and (kb+1)*blk - 1 > qb*blk + (S_k - S_q), or if
 *   (kb+1)*blk > S_k.
 *
 *   row_ptr  int32 [R+1], device: exclusive prefix sum of the live counts
 *   col      uint32 [capacity], device: for row r, entries
 *            row_ptr[r] .. row_ptr[r+1]-1 hold the live kb in increasing
 *            order, bit 31 set for a partial block.  Capacity must be at
 *            least R*nKB (the live total is only known on the device).
 *   order    int32 [R], device: the rows sorted by the bin of their live
 *            count, heaviest first, equal bins in increasing row order.  The
 *            bin of a count c is c itself when c < 128; above, with
 *            e = floor(log2 c), it is 128 + 16*(e - 7) + ((c >> (e - 4)) & 15)
 *            (16 bins per octave, all bins below 512).
 *
 * The arguments shared with steel_attn_fwd mean the same and are checked the
 * same way; D and the tensors are not needed here.
 */
int steel_block_index(const uint8_t* block_mask, int B, int Hq, int S_q, int S_k,
                      int blk, int causal, int32_t* row_ptr, uint32_t* col,
                      int32_t* order, void* stream);

/*
 * Two-phase form of steel_attn_fwd for callers that reuse one mask over many
 * calls (for example every layer of a model): steel_attn_plan builds the
 * live-block index once into caller-owned device workspace, steel_attn_run
 * runs the fused pass over it.  plan + run computes what steel_attn_fwd
 * computes for the mask as a tensor, bit for bit; without one, bit for bit but
 * for split lists and shared tiles (see there).
 *
 *   steel_attn_workspace_bytes  size of the workspace for these sizes, or 0
 *                               after an argument error (see
 *                               steel_last_error())
 *   workspace                   device memory, 256-byte aligned, at least
 *                               that many bytes, owned by the caller; run
 *                               only reads it, so several runs may share one
 *                               plan concurrently
 *
 * run must be given the same B, Hq, Hkv, S_q, S_k, blk and causal as the plan:
 * the plan writes a header with every one of them (and the head packing and
 * causal limit derived from them) into the workspace, the attention kernels
 * compare it with their own arguments, and on any mismatch they return
 * without writing out (the call itself still returns STEEL_OK: the header is
 * only readable on the device).  run must be ordered after the plan on the
 * device (same stream, or an event).  Arguments mean what they mean for
 * steel_attn_fwd.
 */
size_t steel_attn_workspace_bytes(int B, int Hq, int Hkv, int S_q, int S_k, int blk);

int steel_attn_plan(const uint8_t* block_mask, int B, int Hq, int Hkv, int S_q, int S_k,
                    int blk, int causal, void* workspace, size_t workspace_bytes, void* stream);

int steel_attn_run(const void* q, const void* k, const void* v, void* out,
                   int B, int Hq, int Hkv, int S_q, int S_k, int D, int blk,
                   float scale, int causal, const void* workspace, size_t workspace_bytes,
                   void* stream);

/*
 * steel_attn_fwd with two additions for work split over key chunks
 * (chunked prefill, keys held on several devices):
 *
 *   lse            float [B][Hq][S_q] device buffer, or NULL: receives each
 *                  query row's log sum_j exp(scale * q_i . k_j) over its
 *                  visible keys (natural log; -inf when no key is visible).
 *                  It is the row statistic Algorithm 1 carries (running
 *                  maximum m and sum l: lse = m + log l).
 *   causal_offset  when causal, key j is visible to query i iff
 *                  j <= i + causal_offset (steel_attn_fwd uses S_k - S_q);
 *                  a chunk [k0, k1) of a sequence of S_k_total keys is passed
 *                  as its own K, V with causal_offset = S_k_total - S_q - k0.
 *                  Ignored when causal == 0; otherwise within [-2^30, 2^30].
 *   flags          0 or an OR of:
 *     STEEL_OUT_BF16  out is bf16, each value the round-to-nearest-even of
 *                     the fp32 result (half the output bytes); without it
 *                     out is fp32 [B][Hq][S_q][D] as for steel_attn_fwd.
 *     STEEL_FP8_PV    the fp8 form for P V only: the scores come from bf16
 *                     Q and K as without flags; V and the softmax weights
 *                     are rounded to E4M3 as described under STEEL_FP8.
 *     STEEL_FP8       the fp8 form: both products of Algorithm 1 take E4M3
 *                     operands (OCP 8-bit float: 4 exponent bits, 3 mantissa
 *                     bits, largest value 448) instead of the bf16 operands
 *                     of the paper's datapath (Section II-C), accumulating in
 *                     fp32 as before.  Q is rounded per query row after a
 *                     power-of-two scale that maps the row's largest |value|
 *                     into (224, 448]; K and V likewise with one scale each
 *                     per (batch, key/value head), found by a pre-pass over
 *                     K and V; the softmax weights 2^(s - m + 8) (m the exact
 *                     running row maximum, so the weights lie in (0, 256])
 *                     are rounded for P V, while the row sum adds them
 *                     unrounded.  Scales are divided out exactly.  The
 *                     result follows the same recurrence with larger
 *                     rounding: its error against exact attention is the
 *                     form's own budget, measured per workload in the
 *                     library's design notes, not the bf16 tolerance.  The
 *                     E4M3 copies of K and V (B*Hkv*ceil(S_k/64)*64*D bytes
 *                     each) live in the calling stream's scratch buffer.
 *                     Scores of large magnitude (sharply peaked attention)
 *                     lose the most: their absolute error grows with |s|,
 *                     and STEEL_FP8_PV keeps them at bf16 precision.
 *                     STEEL_FP8 together with STEEL_FP8_PV is STEEL_FP8.
 *
 * Other flag bits: STEEL_ERR_INVALID_ARGUMENT.  Everything else as
 * steel_attn_fwd; with lse == NULL, causal_offset = S_k - S_q and flags == 0
 * the output is bitwise that of steel_attn_fwd.
 */
#define STEEL_OUT_BF16 1
#define STEEL_FP8 2
#define STEEL_FP8_PV 4
int steel_attn_fwd_ex(const void* q, const void* k, const void* v,
                      const uint8_t* block_mask, void* out, float* lse,
                      int B, int Hq, int Hkv, int S_q, int S_k, int D, int blk,
                      float scale, int causal, int causal_offset, int flags,
                      void* stream);

/*
 * Merge of partial results over disjoint key sets: with n_parts outputs O_c
 * and row log-sum-exps lse_c (from steel_attn_fwd_ex over each key chunk),
 *   out = sum_c exp(lse_c - L) O_c / sum_c exp(lse_c - L),   L = max_c lse_c
 *   lse_out = L + log sum_c exp(lse_c - L)
 * per row; rows with every lse_c = -inf get out = 0 and lse_out = -inf.
 *
 *   o_parts    float [n_parts][rows][D] device, 16-byte aligned
 *   lse_parts  float [n_parts][rows] device
 *   rows       rows per part (B*Hq*S_q for attention outputs), >= 1
 *   D          positive multiple of 4
 *   out        float [rows][D] device, 16-byte aligned (may not alias a part)
 *   lse_out    float [rows] device, or NULL
 *
 * Invalid arguments: STEEL_ERR_INVALID_ARGUMENT before any HIP call.  The
 * call only enqueues; it allocates nothing.
 */
int steel_attn_merge(const float* o_parts, const float* lse_parts, int n_parts, long long rows,
                     int D, float* out, float* lse_out, void* stream);

/*
 * Structured-mask forms: the block mask is generated from block coordinates
 * instead of read from a tensor (the paper builds masks on the core rather
 * than fetching them, Section III-B, and names windowed attention among the
 * masking schemes its coordinate tracking covers, Section IV-A).  Block
 * (qb, kb) is in the mask iff
 *     qb - window_blocks < kb <= qb      (window ending at the block diagonal)
 *  or kb < sink_blocks                   (sink blocks at the start)
 * and the causal structure is then applied exactly as for a mask tensor.  The
 * result is that of steel_attn_fwd / steel_attn_plan given that mask as a
 * [B][Hq][nQB][nKB] tensor, bit for bit but for split lists and shared tiles
 * (see steel_attn_fwd); no mask is read.  Every query head shares the pattern,
 * so head packs always run together.
 *
 *   window_blocks  >= 1 (STEEL_ERR_INVALID_ARGUMENT otherwise)
 *   sink_blocks    >= 0
 *
 * All other arguments, the workspace (same size as for steel_attn_plan),
 * ownership and error behaviour are those of steel_attn_fwd and
 * steel_attn_plan; a window plan is run with steel_attn_run.
 */
int steel_attn_fwd_window(const void* q, const void* k, const void* v, void* out,
                          int B, int Hq, int Hkv, int S_q, int S_k, int D, int blk,
                          float scale, int causal, int window_blocks, int sink_blocks,
                          void* stream);

int steel_attn_plan_window(int B, int Hq, int Hkv, int S_q, int S_k, int blk, int causal,
                           int window_blocks, int sink_blocks, void* workspace,
                           size_t workspace_bytes, void* stream);

/*
 * Block-mask producer run ahead of the pass: top-k key blocks per query block
 * by mean-pooled score, plus the diagonal block.  (The paper generates masks
 * on the compute core rather than fetching them, Section III-B, and any block
 * mask then goes through the tile classes of Section IV-A.)  For every
 * (b, query head h, query block qb), with g = h / (Hq/Hkv):
 *   mean_q(qb)  float64 mean of the block's rows of Q[b][h] (a ragged last
 *               block averages the rows it has); mean_k(kb) likewise of
 *               K[b][g]
 *   score(kb)   dot(mean_q(qb), mean_k(kb)) in float64
 *   candidates  kb < min(qb + 1, nKB) when causal, kb < nKB otherwise
 *   kept        the ceil(keep_num / keep_den * #candidates) candidates with
 *               the largest scores (equal scores: the smaller kb first), and
 *               kb = qb when qb < nKB
 * block_mask[b][h][qb][kb] = 1 for kept blocks and 0 for all others (every
 * byte of the [B][Hq][nQB][nKB] mask is written).  The float64 operation
 * order is fixed (rows summed in increasing order, mean = sum / row count,
 * products summed in increasing d without fused multiply-add), so the mask is
 * reproducible bit for bit.
 *
 *   q, k        bf16 device tensors laid out as for steel_attn_fwd
 *   D           64 or 128; blk 64; nKB <= 4096 (STEEL_ERR_UNSUPPORTED)
 *   keep_num, keep_den   1 <= keep_num <= keep_den (1 and 10: 10%)
 *   block_mask  uint8 device buffer of B*Hq*nQB*nKB bytes, caller-owned
 *
 * Float64 workspace for the block means and scores lives in the calling
 * stream's scratch buffer (as for steel_attn_fwd); the call only enqueues,
 * unless the buffer must grow.  Errors as for steel_attn_fwd.
 */
int steel_topk_block_mask(const void* q, const void* k, int B, int Hq, int Hkv, int S_q,
                          int S_k, int D, int blk, int causal, int keep_num, int keep_den,
                          uint8_t* block_mask, void* stream);

/*
 * steel_attn_fwd for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc):
 * the same computation, arguments, checks and kernels, bitwise the same
 * output, but the live-block index is built in a fixed array of
 * STEEL_NOALLOC_SCRATCH_BYTES that the library holds on each device it runs on
 * (a file-scope device array, present from the library's load until the
 * process ends).  The call allocates nothing: no hipMalloc, hipFree or
 * allocating library routine.  The first call on a device looks up that
 * device's copy of the array (hipGetSymbolAddress); later calls only enqueue.
 *
 *   Limit: the index of the problem must fit the array.  It needs about
 *   4 * R * (nKB + 4) bytes plus 2 KiB per 256 rows (R = B*Hq*ceil(S_q/64),
 *   nKB = ceil(S_k/64)): 24.3 MiB for 24 heads at S = 32768, 8.2 MiB for
 *   32 heads at S = 16384 (steel_attn_workspace_bytes gives the exact
 *   figure).  A larger problem returns STEEL_ERR_UNSUPPORTED before any HIP
 *   call (use steel_attn_fwd or plan/run).
 *
 *   Every call on one device shares that device's array, which keeps the last
 *   call's index: calls that overlap on one device (concurrent streams, or
 *   threads enqueueing on different streams) race on it and must be ordered
 *   by the caller; calls queued on one stream are ordered by the stream.
 *   Nothing in the array needs to start at zero (each call writes all it
 *   reads).
 */
#define STEEL_NOALLOC_SCRATCH_BYTES ((size_t)32 << 20)

int steel_attn_fwd_noalloc(const void* q, const void* k, const void* v,
                           const uint8_t* block_mask, void* out,
                           int B, int Hq, int Hkv, int S_q, int S_k, int D, int blk,
                           float scale, int causal, void* stream);

/*
 * Paged 4-bit key/value cache: keys and values of many sequences in a pool of
 * pages, attention that reads it, and the bookkeeping of its pages.
 *
 * Pool.  A page holds 64 tokens of every key/value head (the block edge of the
 * masks above: a page is one key tile).  ``pages`` is uint8 [n_pages][Hkv][68 D],
 * 16-byte aligned; the 68 D bytes of a page and a head are, in this order,
 *   key codes [64][D/2]     token t, channels 2c (low nibble) and 2c + 1
 *   value codes [64][D/2]
 *   key scales [64][D/32], value scales [64][D/32]
 * A code is an E2M1 number: bits 0-2 select 0 0.5 1 1.5 2 3 4 6, bit 3 is the
 * sign.  A scale byte b stands for 2^(b - 127) and covers 32 channels of one
 * token.  A stored vector x has, per 32 channels, the smallest scale 2^e with
 * max |x| <= 6 * 2^e, e in [-125, 125], and codes x / 2^e rounded to nearest
 * (ties to the even code, magnitudes above 6 to 6).  A vector with a NaN or an
 * infinity has code 0 and scale bytes 255 throughout: all its values stand for
 * NaN.  D is 64 or 128 (others: STEEL_ERR_UNSUPPORTED).
 *
 * Sequences.  page_table int32 [B][max_pages]: entry j of row b is the page of
 * tokens 64 j .. 64 j + 63 of sequence b.  lens int32 [B]: the tokens that each
 * sequence has.  Only entries j < ceil(lens[b] / 64) of a row are held; the
 * others (-1 where the calls below write them) are not read as pages.  Tables, lengths, reference
 * counts and page numbers are device memory and are read by the kernels: a
 * page number outside [0, n_pages) is a page that does not exist (nothing is
 * written to it, no key of it is visible), a length outside [0, 64 max_pages]
 * counts as the nearer end of it where keys are read or pages held.  A caller that writes a
 * smaller length (drafted tokens that were rejected) lowers the counts of the entries behind
 * the new end itself: the calls below count what a row holds when they run.
 *
 * n_new int32 [B], device, or NULL: how many of the S tokens (or S_q queries)
 * of a padded batch sequence b has, at the front of its S (clamped to [0, S];
 * NULL: all S).  lens counts them already: token or query i < n_new[b] stands at
 * position lens[b] - n_new[b] + i.
 *
 * None of these calls allocates or waits for the host; all may be captured into a
 * HIP graph.  Workspaces are the caller's: device memory, 256-byte aligned,
 * contents arbitrary, in use until the call's work is done (two captured graphs
 * that may run at one time need one each).
 */

/*
 * Writes new keys and values into the cache.
 *
 *   k, v     bf16 [B][Hkv][S][D]: element (b, h, i, d) at b * sb + h * sh + i * ss
 *            + d (strides in elements, multiples of 8, >= 0), 16-byte aligned
 *   pages    see above; the tokens' slots are overwritten, all else is kept
 *
 * A token whose position is negative, whose entry lies past the table or whose page does
 * not exist is dropped.  Two rows of one call that write the same slot (a shared
 * page written without steel_pages_grow and steel_pages_copy) leave either's
 * bytes in it.  lens has to count the new tokens: after a growth that did not fit it does
 * not, and the positions would be those of tokens that are there; pass n_new then
 * as steel_pages_grow_ex's took (0: nothing is written).
 */
int steel_cache_append(const void* k, const void* v, long long k_sb, long long k_sh,
                       long long k_ss, long long v_sb, long long v_sh, long long v_ss,
                       uint8_t* pages, const int32_t* page_table, const int32_t* lens,
                       const int32_t* n_new, int B, int Hkv, int S, int D, int max_pages,
                       int n_pages, void* stream);

/*
 * Reads keys and values back as bf16 (exact: every value of the cache is a bf16
 * number), for example to hand a cached prefix to steel_attn_fwd.
 *
 *   start    int32 [B], device, or NULL (0): first token of each sequence
 *   k, v     bf16 [B][Hkv][S][D], 16-byte aligned: token start[b] + i at row i; rows
 *            of tokens that do not exist are 0
 */
int steel_cache_load(const uint8_t* pages, const int32_t* page_table, const int32_t* lens,
                     const int32_t* start, void* k, void* v, int B, int Hkv, int S, int D,
                     int max_pages, int n_pages, void* stream);

/*
 * steel_attn_fwd_ex for queries against the cache: single tokens, drafted
 * tokens, chunks of prompts.
 *
 *   q        bf16 [B][Hq][S_q][D] by strides as for steel_cache_append
 *   out      [B][Hq][S_q][D], 16-byte aligned, fp32, or bf16 with
 *            STEEL_OUT_BF16 (the only flag); every element is written
 *   lse      float [B][Hq][S_q] or NULL: row log-sum-exp (natural log)
 *   block_mask   uint8 [B][Hkv][max_pages], device, or NULL: pages with byte 0 are
 *            not visible to the query heads of that key/value head
 *   window_blocks, sink_blocks   window_blocks > 0: the structured mask of
 *            steel_attn_fwd_window over blocks of 64 positions; 0: none
 *   causal   0 or 1
 *
 * With p the position of query i (see n_new), key j of sequence b is visible iff
 * 0 <= j < lens[b], p >= 0, (j <= p or not causal), its page exists and is live,
 * and with a window p/64 - window_blocks < j/64 <= p/64 or j/64 < sink_blocks.
 * Queries without a visible key, and queries i >= n_new[b], get out 0 and lse
 * -inf.  A token whose keys or values stand for NaN makes the rows that see it
 * NaN, and no others, and so does a query with a NaN or an infinity.
 *
 * Precision: queries, keys and values are exact and the sums fp32; the softmax weights are
 * rounded to bf16 where they meet V, so out is off by up to 2^-8 of sum_j p_j |v_j|, and by
 * the rounding of a bf16 output.  lse has no such rounding.  Values whose magnitude is below
 * 2^-100 may be lost, a key counts for up to 2^-126 of its value however small its weight is,
 * and the scores, as q . k and scaled, and the sum of weights times values, n times the mean
 * at most, have to be fp32 numbers.
 * Results are bitwise reproducible run to run.  Which bits a row gets inside these bounds may
 * depend on the other rows of its call and on what its pages hold beyond its own keys (a
 * key that only a later query sees): rows share the steps of their running maxima.
 *
 *   workspace   at least steel_attn_cache_workspace_bytes of the same sizes (0 after an
 *               argument error); where that is 256 none is used and it may be NULL.
 *               Without a block_mask steel_attn_cache_workspace_bytes_ex with masked = 0
 *               will do: 8 B Hkv max_pages bytes less, the room for lists of live pages
 */
size_t steel_attn_cache_workspace_bytes(int B, int Hq, int Hkv, int S_q, int D, int max_pages);
size_t steel_attn_cache_workspace_bytes_ex(int B, int Hq, int Hkv, int S_q, int D, int max_pages,
                                           int masked);

int steel_attn_cache(const void* q, long long q_sb, long long q_sh, long long q_ss,
                     const uint8_t* pages, const int32_t* page_table, const int32_t* lens,
                     const int32_t* n_new, const uint8_t* block_mask, void* out, float* lse, int B,
                     int Hq, int Hkv, int S_q, int D, int max_pages, int n_pages, float scale,
                     int causal, int window_blocks, int sink_blocks, int flags, void* workspace,
                     size_t workspace_bytes, void* stream);

/*
 * New rows of the page table from old ones: beams reordered, sequences forked
 * (two rows with one parent share its pages) and freed (parent -1).
 *
 *   refs       int32 [n_pages]: rows that hold each page; 0 = free.  Updated: plus
 *              one for every page that a new row holds, minus one for every
 *              page that an old row held
 *   parent     int32 [B_out]: the old row that new row b continues; anything outside
 *              [0, B_in): an empty row
 *   table_out, lens_out   the new rows [B_out][max_pages] and lengths; entries that a
 *              row does not hold are -1.  They may not alias page_table and lens
 */
int steel_pages_fork(const int32_t* page_table, const int32_t* lens, int32_t* refs,
                     const int32_t* parent, int32_t* table_out, int32_t* lens_out, int B_in,
                     int B_out, int max_pages, int n_pages, void* stream);

/*
 * Room for n_new[b] more tokens of every sequence (negative: 0): lens grows, and
 * rows take free pages, in increasing order of page number, row after row.  A row
 * that writes into a last page which other rows hold too takes a page of its own in
 * its place first and lets go of the shared one; of several such rows in one call
 * the last keeps the page if no other row holds it then.  The bytes are not copied here:
 * src[b] and dst[b] (int32 [B]) are the pages to copy for row b, or -1, for
 * steel_pages_copy.
 *   left       int32 [1]: free pages that remain.  Negative: that many were missing,
 *              or INT32_MIN: a row would need more than max_pages entries; then
 *              nothing has changed and every src and dst is -1
 *   took       (steel_pages_grow_ex) int32 [B], or NULL: the tokens that there is room for,
 *              max(n_new[b], 0), or 0 in every row where nothing has changed.  As n_new of
 *              the calls that write and read the new tokens it makes a step that does
 *              not fit one that does nothing, without a look at left from the host (as
 *              in a graph).  It may not alias n_new
 *   workspace  at least steel_pages_workspace_bytes, or NULL where
 *              steel_pages_grow_workspace_bytes is 256: none is used
 * n_pages up to 2^22.
 */
size_t steel_pages_workspace_bytes(int n_pages, int B);
size_t steel_pages_grow_workspace_bytes(int n_pages, int B);

int steel_pages_grow(int32_t* page_table, int32_t* lens, int32_t* refs, const int32_t* n_new,
                     int32_t* src, int32_t* dst, int32_t* left, int B, int max_pages, int n_pages,
                     void* workspace, size_t workspace_bytes, void* stream);

int steel_pages_grow_ex(int32_t* page_table, int32_t* lens, int32_t* refs, const int32_t* n_new,
                        int32_t* src, int32_t* dst, int32_t* left, int32_t* took, int B,
                        int max_pages, int n_pages, void* workspace, size_t workspace_bytes,
                        void* stream);

/*
 * Copies page src[i] onto page dst[i] for i < n, in each of ``layers`` pools
 * (layer l begins at pages + l * n_pages * page_bytes; page_bytes, a multiple of 16, is
 * Hkv * 68 * D for a cache).  Pairs with a page number outside [0, n_pages) are
 * skipped.  The destinations are distinct and no source: a page that is written
 * twice, or read and written, has unspecified bytes afterwards.
 */
int steel_pages_copy(uint8_t* pages, const int32_t* src, const int32_t* dst, int n, int layers,
                     int n_pages, size_t page_bytes, void* stream);

/*
 * Moves the live pages (refs > 0) to the front of the pool, in each of ``layers``
 * pools: with n of them, those numbered n or more move, in order, to the free
 * pages below n, in order.  page_table (the held entries) and refs follow.
 * Live pages that no row of this table holds (a kept prefix, another table) move too.
 *   live       int32 [1]: n
 *   to         (steel_pages_compact_ex) int32 [n_pages], or NULL: the number that each live
 *              page has now, by the one it had, and -1 for free ones: what other holders
 *              look theirs up in.  It may not alias refs
 *   workspace  at least steel_pages_workspace_bytes
 */
int steel_pages_compact(uint8_t* pages, int32_t* page_table, const int32_t* lens, int32_t* refs,
                        int32_t* live, int B, int max_pages, int layers, int n_pages,
                        size_t page_bytes, void* workspace, size_t workspace_bytes, void* stream);

int steel_pages_compact_ex(uint8_t* pages, int32_t* page_table, const int32_t* lens, int32_t* refs,
                           int32_t* live, int32_t* to, int B, int max_pages, int layers,
                           int n_pages, size_t page_bytes, void* workspace, size_t workspace_bytes,
                           void* stream);

/* Text of the last non-OK status returned on the calling thread ("" if none). */
const char* steel_last_error(void);

/* Library version string. */
const char* steel_version(void);

#ifdef __cplusplus
}
#endif

#endif /* STEEL_H */
