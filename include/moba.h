/*
 * moba.h -- C ABI of the MI355X (gfx950) MoBA causal prefill library.
 *
 * MoBA (Mixture of Block Attention, arXiv 2502.13189) lets every query attend
 * to its own block plus the top-scoring past blocks of its sequence.  The
 * library computes, on one GPU:
 *   block mean-pool of the keys  -> gate (unscaled q . block key, causal mask,
 *   forced current block, top-k)  -> routing inversion (queries per block)
 *   -> attention over the routed history blocks and the causal current block
 *   -> log-sum-exp merge of the partial results,
 * following Sec. 2.2 (Eq. 2-6) and Algorithm 1 of the paper; plus dense causal
 * attention (Eq. 1) built from the same kernels, for comparison.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Tensors are passed as moba_tensor descriptors: a data pointer, a dtype, and
 * shape/stride in ELEMENTS.  The caller owns every tensor; the library never
 * frees caller memory.  All tensors except cu_seqlens live in device memory of
 * the current HIP device.
 *
 *   q    [T, Hq,  D]  bf16 or f32; last dim contiguous, any token/head stride
 *   k, v [T, Hkv, D]  same dtype as q; last dim contiguous
 *   out  [T, Hq,  D]  same dtype as q; last dim contiguous; may be q's own memory
 *                      (with q's strides)
 *   lse  [Hq, T]      f32, contiguous; natural-log log-sum-exp of the scaled
 *                      logits over the keys each query attended
 *   cu_seqlens [S+1]  int32, contiguous, host OR device memory: cu[0] = 0,
 *                      non-decreasing, cu[S] = T.  Sequence s holds tokens
 *                      [cu[s], cu[s+1]); blocks restart at every sequence and
 *                      nothing is attended across sequences.  A device
 *                      cu_seqlens is copied to the host on `stream` (after
 *                      the work enqueued there before the call) and the
 *                      stream is waited for; pass it in host memory to keep
 *                      the call asynchronous.
 *
 * Head dimension D must be 128.  Hq must be a multiple of Hkv (GQA: query head
 * h uses kv-head h / (Hq / Hkv)) and Hq / Hkv <= 128.  Logits are scaled by
 * 1/sqrt(D); gate scores are not scaled (Eq. 6).
 *
 * Every call enqueues its device work on `stream` and returns without waiting,
 * except as noted.  Arguments are validated before any HIP call; invalid
 * arguments return a status code and touch nothing.  Kernel launch failures
 * return MOBA_ERR_HIP.  No function throws.
 *
 * Per-shape tables (sequence offsets, tile lists) are built on the host for
 * each new (cu_seqlens, heads, block size, top-k) and copied on `stream`; the
 * last few are kept per device.  Their buffers grow in powers of two, and
 * growing one synchronizes the device.
 *
 * The library keeps one cached device workspace per device, grown on demand
 * (growing it synchronizes the device) and capped by the environment variable
 * MOBA_WORKSPACE_LIMIT_BYTES (default 64 GiB).  When one call needs more, the
 * attention runs in chunks of kv-heads.  The workspace is shared by all calls
 * on a device: calls on one device must come from one host thread, and calls
 * enqueued on different streams of one device must not overlap in time.
 */
#ifndef MOBA_H_
#define MOBA_H_

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* MOBA_F8E4M3: 8-bit floats, 4 exponent and 3 mantissa bits, largest 448, no infinities
 * (only in the paged cache) */
typedef enum { MOBA_F32 = 0, MOBA_BF16 = 1, MOBA_I32 = 2, MOBA_I64 = 3, MOBA_F8E4M3 = 4 } moba_dtype;

typedef struct {
  void* data;        /* host or device pointer, see each argument */
  int32_t dtype;     /* moba_dtype */
  int32_t ndim;      /* 1..4 */
  int64_t shape[4];  /* elements per dimension */
  int64_t stride[4]; /* elements between consecutive indices of a dimension */
} moba_tensor;

typedef enum {
  MOBA_OK = 0,
  MOBA_ERR_NULL = 1,        /* a required descriptor or data pointer is NULL */
  MOBA_ERR_DTYPE = 2,       /* dtype mismatch or unsupported dtype */
  MOBA_ERR_SHAPE = 3,       /* shapes disagree with each other or with cu_seqlens */
  MOBA_ERR_LAYOUT = 4,      /* last dim not contiguous, or a contiguous tensor required */
  MOBA_ERR_BLOCK_SIZE = 5,  /* block_size < 1, or (paged cache) no multiple of the page size */
  MOBA_ERR_TOPK = 6,        /* topk < 1 */
  MOBA_ERR_SEQLENS = 7,     /* cu[0] != 0, decreasing, or cu[S] != T */
  MOBA_ERR_UNSUPPORTED = 8, /* D != 128, Hq/Hkv > 128, > 4096 blocks per sequence,
                               1 < topk-1 < #blocks with topk > 64, a page size the paged
                               cache does not have, or index overflow */
  MOBA_ERR_NO_MEMORY = 9,   /* workspace over MOBA_WORKSPACE_LIMIT_BYTES, hipMalloc failed, or
                               a workspace passed in is too small */
  MOBA_ERR_HIP = 10         /* a HIP call or kernel launch failed */
} moba_status;

/*
 * MoBA causal prefill forward (Sec. 2.2 Eq. 2-6; Algorithm 1).
 *
 * For query token t of sequence s at local position tau = t - cu[s] and
 * query head h: c = tau / block_size is its current block.  The gate scores
 * every past block j < c with <q, mean of block j's keys> (unscaled, fp32),
 * keeps the min(topk-1, c) highest (equal scores: lower block index wins),
 * and adds block c (the current block counts toward topk).  out[t, h] is
 * softmax attention over every key of the kept past blocks plus the keys of
 * block c up to and including t.  lse[h, t] is its log-sum-exp.
 * topk larger than the number of blocks selects every causal block: when
 * topk is at least the block count of the longest sequence, every row
 * attends its whole causal prefix and the call runs moba_dense_forward's
 * kernels (the same result up to rounding).
 * A row whose gate scores are not all finite has no defined selection, so its
 * results are unspecified; it changes no other row's.
 *
 * Arguments: see the conventions above.  block_size >= 1, topk >= 1.
 * Returns MOBA_OK or an error status; on error nothing has been enqueued
 * unless the status is MOBA_ERR_HIP.
 */
moba_status moba_forward(const moba_tensor* q, const moba_tensor* k, const moba_tensor* v,
                         const moba_tensor* cu_seqlens, int32_t block_size, int32_t topk,
                         moba_tensor* out, moba_tensor* lse, hipStream_t stream);

/*
 * MoBA backward: gradients of moba_forward's output w.r.t. q, k and v.  The
 * gate (Eq. 3 and Eq. 5) is a hard 0/1 choice and passes no gradient, so
 * these are the gradients of softmax attention (Eq. 2) over the key set of
 * Eq. 4 that the forward selected.
 *
 * q, k, v, cu_seqlens, block_size, topk: exactly as passed to moba_forward;
 *   the selection is recomputed from them and equals the forward's.
 * out [T, Hq, D], lse [Hq, T]: moba_forward's results for these inputs.
 * dout [T, Hq, D]: gradient of the loss w.r.t. out.
 * dq [T, Hq, D], dk, dv [T, Hkv, D]: outputs, overwritten; dk and dv of a
 *   kv-head sum over the query heads of its group.
 * bf16 only: f32 inputs return MOBA_ERR_DTYPE.  Layout rules as for
 * moba_forward (last dim contiguous, 16-byte aligned rows, any token/head
 * stride).  Products accumulate in fp32; the softmax weights P and the score
 * gradients dS are rounded to bf16 for the second matrix-core products;
 * Delta = <dout, out> per row uses the bf16 out.  Deterministic: no atomics,
 * fixed summation order.  When topk is at least the block count of the
 * longest sequence, this is moba_dense_backward, as in moba_forward.
 */
moba_status moba_backward(const moba_tensor* q, const moba_tensor* k, const moba_tensor* v,
                          const moba_tensor* cu_seqlens, int32_t block_size, int32_t topk,
                          const moba_tensor* out, const moba_tensor* lse, const moba_tensor* dout,
                          moba_tensor* dq, moba_tensor* dk, moba_tensor* dv, hipStream_t stream);

/*
 * Dense causal attention (Eq. 1 with a causal mask and scale 1/sqrt(D)):
 * every query attends to every key of its sequence up to and including
 * itself.  Same tensor conventions as moba_forward.
 */
moba_status moba_dense_forward(const moba_tensor* q, const moba_tensor* k, const moba_tensor* v,
                               const moba_tensor* cu_seqlens, moba_tensor* out, moba_tensor* lse,
                               hipStream_t stream);

/*
 * Backward of moba_dense_forward: gradients of causal full attention (Eq. 1)
 * w.r.t. q, k and v, with out and lse from moba_dense_forward.  Same
 * conventions, dtype (bf16 only) and precision as moba_backward.  With
 * moba_dense_forward it lets a caller switch any attention call between
 * full attention and MoBA, in both directions (the per-layer choice of
 * Sec. 2.2 "Hybrid of MoBA and Full Attention" and the layer-wise hybrid of
 * Sec. 3.2, whose last layers stay full attention).
 */
moba_status moba_dense_backward(const moba_tensor* q, const moba_tensor* k, const moba_tensor* v,
                                const moba_tensor* cu_seqlens, const moba_tensor* out,
                                const moba_tensor* lse, const moba_tensor* dout, moba_tensor* dq,
                                moba_tensor* dk, moba_tensor* dv, hipStream_t stream);

/*
 * Decode: one new query per sequence against its key/value cache.
 *
 * q [S, Hq, D] bf16: the new token of each sequence.  k_cache, v_cache
 * [T, Hkv, D] bf16 hold every sequence's cached keys and values, packed as
 * described by cu_seqlens [S+1] (int32, host or device; every sequence
 * non-empty), and already include each new token's key and value as its
 * sequence's last entry.  So query s sits at position L_s - 1 of sequence s
 * and its result is the last row of the prefill over the cache:
 *   topk >= 1: MoBA with block_size and topk (the gate of Eq. 5 / Eq. 6 over
 *              the sequence's complete past blocks, top-k with the current
 *              block counted, attention over the selected blocks and the
 *              current block up to the query); a topk of at least the
 *              longest sequence's block count selects everything and runs
 *              as topk == 0;
 *   topk == 0: causal full attention over the whole cache (Eq. 1), which is
 *              what the paper uses for generation (Sec. 3.3); block_size is
 *              then ignored.
 * kbar (nullable, MoBA only): the cache's block means as written by
 * moba_pool for the same cu_seqlens and block_size; when NULL they are
 * computed on the fly, which reads the whole key cache.  A decode loop keeps
 * kbar and recomputes it only when a block completes.
 * out [S, Hq, D] bf16 and lse [Hq, S] f32 (natural log) as for moba_forward.
 * Hq / Hkv must not exceed 16.  Gate scores are fp32 sums in a fixed order
 * (four sequential 32-dim partial sums, added in order); near-ties may be
 * broken differently from moba_select's matrix-core gate.  A call whose cu_seqlens differs from those of recent calls (every
 * step of a growing cache) builds new per-shape tables on the host and copies
 * them on `stream`; it does not synchronize the device.
 */
moba_status moba_decode(const moba_tensor* q, const moba_tensor* k_cache,
                        const moba_tensor* v_cache, const moba_tensor* cu_seqlens,
                        const moba_tensor* kbar, int32_t block_size, int32_t topk, moba_tensor* out,
                        moba_tensor* lse, hipStream_t stream);

/*
 * moba_decode without any allocation, for callers that cannot allocate
 * device memory: code under HIP graph capture, tight serving loops, and
 * harnesses that forbid hipMalloc.  Same arguments, conventions and results
 * as moba_decode (the same kernels; the outputs are bit-identical), except:
 *   - cu_seqlens must be in host memory (a device pointer returns
 *     MOBA_ERR_UNSUPPORTED);
 *   - every intermediate buffer (the per-sequence table, block means when
 *     kbar is NULL, selections, block lists, partial results) lives in one
 *     static device array of MOBA_DECODE_NOALLOC_MAX_BYTES bytes, which each
 *     GPU the library runs on holds from module load until the process ends;
 *     a call needing more returns MOBA_ERR_NO_MEMORY before enqueueing
 *     anything (full attention needs about S * Hq * ceil(L_max / 256) * 516
 *     bytes: a 1M-token cache with 32 query heads fits for one sequence);
 *   - no library call allocates memory, device or pinned, and no profiling
 *     events are recorded.
 * All calls on one GPU share that array and the last call's contents stay
 * in it: calls whose execution overlaps on one GPU (different streams, or
 * host threads) race and give wrong results.  Calls on one stream are
 * ordered and safe.
 */
#define MOBA_DECODE_NOALLOC_MAX_BYTES ((size_t)96 << 20)
moba_status moba_decode_noalloc(const moba_tensor* q, const moba_tensor* k_cache,
                                const moba_tensor* v_cache, const moba_tensor* cu_seqlens,
                                const moba_tensor* kbar, int32_t block_size, int32_t topk,
                                moba_tensor* out, moba_tensor* lse, hipStream_t stream);

/*
 * Block mean-pool of the keys (Eq. 6; Algorithm 1, mean_pool).
 * kbar [nblk_total, Hkv, D] f32 contiguous, device: row b = blk_off[s] + j
 * holds the mean of k over the tokens of block j of sequence s (a short last
 * block uses its own token count), with blk_off[s] = sum over s' < s of
 * ceil(len_s' / block_size).  Accumulated in fp64, rounded once to f32.
 */
moba_status moba_pool(const moba_tensor* k, const moba_tensor* cu_seqlens, int32_t block_size,
                      moba_tensor* kbar, hipStream_t stream);

/*
 * Gate and top-k selection (Eq. 5 and Eq. 6 with the causal rules of
 * Sec. 2.2), including the pool.
 * sel [T, Hq, topk] int32 contiguous, device: the kept past blocks in
 * ascending order, then the current block c, then -1 padding; local block
 * indices of the query's sequence.
 * scores (nullable) [T, Hq, nmax] f32 contiguous, device: the fp32 gate score
 * of every past block j < min(c, nmax), NaN elsewhere (a debugging aid; costs
 * one extra write pass).
 */
moba_status moba_select(const moba_tensor* q, const moba_tensor* k, const moba_tensor* cu_seqlens,
                        int32_t block_size, int32_t topk, moba_tensor* sel, moba_tensor* scores,
                        hipStream_t stream);

/*
 * Routing inversion (Algorithm 1, index_select_moba_attn_block; Sec. 2.3
 * "arrange the ordering of query tokens based on their assigned KV blocks"):
 * for every bin (kv-head g, global block b = blk_off[s] + j) the list of
 * history selections that chose it, by a stable counting sort.
 *   sel      [T, Hq, topk] int32 contiguous, device (as written by moba_select)
 *   counts   [Hkv * nblk_total] int32 contiguous, device: entries per bin,
 *            bins ordered g-major
 *   offsets  [Hkv * nblk_total + 1] int64 contiguous, device: exclusive scan
 *   entries  [E] int32 contiguous, device, E = offsets[last]: entry value
 *            e = r * (topk - 1) + x, where x is the selection slot (position
 *            in sel) and r = g * (T * G) + t * G + (h - g * G) with G = Hq/Hkv;
 *            ascending within a bin.  E must equal the number of history
 *            selections, sum over rows of min(topk - 1, c) (moba_route_size
 *            reports it).
 * num_kv_heads gives Hkv.  The current block is not routed.  A history slot
 * (x < min(topk - 1, c)) whose value is not a past block (outside [0, c)) is
 * skipped, by the counts and the entries alike, so no access leaves the
 * row's bins; offsets[last] then falls short of E and the rest of entries is
 * left unwritten.  moba_select never writes such a slot.
 */
moba_status moba_route(const moba_tensor* sel, const moba_tensor* cu_seqlens, int32_t block_size,
                       int32_t num_kv_heads, moba_tensor* counts, moba_tensor* offsets,
                       moba_tensor* entries, hipStream_t stream);

/*
 * Paged 8-bit cache
 * -----------------
 * For serving many requests whose lengths change every step.  A pool of N pages holds
 * P tokens each (page_size: 64, 128, 192 or 256); a request's pages stand in its row of
 * a block table.  Lengths, tables and the free list live in device memory and no call
 * reads them back, allocates, or keeps anything between calls, so a step (plan, write, decode)
 * can be captured into a HIP graph and replayed while the requests grow.  Calls that
 * share no memory (workspaces included) may overlap on different streams.  None of the
 * tensors may overlap another one unless its description says so.
 *
 *   k       [N, Hkv, P, 128] f8e4m3; the last two dims contiguous
 *   v       [N, Hkv, 2 P, 64] f8e4m3: value d of token i of the page at
 *           [.., 128 (i / 64) + d, i % 64], i.e. 64-token tiles [128, 64] with the token
 *           index innermost; the last two dims contiguous
 *   k_scale, v_scale [N, Hkv] f32 contiguous: a page's key is k * k_scale, for all P
 *           tokens of a kv-head
 *   k_sum   [N, Hkv, 128] f32 contiguous: the sum of the page's keys as they are held
 * k, v and k_sum must be 16-byte aligned, k and v with page and head strides that are multiples
 * of 16.
 * The pool's contents need no initialisation: what a page holds past a request's length is
 * never used, whatever its bits.
 */
typedef struct {
  const moba_tensor* k;
  const moba_tensor* v;
  const moba_tensor* k_scale;
  const moba_tensor* v_scale;
  const moba_tensor* k_sum;
} moba_cache;

/*
 * Block tables and slot maps of a step, from the requests' lengths.
 *
 * add      [S] i32: the tokens request s gets in this step (0: none); negative: the
 *          request ends
 * lens     [S] i32: tokens it holds; lens_out [S] i32: after the step (may be lens)
 * table    [S, W] i32, rows contiguous, any row stride: its pages in order; entries of new
 *          pages are written, all others stay
 * free_pages [N] i32, num_free [1] i32: the first num_free entries are the free pages;
 *          num_free_out [1] i32: after the step (may be num_free)
 * cu_new   [S + 1] i32, output: exclusive sums of max(add, 0), at most T: request s's new
 *          tokens are rows cu_new[s] .. cu_new[s + 1] - 1 of the step's arrays
 * slots    [T] i64, output: page * page_size + offset of every new token, -1 for those of
 *          refused requests and past the last one (where a page, as the table or the free list
 *          has it, is negative, so are its tokens' slots)
 * refused  [1] i32, output: requests refused
 *
 * The pages of ended requests go back first: they are appended to the free list, request
 * by request, each one's in order, and their lengths become 0.  New pages are then taken
 * from the list's end, request by request.  A request is refused, as a whole, where its
 * pages would not fit its table row or its tokens would end past T; or where it needs pages and the
 * list does not hold those of every request up to it that was not refused for the first
 * reason.  (A request that gets no token counts as refused, too, where those of the requests
 * before it end past T.)  A refused request keeps its length, pages and free list untouched; the
 * caller sees it in lens_out, and in slots.
 * A request is cut back by lowering its length between two steps.  The pages it is taken to hold
 * are the first ceil(lens[s] / page_size) of its row, so the caller who lowers it past a page's
 * begin also appends the pages behind the new end to the free list (and raises num_free):
 * nothing else gives them back.
 * All tensors are contiguous but for the table's row stride.  S <= 4096, S * W and N below
 * 2^31.  Lengths below 0 or above W * page_size count as 0 and W * page_size, a num_free outside [0, N]
 * as the nearer end; pages returned beyond N are dropped.
 */
moba_status moba_cache_plan(const moba_tensor* add, const moba_tensor* lens, moba_tensor* table,
                            moba_tensor* free_pages, const moba_tensor* num_free,
                            int32_t page_size, moba_tensor* lens_out, moba_tensor* num_free_out,
                            moba_tensor* cu_new, moba_tensor* slots, moba_tensor* refused,
                            hipStream_t stream);

/*
 * Writes new keys and values into their slots, in 8 bits.
 *
 * k, v [T, Hkv, 128] bf16 or f32 (the same), last dim contiguous, rows 16-byte aligned;
 * slots [T] i64 contiguous as moba_cache_plan writes them: a token whose slot is negative or not
 * of the pool is left out.  The tokens of one page must be consecutive rows with ascending slots
 * (a run), and the call may hold one run per page; two runs of a page race for it (its
 * contents are then unspecified, no other page's).
 *
 * A run at offset o of its page, n tokens:
 *   e     = the least integer with max |x| <= 448 * 2^e over its finite values x of the
 *           kv-head (k and v apart), from -100 up, at most 119 (larger values saturate);
 *           where o > 0 not less than the exponent the page's scale has
 *   held  = x * 2^-e rounded to the nearest e4m3 (ties to even); NaN for an x that is
 *           not finite
 *   tokens before o are rescaled, with one more such rounding, where e grew; tokens from
 *   o + n on keep their bits and no longer count
 *   scale = 2^e,  k_sum = the exact sum over tokens 0 .. o + n - 1, rounded once (NaN if
 *           one of the keys is NaN)
 * A power of two costs e4m3 no precision, and rescaling by one none above its subnormals.
 * Writing the same tokens to the same slots again changes nothing; a request that was cut back
 * (see moba_cache_plan) is written on from any offset.
 */
moba_status moba_cache_write(const moba_tensor* k, const moba_tensor* v, const moba_tensor* slots,
                             const moba_cache* cache, hipStream_t stream);

/*
 * moba_decode over the paged cache: one new query per request, at the last position of
 * what the request holds.
 *
 * q [S, Hq, 128] bf16; table [S, W] i32 (rows contiguous, any row stride), lens [S] i32.
 * topk == 0: full attention over the lens[s] tokens; block_size is ignored.
 * topk >= 1: MoBA with blocks of block_size tokens, a multiple of the page size: a past
 *   block's score for a query head is <q, sum of its pages' k_sum> (its mean but for a
 *   common factor), computed in 64 bits, NaN counting as the lowest; the topk - 1 highest (equal
 *   scores: lower block) and the current block are attended.  A topk of at least
 *   ceil(W * page_size / block_size) attends everything and runs as topk == 0.  At most
 *   4096 blocks per table row.  NaN among a block's keys or values reaches no query head that
 *   does not attend it.
 * S * W pages of page_size / 64 tiles, times Hkv, must be below 2^30, S * Hkv below 2^23.
 * out [S, Hq, 128] bf16 (may be q itself, with its strides; another view of q's memory is
 * MOBA_ERR_LAYOUT), lse [Hq, S] f32.
 * A request with lens[s] <= 0 (an empty place of the batch) gets out 0 and lse -inf;
 * lens[s] above W * page_size counts as W * page_size.  The tokens of a table entry outside [0, N)
 * are left out as if masked (their page's k_sum counts as 0).  Hq / Hkv must not exceed 16.
 * workspace: moba_cache_decode_workspace_bytes of device memory, 16-byte aligned; it needs no
 * initialisation and nothing is kept in it after the call.  fp32 softmax and sums; the keys, the
 * queries and the values enter the matrix cores exactly, the weights with all 24 bits (as
 * three bf16 terms).
 * Results do not depend on timing; a request's split over work-groups, and with it its
 * rounding, depends on the whole batch.
 */
moba_status moba_cache_decode(const moba_tensor* q, const moba_cache* cache,
                              const moba_tensor* table, const moba_tensor* lens,
                              int32_t block_size, int32_t topk, moba_tensor* out, moba_tensor* lse,
                              void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Workspace of a moba_cache_decode call for S requests with tables W pages wide.  Returns 0
 * for arguments such a call would refuse, or S == 0.  Host-only arithmetic: no HIP call.
 */
size_t moba_cache_decode_workspace_bytes(int64_t S, int64_t W, int32_t Hq, int32_t Hkv,
                                         int32_t page_size, int32_t block_size, int32_t topk);

/*
 * Workspace sizing query: the device workspace bytes moba_forward needs to
 * run in one pass (no kv-head chunking) for any batch of T tokens in
 * nblk_total blocks (sum over sequences of ceil(len / block_size)), with
 * Hq / Hkv heads, head dimension D and topk, for either input dtype.  It is
 * an upper bound over every cu_seqlens with these totals; moba_dense_forward,
 * moba_select and moba_route need no more.  With MOBA_WORKSPACE_LIMIT_BYTES
 * below it the forward runs in more kv-head chunks instead.  The backward
 * needs more (fp32 dQ partials).  Returns 0 for invalid or empty arguments
 * (T < 0, Hq or Hkv < 1, Hq % Hkv != 0, Hq / Hkv > 128, D != 128,
 * topk < 1; T == 0 or nblk_total == 0).  Host-only arithmetic: no HIP call.
 */
size_t moba_workspace_bytes(int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int64_t nblk_total,
                            int32_t topk);

/* Bytes of device workspace the library currently holds on the current device. */
size_t moba_workspace_held_bytes(void);

/*
 * Sizes of moba_route's outputs for a batch (Algorithm 1,
 * index_select_moba_attn_block):
 *   *nblk_total = sum over sequences of ceil(len / block_size), so counts has
 *                 Hkv * *nblk_total entries and offsets one more;
 *   *entries    = E, the number of history selections: num_q_heads times the
 *                 sum over tokens of min(topk - 1, c), c the token's block
 *                 (Eq. 5 keeps min(topk - 1, c) past blocks besides the
 *                 current one; Sec. 3.1 footnote).
 * cu_seqlens as for moba_forward (host or device; a device copy is read on
 * `stream`, which is then waited for).  Errors: MOBA_ERR_NULL,
 * MOBA_ERR_SEQLENS, MOBA_ERR_BLOCK_SIZE, MOBA_ERR_TOPK, MOBA_ERR_SHAPE
 * (num_q_heads < 1).  No device work besides that copy.
 */
moba_status moba_route_size(const moba_tensor* cu_seqlens, int32_t block_size, int32_t topk,
                            int32_t num_q_heads, int64_t* nblk_total, int64_t* entries,
                            hipStream_t stream);

/*
 * The dK/dV kernel of moba_backward hands each 32-row subtile's softmax
 * weights from one wave to another through a flag, with a bounded wait (so
 * that the kernel always ends).  A wait that gives up leaves that subtile's
 * dK wrong; every give-up is counted on the device.  This call waits for the
 * current device, stores the count since the last call in *count and resets
 * it.  With MOBA_DEBUG_SYNC set (non-zero), moba_backward checks the count
 * itself and returns MOBA_ERR_HIP if it is not zero.  Testing aid: with
 * MOBA_FORCE_WAIT_TIMEOUT set (non-zero) every such wait gives up after a
 * few polls.
 */
moba_status moba_take_wait_timeouts(uint64_t* count);

/* Free the cached workspace, tables and counters of the current device
 * (synchronizes the device). */
moba_status moba_release_workspace(void);

/* Static, human-readable name of a status. */
const char* moba_status_string(moba_status status);

/*
 * Per-phase timing.  While enabled, every entry point records HIP events
 * around each phase on the caller's stream (but not while a graph captures that
 * stream: replays are not timed).  moba_profile_read waits for the
 * recorded events, writes up to max_phases entries and resets the counters;
 * it returns the number of phases written.
 */
typedef struct {
  char name[24];     /* "pool", "gate", "route", "attn_hist", "merge", ... */
  int64_t launches;  /* phase executions recorded */
  double total_ms;   /* summed event-to-event time */
} moba_phase_stat;

void moba_profile_enable(int enabled);
int moba_profile_read(moba_phase_stat* stats, int max_phases);

#ifdef __cplusplus
}
#endif

#endif /* MOBA_H_ */
