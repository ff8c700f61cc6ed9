/*
 * cover.h - C ABI of the COVER override-attention and seed-scoring kernels
 * (single GB300 GPU, sm_103a).
 *
 * COVER ("Stop the Flip-Flop: Context-Preserving Verification for Fast
 * Revocable Diffusion Decoding") verifies previously decoded "seed" positions
 * in the same forward pass that drafts new tokens. Section 5.1: the seeds are
 * masked in the input, their key/value columns are overridden with the states
 * cached at the previous step (memory K', V'), every query attends once over
 * K', V', and each seed query's own diagonal entry is restored to the pair
 * (k_i, v_i) computed from the masked input (leave-one-out view). Appendix B
 * gives the closed form of that diagonal correction.
 *
 * Conventions for every entry point:
 *  - Pointers are DEVICE pointers owned by the caller, unless stated otherwise.
 *    The library allocates no device memory and keeps no per-call state.
 *  - Calls are asynchronous on `stream` (a cudaStream_t; NULL = legacy default
 *    stream). Argument errors are returned synchronously, before any launch.
 *  - Every kernel is launched as a programmatic dependent of the stream's
 *    previous kernel: its CTAs may start while that kernel finishes, but they
 *    read and write no global memory before it has completed and its writes
 *    are visible, so stream order holds as for plain launches. Work after an
 *    event wait or a copy on the stream is ordered as usual.
 *  - Kernels never trap. A kernel that gives up on an internal wait (bounded at
 *    about one second) records COVER_ERR_DEVICE_TIMEOUT in a per-device status
 *    word; read and clear it with cover_device_status().
 *  - Tensors are dense and contiguous (row-major, last index fastest), but where an
 *    entry point takes strides.
 */
#ifndef COVER_H_
#define COVER_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  COVER_OK = 0,
  COVER_ERR_INVALID_ARG = -1,    /* null required pointer, bad size, misaligned pointer */
  COVER_ERR_UNSUPPORTED = -2,    /* valid request outside what the kernels implement (e.g. head dim) */
  COVER_ERR_CUDA = -3,           /* a CUDA runtime call or launch failed */
  COVER_ERR_DEVICE_TIMEOUT = -4  /* a kernel gave up on a bounded internal wait (status word only) */
} cover_status_t;

/*
 * Two-view override attention, bf16 in / bf16 out, fp32 accumulation.
 * Section 5.1 (Attn(Q, K', V') over the overridden memory, softmax scale
 * 1/sqrt(d)) and Appendix B.1-B.4 (diagonal correction of seed queries).
 *
 *   q          [B, Hq,  L, D] bf16  queries from the masked-seed input
 *   k_cached   [B, Hkv, L, D] bf16  overridden memory K' (seed columns already
 *   v_cached   [B, Hkv, L, D] bf16  hold the previous step's cached states)
 *   k_seedmask [B, Hkv, n_seeds, D] bf16  row s = key   of position seed_idx[b, s]
 *   v_seedmask [B, Hkv, n_seeds, D] bf16  row s = value of position seed_idx[b, s]
 *                                   computed from the masked input (may be NULL
 *                                   when n_seeds == 0)
 *   seed_idx   [B, n_seeds] int32   seed positions per batch row, any order.
 *                                   Entries outside [0, L) are ignored; if a
 *                                   position repeats, the lowest slot s is used.
 *   out        [B, Hq, L, D] bf16   o_i (corrected for seed rows)
 *   lse        [B, Hq, L] fp32      natural-log log-sum-exp of the scaled
 *                                   scores of each row's own view (NULL = skip)
 *
 * Query head hq reads KV head hq / (Hq / Hkv) (contiguous groups). No causal
 * mask. For non-seed rows the result is plain attention over K', V'; for a
 * seed row i the diagonal term uses (k_i, v_i) instead of (k'_i, v'_i).
 *
 * Requirements: D == 128 (else COVER_ERR_UNSUPPORTED); B, Hq, Hkv, L >= 1;
 * Hq % Hkv == 0; 0 <= n_seeds <= L; q, k_cached, v_cached, out, k_seedmask,
 * v_seedmask 16-byte aligned; lse 4-byte aligned. Any L >= 1 is supported.
 * Otherwise COVER_ERR_INVALID_ARG. The inputs must not alias out / lse.
 */
int cover_attn_fwd(const void* q, const void* k_cached, const void* v_cached,
                   const void* k_seedmask, const void* v_seedmask,
                   const int32_t* seed_idx, int n_seeds,
                   int B, int Hq, int Hkv, int L, int D,
                   void* out, float* lse, void* stream);

/*
 * The same operation in fp32 throughout (float tensors, fp32 FMA on CUDA
 * cores, accurate expf). Intended for small fp32 checks. D in {64, 128}.
 * Same layouts, ownership and errors as cover_attn_fwd (4-byte alignment).
 */
int cover_attn_fwd_f32(const float* q, const float* k_cached, const float* v_cached,
                       const float* k_seedmask, const float* v_seedmask,
                       const int32_t* seed_idx, int n_seeds,
                       int B, int Hq, int Hkv, int L, int D,
                       float* out, float* lse, void* stream);

/*
 * Prefix-cache variant (Section 6.6 "Compatibility with Fast-dLLM": only the
 * active block's queries are recomputed while the memory holds every
 * position). The memory k_cached / v_cached is [B, Hkv, Lk, D] (overridden at
 * the seeds, as above); the queries q and the outputs out / lse are
 * [B, Hq, Lq, D] / [B, Hq, Lq], and query row r sits at memory position
 * q0 + r (0 <= q0, q0 + Lq <= Lk). seed_idx holds memory positions in
 * [0, Lk); a seed inside [q0, q0 + Lq) gets its leave-one-out view on the
 * diagonal column q0 + r, a seed outside the window affects only the memory.
 * With Lq = Lk and q0 = 0 this is cover_attn_fwd. Types, layouts, ownership
 * and errors as cover_attn_fwd / cover_attn_fwd_f32, plus
 * COVER_ERR_INVALID_ARG for Lq < 1, Lk < 1, q0 < 0 or q0 + Lq > Lk.
 * The bf16 call may run a window of grouped-query heads (G = Hq / Hkv >= 2,
 * Lq <= 256, G * Lq <= 1024, Lk <= 8192) on a kernel of its own: the G query
 * heads of a KV head packed into common Q tiles, the keys split over a cluster
 * of up to 8 CTAs that combine their partial softmax states. It does so where
 * a launch-time model (the clusters that fit on the GPU at once, the KV steps
 * of each kernel's longest chain) predicts it to be faster than the square
 * kernel. Its rows agree with the square kernel's up to rounding (not bit for
 * bit). Any other window runs on the square kernel, where the rows of a KV
 * head's query heads may share Q tiles too; its window rows equal the square
 * launch's, bit for bit unless one of the two launches splits the rows' keys in
 * two halves (merged up to rounding) and the other does not.
 */
int cover_attn_fwd_prefix(const void* q, const void* k_cached, const void* v_cached,
                          const void* k_seedmask, const void* v_seedmask,
                          const int32_t* seed_idx, int n_seeds,
                          int B, int Hq, int Hkv, int Lq, int Lk, int q0, int D,
                          void* out, float* lse, void* stream);
int cover_attn_fwd_prefix_f32(const float* q, const float* k_cached, const float* v_cached,
                              const float* k_seedmask, const float* v_seedmask,
                              const int32_t* seed_idx, int n_seeds,
                              int B, int Hq, int Hkv, int Lq, int Lk, int q0, int D,
                              float* out, float* lse, void* stream);

/*
 * Seed routing as the attention kernels see it (seed-set semantics of
 * Sections 3 and 5.1), exported for checking.
 *   slot_out   [B, L] int32: slot s of the seed naming position r, else -1
 *   bitmap_out [B, ceil(L/128), 4] uint32: bit r%32 of word (r%128)/32 of
 *              tile r/128 is set iff slot_out[b, r] >= 0
 *   n_invalid_out [1] int32: entries out of [0, L) plus repeated positions
 * seed_idx may be NULL when n_seeds == 0. Requirements: B, L >= 1,
 * 0 <= n_seeds <= L (else COVER_ERR_INVALID_ARG).
 */
int cover_seed_route(const int32_t* seed_idx, int n_seeds, int B, int L,
                     int32_t* slot_out, uint32_t* bitmap_out, int32_t* n_invalid_out,
                     void* stream);
/* The same function under the name the boundary's specification gives it
 * (cover_seed_route_debug); identical arguments, results and errors. */
int cover_seed_route_debug(const int32_t* seed_idx, int n_seeds, int B, int L,
                           int32_t* slot_out, uint32_t* bitmap_out, int32_t* n_invalid_out,
                           void* stream);

/*
 * Bytes of device workspace cover_score_fwd needs for n_seq segments.
 * The caller allocates it once, fills it with zeros, and may pass the same
 * buffer to every later call (each call leaves it zeroed again). Calls that
 * share one workspace must not run concurrently on the GPU.
 */
size_t cover_score_workspace_bytes(int n_seq);

/*
 * Fused per-position scoring over the vocabulary and top-k seed selection.
 * Section 3 (greedy token y_hat = argmax p, confidence c = max p), Section 6.1
 * (entropy-ordered unmasking: H = -sum p ln p), Section 5.3 (uncertainty
 * u = -log p(y), Score = u (1 + d_in)/(1 + d_out), top-k over eligible rows).
 *
 *   logits  [N, V] bf16   one row per scored position, softmax at temperature 1
 *   n_seq               rows split into n_seq equal consecutive segments
 *                       (sequences); top-k is taken per segment
 *   cur_tok [N] int32   current token y of each row; NULL => y = argmax row
 *   d_in, d_out [N] f32 influence / drift terms of the score; NULL => 0
 *   eligible [N] uint8  nonzero = row may be selected; NULL => all rows
 *   topk                k per segment (0 <= k <= N / n_seq)
 * Outputs (per row): maxprob = c, entropy = H, argmax = y_hat (lowest index
 * among equal maxima), score = Score. Per segment: topk_idx [n_seq, topk]
 * (row offsets within the segment, by score descending then index
 * ascending; -1 where fewer than k rows are eligible) and topk_score
 * [n_seq, topk] (NULL = skip; -inf where idx is -1).
 * workspace: cover_score_workspace_bytes(n_seq) zero-filled bytes (see above).
 *
 * Requirements: N, V >= 1; 1 <= n_seq; N % n_seq == 0; N / n_seq <= 4096;
 * logits 16-byte aligned (any V; rows need not be 16-byte aligned).
 * A cur_tok entry outside [0, V) yields NaN u and score for that row.
 * Non-finite logits give unspecified results. Otherwise COVER_ERR_INVALID_ARG.
 */
int cover_score_fwd(const void* logits, int N, int V, int n_seq,
                    const int32_t* cur_tok, const float* d_in, const float* d_out,
                    const uint8_t* eligible, int topk,
                    float* maxprob, float* entropy, int32_t* argmax, float* score,
                    int32_t* topk_idx, float* topk_score,
                    void* workspace, void* stream);

/*
 * cover_score_fwd without a workspace argument. The paper has no counterpart:
 * this entry point exists for callers that cannot allocate device memory for
 * a workspace - for example a serving loop that reserves all of its GPU
 * memory up front and forbids allocation afterwards, or a plugin interface
 * that hands the library its inputs and outputs but no allocator.
 *
 * Same arguments, layouts, results and errors as cover_score_fwd. The
 * per-sequence counters that cover_score_fwd keeps in the caller's workspace
 * live here in one fixed device array of the library, sized for at most
 * COVER_NOALLOC_MAX_SEQ (4096) sequences; n_seq beyond that returns
 * COVER_ERR_INVALID_ARG. Every device that loads the library holds this
 * 16 KB array until the process exits. The call allocates nothing: no
 * cudaMalloc / cudaFree, no allocating library routine; it clears the
 * counters it uses with an asynchronous memset on `stream`, then launches.
 *
 * The first call on each device looks up the array's device address
 * (cudaGetSymbolAddress, with that device current); make that first call
 * before any stream capture begins. The address is kept per context: after
 * cudaDeviceReset the next call (again outside any capture) looks it up in
 * the new context. All calls share the one array: calls
 * that overlap on the GPU (different streams, or different host threads
 * without ordering) race on it and can return wrong top-k results.
 */
#define COVER_NOALLOC_MAX_SEQ 4096
int cover_score_fwd_noalloc(const void* logits, int N, int V, int n_seq,
                            const int32_t* cur_tok, const float* d_in, const float* d_out,
                            const uint8_t* eligible, int topk,
                            float* maxprob, float* entropy, int32_t* argmax, float* score,
                            int32_t* topk_idx, float* topk_score, void* stream);

/*
 * Seed key/value cache (Section 5.1, "KV cache override yields a stable
 * drafting view"), per layer. k, v: the layer's states [B, Hkv, L, D];
 * k_cache, v_cache: [B, Hkv, n_seeds, D]; seed_idx: int32 [B, n_seeds]
 * positions (the row of the previous step's cover_score_decide_fwd output
 * works as is). Elements are elem_bytes (2 for bf16, 4 for fp32) bytes; a row
 * (D * elem_bytes) must be a multiple of 16 bytes and every pointer 16-byte
 * aligned. All pointers are device pointers owned by the caller.
 *
 * A slot names its position when the position is in [0, L) and no lower slot
 * of the same batch row names it (the lowest slot wins, as in cover_attn_fwd).
 *
 * cover_seed_kv_gather (at selection, step t-1): k_cache[b, h, s] =
 *   k[b, h, seed_idx[b, s]], likewise v; a slot with an out-of-range position
 *   gets zeros (a repeated position is copied again).
 * cover_seed_kv_override (at step t, after the layer's k, v were computed from
 *   the input with the seeds masked): swaps row seed_idx[b, s] of k / v with
 *   row s of k_cache / v_cache for every slot that names a position. Afterwards
 *   k, v hold the overridden memory K', V' and k_cache, v_cache hold the
 *   masked-input pairs (k_i, v_i): exactly cover_attn_fwd's k_cached,
 *   v_cached, k_seedmask, v_seedmask. Slots that name no position leave both
 *   buffers untouched.
 * n_seeds = 0 is a no-op (seed pointers may then be NULL).
 * Errors: COVER_ERR_INVALID_ARG for a NULL required pointer, B, Hkv, L or D
 * < 1, n_seeds < 0, elem_bytes not 2 or 4, a row that is not a multiple of 16
 * bytes or is longer than 64 KB, or a misaligned pointer; COVER_ERR_UNSUPPORTED if B * Hkv > 2^31 - 1 or
 * n_seeds > 1048560; COVER_ERR_CUDA for a launch failure.
 */
int cover_seed_kv_gather(const void* k, const void* v, const int32_t* seed_idx, int n_seeds,
                         int B, int Hkv, int L, int D, int elem_bytes,
                         void* k_cache, void* v_cache, void* stream);
int cover_seed_kv_override(void* k, void* v, const int32_t* seed_idx, int n_seeds,
                           int B, int Hkv, int L, int D, int elem_bytes,
                           void* k_cache, void* v_cache, void* stream);

/*
 * Rotary positions of a layer's queries and keys, before the attention or the
 * memory takes them (the paper's models rotate q and k; it gives no formula).
 * Column pair i (0 <= i < R / 2) of a row at position t turns by t * inv_freq[i]
 * radians:
 *   y_a = mscale (x_a cos - x_b sin),  y_b = mscale (x_a sin + x_b cos),
 * (a, b) = (2i, 2i + 1) if interleaved != 0, else (i, i + R / 2); with
 * inverse != 0 by the opposite angle. That is the gradient too: d loss / d x is
 * the inverse rotation (same mscale) of d loss / d y. Columns R .. D - 1 are
 * copied. Contexts are stretched by the frequencies and mscale.
 *
 *   q, q_out [B, Hq, L, D], k, k_out [B, Hkv, L, D]: elements of elem_bytes (2: bf16, 4: fp32)
 *   strides  HOST int64 [12]: strides in elements of (B, H, L) of q, k, q_out, k_out (the
 *            last dimension is dense); read before the call returns. Rows laid out as a
 *            projection leaves them ([B, L, H, D] in memory) need no transposition.
 *   inv_freq [R / 2] fp64; the angle is reduced exactly modulo a turn, so positions
 *            far out lose nothing (the columns of one that is not finite are NaN)
 *   pos      [B, L] int32 position of every row (any value), or NULL: row l is at pos0 + l
 * k is NULL and Hkv is 0 where only q is wanted. q_out may be q with the same
 * strides (in place), likewise k; outputs that overlap an input in another way, or
 * rows of one output that overlap, give unspecified results. L = 0 is a no-op.
 * Errors: COVER_ERR_INVALID_ARG for a NULL required pointer, B or Hq < 1, Hkv or
 * L < 0, D < 1, R odd, negative or above D, elem_bytes not 2 or 4, a pointer that
 * is not aligned to its elements; COVER_ERR_UNSUPPORTED for D > 4096;
 * COVER_ERR_CUDA for a launch failure. Rows that are all 16-byte aligned (and R
 * and D that split into 16-byte vectors) run on 16-byte accesses.
 */
int cover_rope_fwd(const void* q, const void* k, void* q_out, void* k_out, const int64_t* strides,
                   int B, int Hq, int Hkv, int L, int D, int R,
                   const double* inv_freq, const int32_t* pos, int pos0,
                   int interleaved, float mscale, int inverse, int elem_bytes, void* stream);

/*
 * An 8-bit key/value memory (the prefix cache of Section 6.6 in half the bytes), per layer:
 *   k8, v8       [B, Hkv, L, D] e4m3 codes
 *   k_exp, v_exp [B, Hkv, L]    e8m0 exponent bytes, one a row
 * A row's values are code * 2^(x - 127), x its byte; x = 255: the row reads as NaN. A power of two
 * scales without rounding: every value is exact in bf16 and fp32.
 *
 * cover_kv8_write quantises rows as they are written: x is the smallest byte with
 *   max |row| <= 448 * 2^(x - 127), held to 17 .. 246 (127 for a row of zeros); the codes are the nearest
 *   e4m3 values of row * 2^(127 - x), ties to even, saturating. A row with an element
 *   that is not finite is stored as NaN (x = 255, codes 0). k, v [B, Hkv, n, D] are bf16 (elem_bytes
 *   2) or fp32 (4); strides: HOST int64 [6], strides in elements of (B, H, n) of k, v, the last
 *   dimension dense. Slot s goes to position pos0 + s, or to pos[b, s] (int32 [B, n]) where pos is not
 *   NULL: a listed position outside [0, L) is left out, and where a position is listed again
 *   the lowest slot is taken (as in cover_attn_fwd). Every other row of the memory is left as it
 *   was. With pos = seed_idx this overrides the memory at the seeds with their cached states. A listed
 *   write compares every slot with the lower ones: 4 x 8 heads, 512 rows of 128 bf16 take 8 us (5 at consecutive
 *   positions), 8191 rows 99 (36).
 * cover_kv8_read reads rows back into k, v [B, Hkv, n, D] (dense, bf16 or fp32): row s from
 *   position pos0 + s or pos[b, s]; a listed position outside [0, L) reads as zeros.
 *
 * n = 0 is a no-op. Errors: COVER_ERR_INVALID_ARG for a NULL required pointer, B, Hkv, L or D < 1, n < 0,
 * elem_bytes not 2 or 4, pos0 < 0 or pos0 + n > L without a list, k, v, k8 or v8 not 16-byte
 * aligned, a stride (of a dimension longer than 1) that is not a multiple of 16 bytes;
 * COVER_ERR_UNSUPPORTED for D other than 64 and 128, or B > 65535; COVER_ERR_CUDA for a launch failure.
 */
int cover_kv8_write(const void* k, const void* v, const int64_t* strides,
                    const int32_t* pos, int pos0, int n, int B, int Hkv, int L, int D, int elem_bytes,
                    void* k8, void* v8, uint8_t* k_exp, uint8_t* v_exp, void* stream);
int cover_kv8_read(const void* k8, const void* v8, const uint8_t* k_exp, const uint8_t* v_exp,
                   const int32_t* pos, int pos0, int n, int B, int Hkv, int L, int D, int elem_bytes,
                   void* k, void* v, void* stream);

/*
 * cover_attn_fwd_prefix over an 8-bit memory (k8, v8, k_exp, v_exp as above, Lk positions; D = 128): bf16
 * queries q [B, Hq, Lq, D] at memory positions q0 + r, bf16 out, fp32 lse (NULL = skip), and the seeds'
 * masked-input pairs k_seedmask, v_seedmask [B, Hkv, n_seeds, D] in bf16. In addition:
 *   key_lo, key_hi [B, Lq] int32 or NULL (0, Lk): row r of batch row b sees the keys key_lo <= j < key_hi
 *     only (held to 0 .. Lk): a padded batch's lengths, a prefix, blocks that see themselves and
 *     those before, documents. A row that sees no key gets out = 0, lse = -inf.
 *     A seed row's own pair is seen where its position is.
 *   softcap  0, or c > 0: every score s = q . k / sqrt(D), a seed's own too, becomes c tanh(s / c)
 *     (c above 2^60 counts as 2^60, c below 2^-30 as 2^-30).
 * What a row does not see does not reach it, NaN included; a row that sees a key with k_exp or
 * v_exp above 246, or with a NaN code in its K or V row (0x7f or 0xff, which cover_kv8_write does
 * not write), gets NaN in out and lse.
 * Which kernel runs depends on the sizes, and on whether key ranges and a cap are given; equal rows of
 * different calls agree up to rounding. The
 * weights are rounded to bf16 or to 9 significant bits for their products with V, and a weight that
 * is, times its value's scale, below 2^-28 of the row's largest such product may count as zero in
 * out (not in lse).
 * Scores and sums are fp32: they hold where the largest elements of a query row and a key row multiply to less than 2^120 and
 * the values seen are at most 2^100, and 2^119 / Lk, in magnitude; beyond, a row may get infinities or NaN or lose small weights.
 * Value rows that are below 2^-80 throughout may lose bits, or count as zeros, beside rows of zeros. lse carries an error of
 * up to 2^-17 where the value rows seen are all zeros or their scales are far from 1.
 * workspace: cover_attn_prefix8_workspace_bytes(B, Hq, Hkv, Lq, Lk) bytes, 16-byte aligned, no initialisation
 * needed (NULL if that is 0): parts of the keys' results, and for windows that fill several tiles of 128 rows the whole
 * memory in bf16 (2048 rows, 32 / 8 heads over 131072 keys: 673 MB, beside a memory of 271). It is scratch of the call alone: calls that share one must not
 * run concurrently on the GPU.
 * The inputs must not alias out, lse or workspace. Errors as cover_attn_fwd_prefix, plus
 * COVER_ERR_INVALID_ARG for NULL k_exp or v_exp, a missing workspace, and a softcap that is
 * negative or not finite.
 */
size_t cover_attn_prefix8_workspace_bytes(int B, int Hq, int Hkv, int Lq, int Lk);
int cover_attn_fwd_prefix8(const void* q, const void* k8, const void* v8,
                           const uint8_t* k_exp, const uint8_t* v_exp,
                           const void* k_seedmask, const void* v_seedmask,
                           const int32_t* seed_idx, int n_seeds,
                           int B, int Hq, int Hkv, int Lq, int Lk, int q0, int D,
                           const int32_t* key_lo, const int32_t* key_hi, float softcap,
                           void* out, float* lse, void* workspace, void* stream);

/*
 * A key/value memory in pages, shared by the sequences of a server (the prefix cache of Section 6.6 for sequences that come and
 * go), per layer:
 *   k_pages, v_pages [n_pages, Hkv, page, D] bf16
 *   table            [B, M] int32: position t of sequence b is row t % page of the page table[b, t / page]; an entry
 *                    outside [0, n_pages) is a page that the sequence does not have
 * page is 16, 32, 64, 128 or 256, and M * page is below 2^31.
 *
 * cover_paged_append writes n rows of every sequence and rotates them on the way: row s of sequence b goes to position
 * start[b] + s where s < count[b] (count NULL: all n; the other rows are padding), or to pos[b, s] where pos is not NULL (start
 * and count are NULL then): of rows that name one position the lowest is taken (as in cover_kv8_write). A position below 0 or
 * without a page is left out; every other row of the pages is left as it was. Sequences that share a page must not write the
 * same of its rows in one call (one of them stays, which is not said).
 *   k, v [B, Hkv, n, D], q [B, Hq, n, D] (NULL with Hq = 0): elements of elem_bytes (2: bf16, 4: fp32); strides: HOST int64
 *     [9], strides in elements of (B, H, n) of k, v, q (the last dimension is dense)
 *   q_out [B, Hq, n, D], k_out [B, Hkv, n, D] (NULL: not wanted): dense, of the same type; all n rows of q and k turned,
 *     k_out where the program needs the rows besides (the seeds' masked-input rows)
 *   inv_freq [R / 2], interleaved, mscale: as in cover_rope_fwd (R = 0: nothing turns); k and q turn by rope_pos[b, s] (int32
 *     [B, n]), or by the row's position in the memory where it is NULL. Rows are turned in fp32 and rounded once.
 * k, v and q must overlap neither the pages nor the outputs, and k_pages not v_pages (the Python call refuses what overlaps the
 * pages). n = 0 is a no-op.
 * Errors: COVER_ERR_INVALID_ARG for a NULL required pointer, B, Hkv, D, M or n_pages < 1, Hq or n < 0, R odd, negative or above
 * D, elem_bytes not 2 or 4, neither or both of start and pos, count with pos, a pointer that is not aligned to its elements (the pages:
 * to 16 bytes); COVER_ERR_UNSUPPORTED for D other than 64 and 128, another page, M * page >= 2^31; COVER_ERR_CUDA for a
 * launch failure. Rows that are all 16-byte aligned (and an R that splits into 16-byte vectors) run on 16-byte accesses.
 */
int cover_paged_append(const void* k, const void* v, const void* q, void* q_out, void* k_out, const int64_t* strides,
                       const int32_t* table, int n_pages, int M, int page,
                       const int32_t* start, const int32_t* count, const int32_t* pos, const int32_t* rope_pos,
                       int n, int B, int Hq, int Hkv, int D, int R, const double* inv_freq, int interleaved,
                       float mscale, int elem_bytes, void* k_pages, void* v_pages, void* stream);

/*
 * cover_attn_fwd_prefix over a memory in pages (D = 128): bf16 queries q [B, Hq, Lq, D], bf16 out, fp32 lse [B, Hq, Lq]
 * (NULL = skip), the seeds' masked-input pairs k_seedmask, v_seedmask [B, Hkv, n_seeds, D] in bf16.
 *   lens [B] int32: keys of each sequence (held to 0 .. M * page). A position without a page holds no key.
 *   q0 [B] int32: position of each sequence's first query row; row r is at q0[b] + r (any value; NULL without seeds). It says which
 *     row is a seed's; what a row sees is said by the lengths and the ranges alone.
 *   key_lo, key_hi [B, Lq] int32 or NULL (0, lens[b]): row r of sequence b sees the keys key_lo <= j < key_hi only (any
 *     values): positions up to its own, blocks, windows, documents. A row that sees no key gets out = 0, lse = -inf.
 *     A seed row's own pair is seen where its position is.
 *   softcap 0, or c > 0: every score s = q . k / sqrt(D), a seed's own too, becomes c tanh(s / c) (c above 2^60 counts as
 *     2^60, c below 2^-30 as 2^-30).
 * What a row does not see does not reach it, NaN included: rows of a page behind a sequence's length may hold anything.
 * A row that sees an element of V that is not finite has no finite number in that column at least, be its weight 0 in fp32, and its lse is
 * as without it. Scores and sums are fp32: they hold where the values seen are at most 2^100 in magnitude, and 2^66 / Lk with a cap.
 * workspace: cover_attn_paged_workspace_bytes bytes, 16-byte aligned, no initialisation needed (NULL if that is 0): scratch of the
 * call alone; calls that share one must not run concurrently on the GPU. The inputs must not alias out, lse or workspace.
 * Errors: COVER_ERR_INVALID_ARG for a NULL required pointer, B, Hq, Hkv, Lq, M or n_pages < 1, Hq % Hkv != 0, n_seeds < 0, a
 * softcap that is negative or not finite, a misaligned pointer, a missing workspace; COVER_ERR_UNSUPPORTED for D != 128, another
 * page, M * page >= 2^31, B Hq Lq >= 2^31 - 256, n_pages Hkv page >= 2^34; COVER_ERR_CUDA for a launch failure; COVER_ERR_DEVICE_TIMEOUT via
 * cover_device_status.
 */
size_t cover_attn_paged_workspace_bytes(int B, int Hq, int Hkv, int Lq, int M, int page);
int cover_attn_fwd_paged(const void* q, const void* k_pages, const void* v_pages,
                         const int32_t* table, int n_pages, int M, int page, const int32_t* lens,
                         const void* k_seedmask, const void* v_seedmask, const int32_t* seed_idx, int n_seeds,
                         const int32_t* q0, int B, int Hq, int Hkv, int Lq, int D,
                         const int32_t* key_lo, const int32_t* key_hi, float softcap,
                         void* out, float* lse, void* workspace, void* stream);

/*
 * Log probabilities of given tokens (softmax at temperature 1 over rows of V logits), beside cover_score_fwd's u = -log p
 * for programs that score, compare or learn from answers: with the row's entropy, its logsumexp and its best alternatives.
 *   logits [N, V], elements of elem_bytes (2: bf16, 4: fp32)
 *   tok [N] int32 or NULL (then logp is not written): logp[i] = log p(tok[i]); a token outside [0, V) has logp = 0 (a row
 *     to be left out of sums)
 *   entropy, lse [N] fp32: H = -sum p ln p, lse = ln sum e^logit
 *   topk 0 .. 64: top_idx [N, topk] int32, top_logp [N, topk] fp32: the tokens of the largest logits (descending; equal
 *     ones by ascending index) and their log probabilities; -1 and -inf where V < topk. (NULL for topk = 0)
 * A logit of -inf is a token of probability 0. A row with NaN or +inf has NaN in logp (of a token in [0, V)), entropy and lse,
 * and unspecified alternatives (indexes in [-1, V)); a row of -inf alone has lse = -inf and NaN in logp, entropy and top_logp.
 * cover_logprob_bwd is the gradient: with p_j = e^(logit_j - lse),
 *   d_logits_j = p_j (d_lse - d_logp - sum_k d_top_k - d_entropy (ln p_j + entropy)) + [j = tok] d_logp
 *                + sum_k [j = top_idx_k] d_top_k,
 * rounded once to the logits' type. d_logp (with tok), d_entropy (with entropy), d_lse [N] and d_top [N, topk] (with
 * top_idx) are fp32 or NULL (0); a token or alternative outside [0, V) gets no gradient; a token listed again gets each
 * share. entropy and lse are the forward call's. d_logits may be logits itself, or must not overlap it.
 * N = 0 is a no-op. Errors: COVER_ERR_INVALID_ARG for a NULL required pointer, N < 0, V < 1, topk < 0, elem_bytes not 2 or 4,
 * a pointer that is not aligned to its elements; COVER_ERR_UNSUPPORTED for topk > 64; COVER_ERR_CUDA for a launch failure.
 */
int cover_logprob_fwd(const void* logits, int N, int V, int elem_bytes, const int32_t* tok, int topk,
                      float* logp, float* entropy, float* lse, int32_t* top_idx, float* top_logp, void* stream);
int cover_logprob_bwd(const void* logits, int N, int V, int elem_bytes, const float* lse,
                      const int32_t* tok, const float* d_logp, const float* entropy, const float* d_entropy,
                      const float* d_lse, const int32_t* top_idx, const float* d_top, int topk,
                      void* d_logits, void* stream);

/*
 * One decoding step's decisions, fused behind the scoring pass
 * (Section 5.2 "Threshold drafting" and the Keep / Replace / ReMask revision
 * rule, Section 3 state update, Section 5.3 stability-aware seed score,
 * adaptive revision rate and seed exclusions).
 *
 * The N rows split into n_seq equal segments (sequences); row i of a segment
 * is response position pos0 + i. Per row the scoring pass computes c = max p,
 * y_hat = argmax p (ties to the lower index) and H exactly as
 * cover_score_fwd, and u = -log p(tok) for the current token. Then, per
 * segment (state arrays updated in place):
 *   1. Drafting: among rows with tok == mask_id and draft_ok != 0 (all such
 *      rows when draft_ok is NULL), those with c > tau_draft; if more than
 *      draft_budget, the largest c are kept (ties to the lower index). If none
 *      is drafted and min_one != 0, the allowed masked row with the lowest H is
 *      drafted (ties to the lower index). Drafted rows take tok = y_hat.
 *   2. Revision of the previous seeds (rows with flag bit COVER_FLAG_SEED set
 *      and tok != mask_id): Keep if y_hat == tok; else Replace (tok = y_hat)
 *      if c > tau_draft; else ReMask (tok = mask_id, remask_cnt + 1, saturating
 *      at 255).
 *   3. Seed score of every unmasked row of the updated state, in fp32:
 *      score = (u * (1 + d_in)) / (1 + d_out), with u = ln Z = -log c for
 *      drafted and replaced rows and the current token's u otherwise (NULL
 *      d_in / d_out = 0). Masked rows and non-finite scores get -INFINITY.
 *   4. Adaptive revision rate: n_t = rows with a finite score, n_above = rows
 *      with n_t * score > sum of the scores (fp64; this is n_t * pi_t),
 *      k = min(ceil(sqrt(n_above)), max_seeds).
 *   5. New seeds: the k highest-scoring rows (ties to the lower index) among
 *      the scored rows that were not previous seeds and have
 *      remask_cnt < remask_budget; fewer if fewer are eligible. Their flag bit
 *      COVER_FLAG_SEED is set and every other row's is cleared (other flag bits
 *      are kept); seed_idx[seg, 0..n_seeds) lists their positions pos0 + i in
 *      order, the rest of the row is -1, so it can be passed to
 *      cover_attn_fwd as the next step's seed_idx with n_seeds = max_seeds.
 *
 * logits   bf16 [N, V] row-major, 16-byte aligned (device).
 * d_in, d_out, draft_ok: [N] or NULL (device).
 * tok      int32 [N] (device, in/out); flags, remask_cnt uint8 [N] (in/out).
 * maxprob, entropy, score float [N]; argmax int32 [N] (device, out).
 * seed_idx int32 [n_seq, max_seeds] (device, out; may be NULL if max_seeds is
 *          0); n_seeds int32 [n_seq] (out); stats int32 [n_seq, 6] or NULL:
 *          drafted, kept, replaced, remasked, n_t, n_above per segment.
 * workspace: cover_decide_workspace_bytes(N, n_seq) bytes of device memory,
 *          16-byte aligned, zero-filled before its first use; it is left ready
 *          for the next call on the same stream.
 * phase COVER_DECIDE_ALL runs steps 1-5 with the given d_in / d_out.
 * phase COVER_DECIDE_UPDATE runs steps 1-2 only: it writes maxprob, entropy,
 *   argmax, the updated tok / remask_cnt, flag bit COVER_FLAG_DRAFTED on the
 *   rows drafted in this step (bit COVER_FLAG_SEED still marks the previous
 *   seeds), stats[.., 0..3], and the uncertainty of every row's updated token
 *   into the workspace; score, seed_idx and n_seeds are not written (they may
 *   be NULL). Then cover_attn_mass_fwd produces d_in / d_out from the updated
 *   state, and cover_seed_select_fwd runs steps 3-5 on the same workspace. This
 *   is the order of Section 5.3, where d_in sums over the masked positions after
 *   the update and d_out over the positions drafted in this step.
 * Errors: COVER_ERR_INVALID_ARG for a NULL required pointer, N, V or n_seq < 1,
 * N % n_seq != 0, N / n_seq > 4096, draft_budget, remask_budget or max_seeds
 * < 0, an unknown phase, or a misaligned pointer. COVER_ERR_CUDA for a launch
 * failure.
 */
#define COVER_FLAG_SEED 1
#define COVER_FLAG_DRAFTED 2
#define COVER_DECIDE_ALL 0
#define COVER_DECIDE_UPDATE 1
size_t cover_decide_workspace_bytes(int N, int n_seq);
int cover_score_decide_fwd(const void* logits, int N, int V, int n_seq,
                           const float* d_in, const float* d_out, const uint8_t* draft_ok,
                           float tau_draft, int draft_budget, int remask_budget, int mask_id,
                           int min_one, int pos0, int max_seeds, int phase,
                           int32_t* tok, uint8_t* flags, uint8_t* remask_cnt,
                           float* maxprob, float* entropy, int32_t* argmax, float* score,
                           int32_t* seed_idx, int32_t* n_seeds, int32_t* stats,
                           void* workspace, void* stream);

/*
 * d_in and d_out of the seed score (Section 5.3) from the attention of the
 * current pass, averaged over the Hq heads: for the response positions
 * pos0 .. pos0 + per - 1 of every batch row (state row b * per + i is
 * position pos0 + i),
 *   d_in(j)  = sum over masked positions q (tok == mask_id) of A[q -> j],
 *   d_out(j) = sum over positions i with flag bit COVER_FLAG_DRAFTED of A[j -> i],
 * where A_h[q -> j] = exp(q_q . k'_j / sqrt(D) - lse_h(q)) and a seed query's
 * diagonal uses its masked-input key (the leave-one-out view; lse is the one
 * cover_attn_fwd wrote, that of the corrected distribution). Only response
 * queries and response keys contribute. Tensor-core recomputation of the
 * per x per block of every head (once per orientation, so that both sums are
 * row sums); partial sums per head are added in a fixed order, so the result
 * is deterministic.
 * q [B, Hq, L, 128], k_cached [B, Hkv, L, 128], k_seedmask [B, Hkv, n_seeds,
 * 128] bf16; seed_idx int32 [B, n_seeds]; lse float [B, Hq, L]; tok int32,
 * flags uint8 [B * per] (cover_score_decide_fwd's state after the update
 * phase); d_in, d_out float [B * per] (out). workspace:
 * cover_attn_mass_workspace_bytes(B, Hq, per) bytes, 16-byte aligned, no
 * initialisation needed. All device pointers, owned by the caller.
 * Errors: COVER_ERR_INVALID_ARG for a NULL required pointer, B, Hq, Hkv, L,
 * per < 1, Hq % Hkv != 0, pos0 < 0 or pos0 + per > L, n_seeds < 0 or > L, or a
 * misaligned pointer; COVER_ERR_UNSUPPORTED for D != 128 or per > 16384 (the
 * per-column data of a response block is staged in shared memory);
 * COVER_ERR_CUDA for a launch failure; COVER_ERR_DEVICE_TIMEOUT via
 * cover_device_status.
 */
size_t cover_attn_mass_workspace_bytes(int B, int Hq, int per);
int cover_attn_mass_fwd(const void* q, const void* k_cached, const void* k_seedmask,
                        const int32_t* seed_idx, int n_seeds, const float* lse,
                        int B, int Hq, int Hkv, int L, int D,
                        const int32_t* tok, const uint8_t* flags, int mask_id, int pos0, int per,
                        void* workspace, float* d_in, float* d_out, void* stream);

/*
 * Steps 3-5 of cover_score_decide_fwd (seed score, adaptive revision rate,
 * selection) after a COVER_DECIDE_UPDATE call on the same workspace and state:
 * score = u * (1 + d_in) / (1 + d_out) with u of the updated token; clears flag
 * bits COVER_FLAG_SEED and COVER_FLAG_DRAFTED, then sets COVER_FLAG_SEED on the
 * new seeds; writes score [N], seed_idx [n_seq, max_seeds], n_seeds [n_seq] and
 * stats[.., 4..5]. Arguments and errors as cover_score_decide_fwd.
 */
int cover_seed_select_fwd(int N, int n_seq, const float* d_in, const float* d_out,
                          int remask_budget, int mask_id, int pos0, int max_seeds,
                          int32_t* tok, uint8_t* flags, uint8_t* remask_cnt, float* score,
                          int32_t* seed_idx, int32_t* n_seeds, int32_t* stats,
                          void* workspace, void* stream);

/*
 * Synchronises `stream`, then returns and clears the current device's status
 * word: COVER_OK, or COVER_ERR_DEVICE_TIMEOUT if a kernel gave up on a
 * bounded wait since the last call. Returns COVER_ERR_CUDA if the
 * synchronisation itself fails.
 */
int cover_device_status(void* stream);

/* Static, human-readable name of a status code. Never NULL. */
const char* cover_status_str(int code);

#ifdef __cplusplus
}
#endif

#endif /* COVER_H_ */
