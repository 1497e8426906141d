/*
 * loopserve.h -- C ABI of libloopserve: the per-layer hot path of LoopServe's online-sparsified
 * prefill attention and its decode-time KV retention scorer (arxiv 2507.13681), for AMD MI355X
 * (gfx950).  Plain C, no exceptions cross this boundary.
 *
 * Conventions for every entry point
 *   - All tensor pointers are DEVICE pointers on the context's GPU, 16-byte aligned, row-major and
 *     contiguous in the stated shape (ls_rows: of the strides it states).  Only the structures and scalars are host data.
 *   - The caller owns every tensor.  The library owns only the context and its workspace, which is
 *     allocated once in ls_create; no entry point below allocates or frees device memory.
 *   - Calls are asynchronous on `hip_stream` (a hipStream_t, NULL = the default stream) and contain
 *     no host synchronisation; outputs are valid once the stream reaches the end of the call.
 *     Counts (v_cnt, s_cnt, keep_cnt) stay on the device, so score -> select -> prefill chain without
 *     a host round trip.  Calls that share a context must be issued on one stream at a time (they
 *     share the workspace, and counters through which the workgroups of a launch find out which of them
 *     is the last).  Calls that overlap all the same spoil their own results, and may leave those
 *     counters off for one or two later calls of ls_decode_attend or ls_paged_attend on that context; the ones after
 *     that are sound again.  A recorded call (HIP graph) always uses the same counters: replays that
 *     overlapped leave it unsound until three other calls of these two have run.
 *   - Return value: LS_OK or a negative ls_status; ls_last_error(ctx) then describes the failure.
 *     Argument errors are detected on the host before anything is launched.
 *   - dtype is the storage type of q / k / v / out (bf16 or fp32); tile products accumulate in fp32
 *     and every line weight, count and index output is fp32 / int32 regardless of dtype.
 *   - Query head h reads KV head h / (Hq / Hkv)  (grouped-query attention).
 *   - Positions: the context has n keys at positions 0..n-1; the newest turn is the last n_hat of
 *     them; new-turn row a sits at absolute position n - n_hat + a and sees keys <= that position.
 */
#ifndef LOOPSERVE_H
#define LOOPSERVE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ls_ctx ls_ctx;

typedef enum {
    LS_OK = 0,
    LS_EINVAL = -1,      /* null or misaligned pointer, bad enum */
    LS_ESHAPE = -2,      /* unsupported or inconsistent shape */
    LS_EALPHA = -3,      /* alpha outside [0, 1] */
    LS_EWORKSPACE = -4,  /* context workspace too small for this call */
    LS_EHIP = -5         /* a HIP runtime call failed */
} ls_status;

typedef enum { LS_BF16 = 0, LS_F32 = 1 } ls_dtype;

/* Limits: d in {64, 128}; w <= 256; n <= LS_MAX_N for ls_select / ls_sparse_prefill. */
#define LS_MAX_N 262144
#define LS_MAX_W 256

typedef struct {
    int32_t B;       /* batch */
    int32_t Hq;      /* query heads */
    int32_t Hkv;     /* KV heads, divides Hq */
    int32_t d;       /* head dimension */
    int64_t n;       /* keys in the context (cache length for ls_kv_compress) */
    int64_t n_hat;   /* rows of the newest turn, 1 <= n_hat <= n (ignored by ls_kv_compress) */
    int32_t w;       /* scoring rows: window size (n_obs for ls_kv_compress) */
    int32_t dtype;   /* ls_dtype */
    float scale;     /* logit scale; <= 0 means 1/sqrt(d) */
} ls_shape;

/* Bytes of workspace that every call on `shape` (and ls_kv_compress with `budget`) fits in: per query head and key
 * 24 bytes, or 16 and w / 16 more where that is larger, and up to 66 MiB that ls_sparse_prefill uses for parts of long
 * row blocks and ls_score for the rows of explicit positions.  Both calls run in less, and ls_score with explicit
 * positions faster in more (up to B * Hq * w * n * 4 bytes on top).
 * Host-only, no GPU needed.  Returns 0 for an invalid shape. */
size_t ls_workspace_bytes(const ls_shape* shape, int32_t budget);

/* Creates a context on GPU `device` with a workspace of `workspace_bytes` (device memory, allocated
 * here, freed by ls_destroy).  The context can serve any shape whose ls_workspace_bytes fits. */
int ls_create(ls_ctx** out, int device, size_t workspace_bytes);
void ls_destroy(ls_ctx* ctx);
/* Message of the last failing call on this context (never NULL; not thread-safe); with ctx == NULL, of the
 * last failing call that takes no context (ls_kv_compress_static). */
const char* ls_last_error(const ls_ctx* ctx);

/*
 * ls_score -- Alg. 2, steps "A = Softmax(Q~ K^T / sqrt(d_k))", SlashSum, VerticalSum (Appendix,
 * Algorithm "Adaptive Prefilling Sparsification"), with the line definitions of Sec. 3.1 (Obs. 1):
 * a vertical line is a key column, a slash line is a diagonal.
 *
 *   q_win  [B,Hq,w,d]   queries of the scoring rows
 *   q_pos  [w] int64    their absolute positions (each clipped to [0, n-1]), device memory; NULL = the last w
 *                       positions n-w .. n-1 (the newest query window)
 *   k      [B,Hkv,n,d]
 * Outputs (fp32):
 *   vert   [B,Hq,n]  vert[b]  = sum_t A[t][b]              (column b)
 *   slash  [B,Hq,n]  slash[o] = sum_t A[t][p_t - o]        (diagonal o = query pos - key pos)
 *   vmax, smax [B,Hq,n]  the largest single entry of each line (the w^max of Alg. 2)
 *   total  [B,Hq]    sum of all entries of A (about w)
 * The softmax is causal (row t sees keys <= p_t).  All sums are formed in a fixed order (bit-reproducible).
 */
int ls_score(ls_ctx* ctx, const ls_shape* shape, const void* q_win, const int64_t* q_pos, const void* k,
             float* vert, float* slash, float* vmax, float* smax, float* total, void* hip_stream);

/*
 * ls_select -- Alg. 2 from Desc_Sort to the end of the while-loop: both line lists are sorted by
 * weight (descending; ties: smaller index first) and the greedy loop takes list heads until the
 * accounted weight reaches alpha * total.  Gain of a slash is w_s - ol_v, of a vertical w_v - ol_s,
 * where ol_* sums w^max of the lines taken from the other list; cost is max(1, length - #taken from
 * the other list) with length min(n_hat, n - index); the slash is taken when gain_s * cost_v >=
 * gain_v * cost_s; gains are not clamped; an empty list defers to the other.  All in binary32.
 *
 *   vert, slash, vmax, smax [B,Hq,n], total [B,Hq]   as produced by ls_score
 * Outputs:
 *   v_idx [B,Hq,cap_v] int32  selected columns, ascending;   v_cnt [B,Hq] int32
 *   s_idx [B,Hq,cap_s] int32  selected diagonals, ascending; s_cnt [B,Hq] int32
 *   accounted [B,Hq] fp32 or NULL: the loop's final sum.
 * A count larger than its capacity means the list was truncated to the smallest `cap` indices
 * (LS_STAT_S_TRUNCATED / LS_STAT_V_TRUNCATED in the status word).
 * With accounted == NULL the loop stops as soon as the result is decided (when no remaining line
 * has a positive gain every line ends up selected); with accounted != NULL it runs to the end.
 * shape->w and dtype are ignored.  n <= LS_MAX_N.
 */
int ls_select(ls_ctx* ctx, const ls_shape* shape, float alpha,
              const float* vert, const float* slash, const float* vmax, const float* smax, const float* total,
              int32_t* v_idx, int32_t* v_cnt, int32_t cap_v,
              int32_t* s_idx, int32_t* s_cnt, int32_t cap_s,
              float* accounted, void* hip_stream);

/*
 * ls_score_window / ls_select_exact -- Alg. 2 with the marginal contribution of a line taken exactly.
 * Sec. 5.1 describes the quantities the loop compares as the marginal contributions of the two list
 * heads; the listing bounds the part of a candidate that is already covered by the sum of w^max of the
 * lines taken from the other list, which is what ls_select computes.  Here that part is added up cell by
 * cell (a diagonal o and a column b share the cell of the scored row at position b + o, if there is one),
 * so gains are never negative, the accounted sum is the weight of the union of the selected lines on the
 * scored rows, and selections that mix columns and diagonals survive.  Opt-in: it needs the window
 * matrix itself (w * n floats per head) and walks the lists one pick at a time.
 *
 * ls_score_window: the softmax step of Alg. 2 with the matrix kept.
 *   q_win, q_pos, k as for ls_score;  a_win [B,Hq,w,n] fp32: A[t][b] for keys b <= p_t, 0 beyond.
 * ls_select_exact: Desc_Sort and the loop.
 *   a_win as above; q_pos [w] int64 device memory or NULL (the last w positions), the same as was scored;
 *   vert, slash [B,Hq,n], total [B,Hq] as produced by ls_score (the lists are ordered by these weights);
 *   outputs, capacities, accounted, status bits and limits as for ls_select (shape->w is used here).
 */
int ls_score_window(ls_ctx* ctx, const ls_shape* shape, const void* q_win, const int64_t* q_pos, const void* k,
                    float* a_win, void* hip_stream);
int ls_select_exact(ls_ctx* ctx, const ls_shape* shape, float alpha, const float* a_win, const int64_t* q_pos,
                    const float* vert, const float* slash, const float* total,
                    int32_t* v_idx, int32_t* v_cnt, int32_t cap_v,
                    int32_t* s_idx, int32_t* s_cnt, int32_t cap_s,
                    float* accounted, void* hip_stream);

/*
 * ls_merge_lines -- the accumulated line set of Alg. 1 (L: the selections of every turn so far), which Sec. 5,
 * Step 1 says can be reused in later dialogue turns.  A column index is a key position and a diagonal index an
 * offset (query position - key position); neither changes when the context grows, so a selection made in an
 * earlier turn is carried into a later one as a union of index sets.  Per (batch, head): v_idx = union of the
 * column lists a and b, s_idx = union of the diagonal lists, each ascending and free of duplicates, with their
 * counts (a count above its capacity: truncated to the smallest indices, LS_STAT_S_TRUNCATED / V_TRUNCATED).
 *   shape: B, Hq and n (the context the result refers to) are used; entries outside [0, n) are dropped
 *          (LS_STAT_MERGE_RANGE).  min(cnt, cap) entries of each input list are read; inputs need not be sorted.
 *   The output lists are valid inputs of ls_sparse_prefill and of a later ls_merge_lines; an output may not
 *   alias an input.
 */
int ls_merge_lines(ls_ctx* ctx, const ls_shape* shape,
                   const int32_t* v_idx_a, const int32_t* v_cnt_a, int32_t cap_va,
                   const int32_t* s_idx_a, const int32_t* s_cnt_a, int32_t cap_sa,
                   const int32_t* v_idx_b, const int32_t* v_cnt_b, int32_t cap_vb,
                   const int32_t* s_idx_b, const int32_t* s_cnt_b, int32_t cap_sb,
                   int32_t* v_idx, int32_t* v_cnt, int32_t cap_v,
                   int32_t* s_idx, int32_t* s_cnt, int32_t cap_s, void* hip_stream);

/*
 * ls_sparse_prefill -- masked attention Softmax(QK^T/sqrt(d_k) - c(1-M)) V of Sec. 2.2 for the
 * rows of the newest turn (Sec. 5, Step 1), with M[a][b] = 1 iff b <= p_a and (b in v_idx or
 * p_a - b in s_idx), masked entries weighing exactly zero, each allowed cell counted once.
 *
 *   q [B,Hq,n_hat,d]; k, v [B,Hkv,n,d]; index lists as written by ls_select (device memory;
 *   min(cnt, cap) entries are read).  v_idx must be strictly ascending with entries in [0, n); a head
 *   whose list is not is computed without its columns and LS_STAT_V_INVALID is set.  s_idx may be in
 *   any order; entries outside [0, n) are ignored (LS_STAT_S_RANGE).
 * Outputs:
 *   out [B,Hq,n_hat,d] in dtype; a row with no allowed cell is all zeros
 *   lse [B,Hq,n_hat] fp32 or NULL: natural log of the softmax denominator (-inf for an empty row)
 * n <= LS_MAX_N.  shape->w is ignored.
 */
int ls_sparse_prefill(ls_ctx* ctx, const ls_shape* shape, const void* q, const void* k, const void* v,
                      const int32_t* v_idx, const int32_t* v_cnt, int32_t cap_v,
                      const int32_t* s_idx, const int32_t* s_cnt, int32_t cap_s,
                      void* out, float* lse, void* hip_stream);

/*
 * ls_kv_compress -- Alg. 3, the re-selection step (Sec. 5.2): for each KV head keep the `budget`
 * cache entries that receive the most attention from the last n_obs = shape->w query rows, summed
 * over the Hq/Hkv query heads of the group; ties go to the smaller index.
 *
 *   q_obs [B,Hq,n_obs,d]  queries at positions len-n_obs .. len-1 (len = shape->n)
 *   k [B,Hkv,len,d]; v [B,Hkv,len,d] or NULL when v_out is NULL
 * Outputs:
 *   keep_idx [B,Hkv,budget] int32 ascending; keep_cnt [B,Hkv] = min(budget, len)
 *   k_out, v_out [B,Hkv,budget,d] compacted copies of the kept rows, or NULL
 * len <= LS_MAX_N (LS_ESHAPE otherwise, before anything is launched).
 */
int ls_kv_compress(ls_ctx* ctx, const ls_shape* shape, int32_t budget,
                   const void* q_obs, const void* k, const void* v,
                   int32_t* keep_idx, int32_t* keep_cnt, void* k_out, void* v_out, void* hip_stream);

/*
 * ls_kv_compress_static -- ls_kv_compress for callers that cannot allocate device memory or hold a
 * context: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, outputs, limits and results as ls_kv_compress on GPU `device`, but no ls_ctx: its
 * intermediate results (softmax partials of the observation rows, the per-group score, the radix
 * histograms and counts of the top-B selection) live in a fixed block of device memory that is part of
 * the library image, ls_static_scratch_bytes() = LS_STATIC_SCRATCH_BYTES bytes on every GPU the
 * library is used on, held until the process ends.  The call allocates and frees nothing (no hipMalloc,
 * hipFree or allocating library routine) and clears what it needs with kernels of its own.
 * A shape that needs more scratch than that (its ls_workspace_bytes says how much) is refused with
 * LS_EWORKSPACE before anything is launched; ls_last_error(NULL) describes the failure.
 * All calls on one GPU share that GPU's block: calls that overlap in time on one GPU (different streams
 * or threads) race and must be ordered by the caller.
 */
#define LS_STATIC_SCRATCH_BYTES (16u << 20)
size_t ls_static_scratch_bytes(void);
int ls_kv_compress_static(int device, const ls_shape* shape, int32_t budget,
                          const void* q_obs, const void* k, const void* v,
                          int32_t* keep_idx, int32_t* keep_cnt, void* k_out, void* v_out, void* hip_stream);

/*
 * ls_decode_attend -- Alg. 3, the Decoding step (Sec. 5.2) seen from one attention layer: the newest
 * token's query attends over the entries its KV head retained at the last ls_kv_compress, followed by
 * the tokens generated since (Alg. 3 adds every generated token to the retained set); all are visible:
 *     out = softmax(scale * q [K_c; K_t]^T) [V_c; V_t].
 *
 *   shape: B, Hq, Hkv, d, dtype (LS_BF16 only), scale are used; n, n_hat, w are ignored.  Hq/Hkv <= 32.
 *   q [B,Hq,d]
 *   k_c, v_c [B,Hkv,cap,d]  retained rows (e.g. k_out / v_out of ls_kv_compress), cap >= 1
 *   cnt [B,Hkv] int32 device memory: the first cnt rows of each [cap,d] block are valid (values are
 *        clamped to [0, cap]; e.g. keep_cnt of ls_kv_compress), or NULL for all cap rows
 *   k_t, v_t [B,Hkv,T,d]    tokens since the retention, in order; T >= 0, NULL allowed when T == 0
 * Outputs:
 *   out [B,Hq,d] in dtype; all zeros when a KV head has no key at all (cnt == 0 and T == 0)
 *   lse [B,Hq] fp32 or NULL: natural log of the softmax denominator (-inf when there is no key)
 * The caller owns every tensor; the call is asynchronous on hip_stream and uses the context's
 * workspace (ls_decode_workspace_bytes).  Returns LS_ESHAPE for fp32 or Hq/Hkv > 32.
 */
int ls_decode_attend(ls_ctx* ctx, const ls_shape* shape, int32_t cap, int32_t T,
                     const void* q, const void* k_c, const void* v_c, const int32_t* cnt,
                     const void* k_t, const void* v_t, void* out, float* lse, void* hip_stream);
/* Host-only: workspace bytes ls_decode_attend needs for these sizes (0 on a bad shape). */
size_t ls_decode_workspace_bytes(const ls_shape* shape, int32_t cap, int32_t T);

/*
 * ---- Paged caches and packed sequences ---------------------------------------------------------------------------
 * The calls below serve dialogues whose keys and values live in pages and whose lengths differ within a batch: attention
 * of whole prompts packed one behind the other, rows into and out of the pages, and a token over them.
 * In the attention, logits, softmax references, normalisers and partial results are fp32; of bf16 inputs the softmax weights are rounded to bf16 for their products
 * with V, while the normaliser adds them up unrounded.  Logits may have magnitudes up to 2^30; rows of larger ones may come out as NaN or zeros.
 * A logit of -inf weighs nothing, and a row that sees no others is as one that sees no key; one of +inf makes its row NaN, as NaN does.
 */

/* Rows of `H` heads of `d` neighbouring values each, as a caller's tensor holds them.  Sequence s's row i of head h begins
 * at element s * seq + i * row + h * head of `data`; packed sequences follow each other (s * seq is left out, i counts on
 * from starts[s]).  Strides are in elements, not negative, and multiples of 16 bytes; `data` is 16-byte aligned.  Rows that a call
 * writes may not overlap. */
typedef struct {
    void* data;
    int64_t seq, row, head;
} ls_rows;

typedef enum { LS_CACHE_BF16 = 0, LS_CACHE_E4M3 = 1, LS_CACHE_E2M1 = 4 } ls_cache_type;

/* A pool of pages.  Page p holds `page` neighbouring positions of one sequence, of all KV heads: k, v [pages,Hkv,page,d],
 * contiguous, 16-byte aligned.  LS_CACHE_BF16: bf16.  LS_CACHE_E4M3: 8-bit floats (1 sign, 4 exponent, 3 fraction bits, bias 7, no
 * infinities, 0x7F and 0xFF are NaN) and, in k_exp, v_exp [pages,Hkv,page], a byte E for each row: a stored value stands
 * for code * 2^(E - 127), and for NaN where E is 255.  ls_cache_write makes E from 10 to 247, of which bf16 and fp32 hold every value exactly (but for
 * 2^128, to which magnitudes from 1.9375 * 2^127 on round: infinity).  Pages that a caller fills may have other bytes: ls_cache_read rounds their values to
 * the rows' type, ls_paged_attend rounds those of K to bf16.  A softmax weight times the power 2^(E - 127) of its row of V is a bf16 there, which has fewer bits below 2^-126.
 * LS_CACHE_E2M1: 4-bit floats (1 sign, 2 exponent, 1 fraction bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) in k, v [pages,Hkv,page,d/2], value 2 i of a row in the low half of its byte i, and in
 * k_exp, v_exp [pages,Hkv,page,d/32] a byte E for each 32 neighbouring values of a row: a stored value stands for code * 2^(E - 127), and for NaN where E is 255.  ls_cache_write makes E
 * from 2 to 253, of which bf16 and fp32 hold every value exactly (but for 2^128 and 1.5 * 2^128: infinity), and 255.  ls_paged_attend rounds the values of K and of V to bf16.
 * Where a sequence's pages are is a row of `table` [B,max_pages] int32, device memory: positions p * page .. of sequence b lie in
 * page table[b][p].  Several sequences may share pages that are read.  A page number outside [0, pages), and a position beyond max_pages * page, is nowhere:
 * rows of it are neither written nor read, keys of it are not seen, and LS_STAT_PAGE_RANGE is set. */
typedef struct {
    int32_t Hkv, d;          /* d in {64, 128} */
    int32_t page;            /* positions of a page: 16, 32, 64, 128 or 256 */
    int32_t type;            /* ls_cache_type */
    int64_t pages;           /* 1 <= pages < 2^31 */
    void *k, *v;
    uint8_t *k_exp, *v_exp;  /* not for LS_CACHE_BF16 */
} ls_cache;

/*
 * ls_packed_prefill -- causal attention of whole prompts, or of the new rows of later turns, without a selection of lines
 * (Sec. 2.2 with M[a][b] = 1 iff b <= p_a), for sequences of different lengths:
 *     out[a] = sum_b softmax_b(scale * <q_a, k_b>) v_b.
 *
 *   shape: B sequences, Hq, Hkv, d, dtype, scale.  n >= 1: rows of k and v, n_hat >= 1: rows of q and out.  w is ignored.  Blocks of 128 rows (a query of a query head is
 *        a row), one more for each sequence where they are packed, are at most 2^24 - 8 of all KV heads, and neighbouring rows of k and of v begin less than 64 MiB apart.
 *   q_starts, k_starts [B+1] int32, device memory: rows q_starts[s] .. q_starts[s+1] - 1 are sequence s's queries, likewise its
 *        keys; n and n_hat count all sequences' rows then.  Both NULL: every sequence has n keys and n_hat queries.
 *   The queries are the last positions of their sequence: query i of m sees the keys up to (keys of the sequence) - m + i,
 *        none where that is negative.  A sequence whose starts descend or leave [0, n] or [0, n_hat] is passed by, with
 *        all behind it (LS_STAT_STARTS).
 * Outputs:
 *   out in dtype; a row that sees no key is all zeros, and one that sees a NaN logit is NaN, with its lse.  Rows of no sequence stay as they are.
 *   lse fp32 or NULL, [Hq,n_hat] (packed) or [B,Hq,n_hat]: natural log of the softmax denominator (-inf without a key)
 * Workspace: ls_packed_workspace_bytes (0 for an invalid shape); less is enough where the rows fill the chip, and slower elsewhere.
 * Few rows on many keys are fast for up to 64 sequences, whose keys are then shared out among workgroups; of more, each workgroup has whole blocks of rows, and the call takes as long
 * as the longest of them.
 */
int ls_packed_prefill(ls_ctx* ctx, const ls_shape* shape, const ls_rows* q, const ls_rows* k, const ls_rows* v,
                      const int32_t* q_starts, const int32_t* k_starts, const ls_rows* out, float* lse, void* hip_stream);
size_t ls_packed_workspace_bytes(const ls_shape* shape);

/*
 * ls_cache_write -- rows of K and V into the pages of their sequences; ls_cache_read -- the way back, in order, for the calls
 * that take whole contexts (ls_score, ls_sparse_prefill, ls_kv_compress).
 *
 *   shape: B sequences, Hkv and d of the cache, dtype of the rows (LS_BF16 or LS_F32).  n_hat: rows of k and of v.  Hq, n, w, scale
 *        are ignored.
 *   starts [B+1] int32, device memory: rows starts[s] .. starts[s+1] - 1 are sequence s's (n_hat counts all rows); a sequence whose
 *        starts descend or leave [0, n_hat] is passed by, with all behind it (LS_STAT_STARTS).  NULL: each sequence has n_hat rows of its own.
 *   count [B] int32, device memory: only the first count[s] of them (clamped to [0, n_hat]); NULL: all.  Not with starts.
 *   pos [B] int32, device memory: the position in the cache at which sequence s's rows begin; NULL: 0.
 * ls_cache_write: bf16 pages hold the rows rounded to nearest even.  E4M3: E is the smallest byte from 10 to 247 with
 *   max |x| <= 448 * 2^(E-127) over the row's finite values, the codes are x * 2^(127-E) rounded to nearest even; infinities and
 *   NaN become NaN.  E2M1: of each 32 values E is the smallest byte from 2 to 253 with max |x| <= 7 * 2^(E-127), the codes are x * 2^(127-E) rounded to the nearest, ties to the one with fraction bit 0, what is
 *   beyond 6 to 6; 32 values with an infinity or NaN among them become NaN: E is 255 and the codes are 0.  What else is in the pages stays.  Of rows that meet in one place (a page that is twice in the table), each value there is one of theirs, and
 *   a byte E may be another row's than its codes.
 * ls_cache_read: rows past count and rows that are nowhere stay as they are.
 * No workspace.
 */
int ls_cache_write(ls_ctx* ctx, const ls_shape* shape, const ls_cache* cache, const ls_rows* k, const ls_rows* v,
                   const int32_t* starts, const int32_t* count, const int32_t* table, int32_t max_pages,
                   const int32_t* pos, void* hip_stream);
int ls_cache_read(ls_ctx* ctx, const ls_shape* shape, const ls_cache* cache, const ls_rows* k, const ls_rows* v,
                  const int32_t* starts, const int32_t* count, const int32_t* table, int32_t max_pages,
                  const int32_t* pos, void* hip_stream);

/*
 * ls_cache_resize -- sequences that grow and shrink: pages for them from a ring of free ones and back to it, and for the rows that a step adds what the other calls
 * take.  Once a step, for all layers whose pools are alike (they share the table).
 *
 *   shape: B sequences, Hkv and d of the cache, B * Hkv <= 65535 (as every call on pages has it), a dtype; n_hat >= 1: rows that positions and slots have room for, in all or of each
 *        sequence.  Hq, n, w, scale are ignored, and it makes no difference which dtype it is.
 *   cache: of which `page` and `pages` are used; it has to be one that the other calls take (its type, sizes and addresses are checked as theirs)
 *   free_pages [pages] int32, state [2] int32: a ring.  The numbers of the free pages are its `state[1]` entries from entry state[0] on, and behind the last entry comes
 *        the first.  (In the beginning: 0 .. pages - 1, and {0, pages}.)
 *   len [B] int32: positions that each sequence has; add [B] int32: by how many it grows, or, negative, shrinks (to none at least)
 *   Sequences that grow take the pages that they have none for from the front of the ring, in order of the sequences; table entries of what they have stay.  One that asks
 *   for more than the ring holds besides what all before it ask for does not grow (LS_STAT_PAGES_OUT), nor one that would be longer than max_pages pages or 2^31 - 1
 *   (LS_STAT_PAGE_RANGE).  Sequences that shrink give the pages that they no longer need to the back of the ring, in order, for calls to come; their table entries stay, and mean nothing.
 *   A length outside [0, max_pages * page] stays as it is, likewise a ring that does not have that many (it holds no page then, and pages that it has no room for are lost; LS_STAT_PAGE_RANGE).
 *   Pages that several sequences share are each sequence's here: give them back once.
 * Outputs (device memory; new_len and new_state may be len and state themselves, and no output overlaps anything else):
 *   new_len [B], new_state [2], table, free_pages
 *   starts [B+1] int32: the rows of the step, packed: sequence b adds rows starts[b] .. starts[b+1] - 1, add[b] of them where that is positive (also where it
 *        does not grow).  A sequence whose rows go beyond n_hat has none and does not grow, like all behind it (LS_STAT_STARTS).
 *        NULL: each sequence has n_hat rows of its own, of which it adds the first add[b]; one that would add more does not grow (LS_STAT_STARTS).
 *   positions int32, slots int64 ([n_hat], without starts [B,n_hat]), or NULL: of each row its position, and page * (positions of a page) + place in it, as
 *        ls_norm_rotate takes them; 0 and -1 of rows whose sequence does not grow, that it does not add, and behind the last sequence
 * No workspace.
 */
int ls_cache_resize(ls_ctx* ctx, const ls_shape* shape, const ls_cache* cache, int32_t* free_pages, const int32_t* state, int32_t* new_state,
                    const int32_t* add, const int32_t* len, int32_t* new_len, int32_t* table, int32_t max_pages,
                    int32_t* starts, int32_t* positions, int64_t* slots, void* hip_stream);

/* The norms and the rotation that ls_norm_rotate gives queries and keys.  Device memory, fp32, 16-byte aligned. */
typedef enum { LS_PAIRS_HALVES = 0, LS_PAIRS_NEIGHBOURS = 1 } ls_pairs;
typedef struct {
    const float* freq;                   /* [dims/2] radians a position; NULL allowed when dims == 0 */
    const float *q_weight, *k_weight;    /* [d], or NULL: that tensor's rows are not normed */
    int32_t dims;                        /* the first `dims` values of a row are rotated: a multiple of 16, at most d */
    int32_t pairs;                       /* ls_pairs: value i with value i + dims/2, or values 2 i and 2 i + 1 */
    float eps;                           /* >= 0 */
} ls_rotation;

/*
 * ls_norm_rotate -- what q and k are given between their projection and the attention, in one pass: each head's row becomes
 *     y = x / sqrt(mean(x^2) + eps) * weight,
 * and of its first `dims` values each pair (a, b) number i is turned by t = position * freq[i]: (a cos t - b sin t, b cos t + a sin t).
 *
 *   shape: Hq, Hkv, d, dtype, n_hat; B sequences of n_hat rows each (packed sequences, however many, are one: B = 1).  n, w, scale are ignored.
 *   q [Hq], k [Hkv heads] as ls_rows;  positions [B,n_hat] int32, device memory, or NULL: row i of a sequence is at position i
 * Outputs:
 *   q_out as ls_rows; k_out as ls_rows, or NULL where keys go into a cache only.  They may be q and k themselves (the same strides), and overlap nothing else that is read.
 *   cache, v, slots (together, or all NULL): the keys, rounded to dtype, and the rows of v as they are go into the cache's pages as ls_cache_write has it: row i to slot
 *        slots[i] = page * (positions of a page) + place in it ([B,n_hat] int64, device memory, e.g. of ls_cache_resize).  A negative slot is nowhere; one beyond the pool
 *        too, with LS_STAT_PAGE_RANGE.  Of rows with one slot, each value there is one of theirs.
 * Sums are fp32, or 64 bits where squares leave its range; the angle is formed in 64 bits (up to |t| = 2^31 its sine and cosine are off by no more than 2^-21), and results are rounded once.
 * No workspace.
 */
int ls_norm_rotate(ls_ctx* ctx, const ls_shape* shape, const ls_rotation* rotation, const ls_rows* q, const ls_rows* k,
                   const int32_t* positions, const ls_rows* q_out, const ls_rows* k_out,
                   const ls_cache* cache, const ls_rows* v, const int64_t* slots, void* hip_stream);

/*
 * ls_paged_attend -- ls_decode_attend over pages: the newest token's query of each sequence attends over the first len[b]
 * positions of its cache.
 *
 *   shape: B, Hq, Hkv, d, scale, dtype (LS_BF16 only); n: no sequence is longer (lengths are clamped to [0, min(n, max_pages *
 *        page)], with LS_STAT_PAGE_RANGE where that is less than len).  n_hat, w are ignored.  Hq/Hkv <= 32.
 *   q [B,Hq,d];  table [B,max_pages], len [B] int32, device memory
 * Outputs:
 *   out [B,Hq,d] in dtype; all zeros where there is no key, NaN (and so the lse) where a logit is
 *   lse [B,Hq] fp32 or NULL: natural log of the softmax denominator (-inf when there is no key)
 * Workspace: ls_paged_workspace_bytes (0 for an invalid shape), of which LS_CACHE_E2M1 pages alone need the last 8 bytes a sequence and KV head (rounded up to 256 in all).
 * What this header says of calls of ls_decode_attend that overlap holds for these too: they share its counters.
 */
int ls_paged_attend(ls_ctx* ctx, const ls_shape* shape, const ls_cache* cache, const void* q,
                    const int32_t* table, int32_t max_pages, const int32_t* len, void* out, float* lse, void* hip_stream);
size_t ls_paged_workspace_bytes(const ls_shape* shape);

/*
 * Timing of the sparse attention itself (the dominant part of ls_sparse_prefill), for roofline
 * reports.  After ls_profile_enable(ctx, 1) every ls_sparse_prefill call attaches a pair of HIP
 * events to the launch of the attention kernel and, where long row blocks may have been cut into
 * parts, another to the launch that puts the parts' results together: they receive the start and
 * stop time of the dispatches themselves, and no marker is put into the stream (this creates events
 * on every call, so leave it off in allocation-free loops).  ls_profile_prefill_kernel_ms waits for the
 * recorded events and returns the mean of a call's kernel time (the sum of the two) in milliseconds
 * and the number of calls seen since profiling was enabled.  ls_profile_enable(ctx, 0) stops recording and drops the events.
 */
int ls_profile_enable(ls_ctx* ctx, int on);
int ls_profile_prefill_kernel_ms(ls_ctx* ctx, double* mean_ms, int32_t* launches);

/*
 * Device status word.  Conditions that a kernel can only see while it runs are reported without a
 * host round trip: the kernel ORs a bit into a word in device memory that belongs to the context, the
 * call still returns LS_OK, and the outputs are as described for each bit.  ls_poll_status waits for
 * everything queued on `hip_stream`, writes the word to *host_out (host memory) and clears it; it is
 * the one call here that synchronises with the host.  (Serves callers of the four entry points above;
 * no passage of the paper defines it.)
 */
#define LS_STAT_WALK_TIMEOUT 1  /* ls_select: a bounded wait inside the greedy loop gave up; the head concerned reports
                                   every line selected (v_cnt = s_cnt = n), which still meets the coverage target */
#define LS_STAT_S_TRUNCATED  2  /* ls_select: s_cnt > cap_s for some head (s_idx holds the smallest cap_s indices) */
#define LS_STAT_V_TRUNCATED  4  /* ls_select: v_cnt > cap_v for some head */
#define LS_STAT_S_RANGE      8  /* ls_sparse_prefill: s_idx entries outside [0, n) were ignored */
#define LS_STAT_V_INVALID   16  /* ls_sparse_prefill: a head's v_idx was not strictly ascending inside [0, n); that
                                   head's columns were ignored (its diagonals still apply) */
#define LS_STAT_MERGE_RANGE 32  /* ls_merge_lines: input entries outside [0, n) were dropped */
#define LS_STAT_PAGE_RANGE  64  /* ls_cache_write, ls_cache_read, ls_norm_rotate, ls_paged_attend: a position lies in no page of the pool or beyond
                                   the table; it was left out.  ls_cache_resize: so would a sequence's, or its length or the ring is none */
#define LS_STAT_STARTS     128  /* ls_packed_prefill, ls_cache_write, ls_cache_read: a sequence's starts descend or leave the rows;
                                   it was passed by, with all behind it.  ls_cache_resize: its rows have no room */
#define LS_STAT_PAGES_OUT  256  /* ls_cache_resize: a sequence did not grow, for want of free pages */
int ls_poll_status(ls_ctx* ctx, int32_t* host_out, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* LOOPSERVE_H */
