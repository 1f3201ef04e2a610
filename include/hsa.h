/*
 * hsa.h -- C ABI of libhsa, the GB300 (sm_103a) hot path of Heterogeneous Step
 * Allocation (HSA), a training-free step-skipping scheme for video diffusion
 * transformers (arXiv 2605.06892).
 *
 * One denoising iteration i of an HSA layer runs, in order:
 *   hsa_partition_active   active set A_i from the token groups     (Sec. 2.2, 2.5)
 *   hsa_gather_active      rows of A_i entering the block            (Sec. 2.3, step 1)
 *   hsa_kv_sync_scatter    fresh K/V of A_i into the layer's cache   (Sec. 2.3, step 2)
 *   hsa_active_attention   |A_i| queries against all N cached keys   (Sec. 2.3, step 3)
 *   hsa_cached_euler       all N latents advanced by one Euler step  (Sec. 2.4, Eq. 6)
 * and, once per sample, hsa_partition assigns tokens to step-budget groups
 * from a per-token statistic (Sec. 2.2 Eq. 3, Eq. 5; App. B, Eq. 7).
 *
 * Conventions for every call below:
 *  - Pointers named as device pointers must be device (or managed) memory of
 *    the current CUDA device; the caller owns all memory.  Host pointers are
 *    read before the call returns.  The library allocates nothing.
 *  - Work is enqueued on `stream` (NULL = the legacy default stream) and the
 *    call returns without waiting for it.  Argument checks happen on the host
 *    before any launch; a failed check launches nothing.
 *  - Errors that only the GPU can see (an index out of range, a non-finite
 *    statistic, a pipeline wait that ran out) do not fault the GPU: the kernel
 *    skips the offending access, records the error in a per-device word, and
 *    hsa_get_device_error() reports it.
 *  - Return values are hsa_status codes (0 = success, negative = error), or a
 *    documented non-negative count.
 *  - Token tensors are row-major with the token index outermost: a [N, H, D]
 *    tensor stores element (n, h, d) at offset (n*H + h)*D + d.
 */
#ifndef HSA_H
#define HSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Same type as cudaStream_t. */
struct CUstream_st;
typedef struct CUstream_st *hsa_stream_t;

typedef enum {
    HSA_BF16 = 0,   /* bfloat16 storage, fp32 accumulation */
    HSA_F32 = 1,    /* fp32 storage and arithmetic */
    HSA_E4M3 = 2    /* 8-bit KV cache: e4m3 codes with one power of two per row; only where
                       a call names it */
} hsa_dtype;

typedef enum {
    HSA_OK = 0,
    HSA_ERR_INVALID_ARG = -1,   /* null pointer, bad size, misaligned pointer */
    HSA_ERR_NOT_DIVISOR = -2,   /* a step budget does not divide T (Eq. 5) */
    HSA_ERR_BAD_COUNTS = -3,    /* group sizes negative or not summing to N */
    HSA_ERR_UNSUPPORTED = -4,   /* shape outside the supported set */
    HSA_ERR_NONFINITE = -5,     /* NaN or infinite statistic (device-side) */
    HSA_ERR_INDEX = -6,         /* index or group id out of range (device-side) */
    HSA_ERR_TIMEOUT = -7,       /* a bounded pipeline wait ran out (device-side) */
    HSA_ERR_CUDA = -8,          /* a CUDA runtime call or launch failed */
    HSA_ERR_WORKSPACE = -9      /* workspace missing, too small or misaligned */
} hsa_status;

/* Static string for a status code. */
const char *hsa_status_string(int status);

/* Library ABI version, currently 1. */
int hsa_version(void);

/* ------------------------------------------------------------ host helpers */

/* Checks step budgets and group sizes against Sec. 2.2: budgets[0] == T (the
 * baseline group G_1), budgets non-increasing, each a positive divisor of T
 * (Eq. 5); counts[k] >= 0 with sum N (counts may be NULL to skip that part).
 * Host only.  Returns HSA_OK, HSA_ERR_INVALID_ARG, HSA_ERR_NOT_DIVISOR or
 * HSA_ERR_BAD_COUNTS. */
int hsa_check_budgets(int T, const int *budgets, const int *counts, int K, int N);

/* Margin m = floor((1 - k) T / 2) of the phase-aware caching window (Sec. 2.5)
 * for k = window_pct / 100, in integer arithmetic.  Iterations i < m and
 * i > T - m - 1 run every token.  Returns m, or HSA_ERR_INVALID_ARG when
 * window_pct is outside [0, 100] or T < 1.  Host only. */
int hsa_window_margin(int T, int window_pct);

/* |A_i| from the group sizes: the sum of counts[k] over the groups active at
 * iteration iter (group k is active iff iter mod (T / budgets[k]) == 0, or
 * iter lies outside the caching window).  Host only, no device access, so a
 * caller can size buffers without synchronising.  Negative on bad input. */
int hsa_active_count(const int *budgets, const int *counts, int K, int T,
                     int iter, int window_pct);

/* Noise levels sigma_0 = 1 > sigma_1 > ... > sigma_T = 0 of the Euler solver
 * (Sec. 2.1, Eq. 2), computed in fp64 into the host array sigma[T + 1]:
 * t_i = 1 - i/T and sigma_i = shift*t_i / (1 + (shift - 1) t_i); shift = 1
 * gives the linear schedule.  The step of iteration i is sigma_{i+1} - sigma_i
 * (negative).  Host only. */
int hsa_sigma_schedule(int T, double shift, double *sigma);

/* ------------------------------------------------------------- a1 partition */

/* Bytes of device workspace hsa_partition needs for N tokens (0 for N == 0). */
size_t hsa_partition_workspace_bytes(int N);

/* Token partition (Sec. 2.2 Eq. 3) by the dynamic selection rule (App. B,
 * Eq. 7): tokens are ranked by stat ascending, ties broken by the lower token
 * index (-0 and +0 are equal); the counts[K-1] lowest go to group K-1 (the
 * smallest budget), the next counts[K-2] to group K-2, ..., the counts[0]
 * highest to group 0, the baseline group with budgets[0] == T.
 *   stat       device, fp32 [N]: per-token statistic (e.g. the mean L1
 *              relative change of the velocity, Eq. 7, or any score).
 *   budgets,   host, int [K]: step budget s_k and size |G_k| of each group,
 *   counts     checked as hsa_check_budgets does; 1 <= K <= 32.
 *   group_of   device, int32 [N], written: group id in [0, K) per token.
 *   workspace  device, >= hsa_partition_workspace_bytes(N) bytes, 256-byte
 *              aligned; overwritten.  Must not overlap stat or group_of.
 * A NaN or infinite statistic is reported as HSA_ERR_NONFINITE by
 * hsa_get_device_error; group_of is then unspecified. */
int hsa_partition(const float *stat, int N, int T, const int *budgets,
                  const int *counts, int K, int32_t *group_of, void *workspace,
                  size_t workspace_bytes, hsa_stream_t stream);

/* Largest N accepted by hsa_partition_static. */
#define HSA_PARTITION_STATIC_MAX_TOKENS 524288

/* hsa_partition without a workspace argument, for callers that cannot
 * allocate device memory for one: a plugin inside a host framework that owns
 * all device memory and offers it no allocator, or a latency-critical loop
 * that must not call cudaMalloc/cudaFree (they may synchronise the device).
 * The paper has no counterpart; the ranking and group assignment are exactly
 * those of hsa_partition (same arguments, same results).
 * Scratch: a fixed device array inside the library, about 8.5 MB, sized for
 * N <= HSA_PARTITION_STATIC_MAX_TOKENS (the sort that partitions layers of more
 * than 360448 tokens uses it; smaller layers take paths that need no scratch);
 * every GPU that loads the library's
 * partition module holds it until the process exits.  The CUDA runtime
 * reserves it when that module is loaded on a device: when the library is
 * loaded if CUDA_MODULE_LOADING=EAGER, otherwise (lazy loading, the default)
 * at the first partition call or symbol query on that device.  A host
 * framework that claims all device memory up front should therefore make one
 * call early, before it does.  Larger N returns HSA_ERR_UNSUPPORTED before any
 * launch.  Nothing is allocated: no cudaMalloc, cudaFree or allocating
 * library call is made.
 * The first call on a device looks up the array's device address (a CUDA
 * runtime query) for that device, so make that first call before any stream
 * capture.  Every call on a device shares the one array and finds the last
 * call's contents there (none need to start at zero); calls whose work
 * overlaps on the GPU (other streams, or other host threads) race on it and
 * must be serialised by the caller. */
int hsa_partition_static(const float *stat, int N, int T, const int *budgets,
                         const int *counts, int K, int32_t *group_of,
                         hsa_stream_t stream);

/* Statistics for the other token allocation strategies of App. B, to be
 * ranked by hsa_partition (the random strategy R ranks any random statistic
 * the caller draws):
 *  - uniform allocation (U): stat[n] = top 24 bits of (n+1) * 2654435769 mod
 *    2^32 (golden-ratio sequence), an exact integer in fp32.  Each group then
 *    holds the tokens of one interval of the sequence, which are spaced by at
 *    most three distinct gaps over the whole token range ("maximally spread").
 *  - first-frame reservation (F): stat[n] = FLT_MAX for n < frame_tokens (the
 *    first latent frame, (H_l/2)*(W_l/2) tokens in row-major order), applied
 *    on top of a random statistic; with counts[0] >= frame_tokens every
 *    first-frame token lands in the baseline group.
 *   stat  device, fp32 [N], written (U) or updated in place (F). */
int hsa_uniform_stat(float *stat, int N, hsa_stream_t stream);
int hsa_reserve_first_frame(float *stat, int N, int frame_tokens, hsa_stream_t stream);

/* Token reordering (Sec. 2.5), applied once before the denoising loop: new
 * position r holds old token order[r]; the tokens of groups 1..K-1 come first
 * in token order, then the n_baseline tokens of the baseline group (group 0),
 * also in token order.  The KV cache then only needs the prefix of
 * M = N - n_baseline rows, because the baseline group is active at every
 * iteration (see hsa_active_attention_prefix).
 *   group_of   device, int32 [N]; exactly n_baseline entries are 0.
 *   order      device, int32 [N], written (new -> old).  Reorder a per-token
 *              tensor with hsa_gather_active(src, .., order, N, dst).
 *   where      device, int32 [N] or NULL, written (old -> new); undo the
 *              reordering with hsa_gather_active(.., where, N, ..).
 *   group_new  device, int32 [N] or NULL, written: group_of[order[r]].
 * None of the three may overlap group_of.
 * A group_of that disagrees with n_baseline is reported as HSA_ERR_INDEX. */
int hsa_reorder_tokens(const int32_t *group_of, int N, int n_baseline, int32_t *order,
                       int32_t *where, int32_t *group_new, hsa_stream_t stream);

/* ---------------------------------------------------- a2 active set per step */

/* Active set A_i (Sec. 2.3; Fig. 1): token n is active at iteration iter iff
 * iter mod (T / budgets[group_of[n]]) == 0 (Sec. 2.2) or iter is outside the
 * caching window of window_pct percent (Sec. 2.5; 100 = no window).
 *   group_of  device, int32 [N] in [0, K).
 *   idx       device, int32 [>= |A_i|], written: active token ids ascending.
 *   pos       device, int32 [N] or NULL, written: rank of n in idx, or -1.
 * idx and pos must not overlap group_of.
 * |A_i| is hsa_active_count(...) of the same groups, known on the host.  A
 * group id outside [0, K) is reported as HSA_ERR_INDEX (that token is then
 * treated as skipped). */
int hsa_partition_active(const int32_t *group_of, int N, int T,
                         const int *budgets, int K, int iter, int window_pct,
                         int32_t *idx, int32_t *pos, hsa_stream_t stream);

/* --------------------------------------------------------------- a3 gather */

/* dst[j, :] = src[idx[j], :] for j < n_active: the rows of the active tokens
 * that enter the transformer block (Sec. 2.3, step 1).
 *   src       device, [N, row_bytes] (any element type).
 *   row_bytes row size in bytes, a positive multiple of 16; src and dst
 *             16-byte aligned.
 *   idx       device, int32 [n_active], values in [0, N).
 *   dst       device, [n_active, row_bytes], written.
 * An index outside [0, N) leaves its dst row untouched (HSA_ERR_INDEX). */
int hsa_gather_active(const void *src, size_t row_bytes, int N,
                      const int32_t *idx, int n_active, void *dst,
                      hsa_stream_t stream);

/* ------------------------------------------------------ a4 KV-cache scatter */

/* KV-cache synchronisation (Sec. 2.3, step 2): k_cache[idx[j]] = k_fresh[j]
 * and v_cache[idx[j]] = v_fresh[j] for j < n_active, one launch for both;
 * rows of skipped tokens are left untouched.
 *   k_cache, v_cache  device, [N, H, D] of dtype, updated in place.
 *   k_fresh, v_fresh  device, [n_active, H, D] of dtype (K/V of A_i).
 *   idx               device, int32 [n_active], distinct values in [0, N)
 *                     (A_i never repeats a token; repeated ids race, and
 *                     hsa_check_indices detects them).
 * H*D*sizeof(dtype) must be a multiple of 16 bytes and every pointer 16-byte
 * aligned.  An index outside [0, N) skips its row (HSA_ERR_INDEX). */
int hsa_kv_sync_scatter(void *k_cache, void *v_cache, const void *k_fresh,
                        const void *v_fresh, const int32_t *idx, int n_active,
                        int N, int H, int D, hsa_dtype dtype,
                        hsa_stream_t stream);

/* Opt-in check of an index array, for debugging (Sec. 2.2: the groups are
 * disjoint, so an active set never names a token twice, and the KV scatter
 * above relies on that).  Reports HSA_ERR_INDEX through hsa_get_device_error
 * when an entry of idx lies outside [0, N) or a value appears more than once;
 * the hot-path calls do not make this check themselves.
 *   idx        device, int32 [n], any order.
 *   workspace  device, >= hsa_check_indices_workspace_bytes(N) bytes (one
 *              bit per token), 256-byte aligned; overwritten.  Calls sharing
 *              one workspace must not overlap on the GPU.
 * Two launches (clear the bitmap, then mark); returns HSA_ERR_WORKSPACE when
 * the workspace is missing, too small or misaligned. */
size_t hsa_check_indices_workspace_bytes(int N);
int hsa_check_indices(const int32_t *idx, int n, int N, void *workspace,
                      size_t workspace_bytes, hsa_stream_t stream);

/* Rotary position embedding of the active rows (Sec. 2.3: the positional
 * frequencies are subsampled to match A_i).  The table holds, for every token
 * n of the grid and rotation pair i, (cos, sin) of its angle; the calls below
 * rotate an active row j by the table row of its token idx[j], pair (x0, x1)
 * of each head becoming (fma(x0, c, -(x1 s)), fma(x0, s, x1 c)) in fp32,
 * rounded to bf16.
 *
 * hsa_rope_table: host-side table of a (F, Hh, Ww) grid, tokens row-major:
 * the D/2 pairs form three bands, p_t = D/2 - 2 floor(D/6) pairs for the
 * frame, then floor(D/6) each for the row and the column; pair i of a band
 * of p pairs turns by pos * theta^(-i/p).  table: host, fp32 [N, D/2, 2]
 * written (fp64 math, rounded once).  D a multiple of 8.
 *
 * hsa_rope_rows: x device bf16 [n, H, D], rotated in place (e.g. Q[A_i]).
 * hsa_kv_sync_scatter_rope: hsa_kv_sync_scatter (bf16) with the fresh K rows
 * rotated on their way into the cache; V is copied unchanged.
 *   table  device, fp32 [N, D/2, 2], 16-byte aligned.
 * An idx entry outside [0, N) skips its row (HSA_ERR_INDEX). */
int hsa_rope_table(int F, int Hh, int Ww, int D, double theta, float *table);
int hsa_rope_rows(void *x, const int32_t *idx, int n, int H, int D, const float *table, int N,
                  hsa_stream_t stream);
int hsa_kv_sync_scatter_rope(void *k_cache, void *v_cache, const void *k_fresh,
                             const void *v_fresh, const int32_t *idx, int n_active, int N,
                             int H, int D, const float *table, hsa_stream_t stream);

/* -------------------------------------------------- a5 active attention */

/* Full-context attention of the active queries (Sec. 2.3, step 3; Sec. 2.1
 * "Self-attention"), per head h and active row j:
 *   out[j, h, :] = sum_n softmax_n(scale * <q_{r,h}, k_{n,h}>) v_{n,h}
 * over all N cached keys, with r = q_idx[j] when q_idx is given (q is then
 * [N, H, D] and rows are read by index) or r = j (q is compact
 * [n_active, H, D]).  No mask; scale <= 0 selects 1/sqrt(D).  The cost is
 * O(|A_i| N) instead of O(N^2).
 *   k_cache, v_cache  device, [N, H, D] of dtype.
 *   out               device, [n_active, H, D] of dtype, written.
 *   workspace         device, optional (NULL = none), 16-byte aligned; see
 *                     hsa_active_attention_workspace_bytes.  With it, the
 *                     (query block, head) units of the last, partly filled
 *                     wave of CTAs are split along the keys and merged
 *                     afterwards, so that the last wave finishes sooner;
 *                     without it the result is the same up to rounding order.
 *                     Overwritten; calls using one workspace must not overlap.
 * Supported: D in {64, 128}; H >= 1; 1 <= N < 2^31; 0 <= n_active.
 * HSA_BF16 runs on the tensor cores (tcgen05, fp32 accumulation); HSA_F32
 * runs in fp32 on the CUDA cores and ignores the workspace.  Pointers must be
 * 16-byte aligned.  A q_idx entry outside [0, N) yields a zero query row
 * (HSA_ERR_INDEX). */
int hsa_active_attention(const void *q, const int32_t *q_idx, int n_active,
                         const void *k_cache, const void *v_cache, int N, int H,
                         int D, float scale, void *out, hsa_dtype dtype,
                         void *workspace, size_t workspace_bytes,
                         hsa_stream_t stream);

/* hsa_active_attention over keys held in two sources, read in order: the M
 * rows of k_cache / v_cache ([M, H, D], the cache of the non-baseline prefix
 * after token reordering, Sec. 2.5) followed by the B rows of k_base /
 * v_base ([B, H, D], the fresh K/V of the baseline group, which is active at
 * every iteration).  Keys total M + B >= 1; either source may be empty.
 * q_idx, when given, indexes a [M + B, H, D] query tensor.  Everything else
 * as hsa_active_attention (which is this call with B = 0). */
int hsa_active_attention_prefix(const void *q, const int32_t *q_idx, int n_active,
                                const void *k_cache, const void *v_cache, int M,
                                const void *k_base, const void *v_base, int B, int H, int D,
                                float scale, void *out, hsa_dtype dtype, void *workspace,
                                size_t workspace_bytes, hsa_stream_t stream);

/* Workspace bytes that let hsa_active_attention balance its last wave (0 when
 * the dtype or shape takes none).  Depends only on the device's SM count and
 * D, so one buffer serves every call of a given D on that device. */
size_t hsa_active_attention_workspace_bytes(int n_active, int N, int H, int D,
                                            hsa_dtype dtype);

/* ------------------------------------------------- the KV cache in 8 bits */

/* A KV cache of N rows of H heads x D values in half the bytes of bf16.  The row of
 * one token and head is held as D e4m3 codes (OCP 8-bit floating point, 4 exponent
 * and 3 fraction bits) and one scale byte s, and stands for code * 2^(s - 127):
 *   codes   [N, H, D], one byte each;   scales  [N, H], one byte each.
 * Written from values x: with a the largest |x_d| of the row, e is the least integer
 * with a * 2^-e <= 448, at least -100; s = e + 127 and the codes are x * 2^-e rounded
 * to nearest, ties to even.  The values held are exact in bf16 and fp32.  A magnitude
 * above 1.875 * 2^127 counts as that.  A NaN or infinite element is stored as NaN and
 * reported (HSA_ERR_NONFINITE); its row goes by the largest finite element.
 *
 * hsa_kv_quant_scatter: the KV-cache synchronisation (Sec. 2.3, step 2; see
 * hsa_kv_sync_scatter) into an 8-bit cache: row idx[j] of the caches takes fresh
 * row j, one launch for K and V.
 *   k_cache, v_cache  device, codes [N, H, D], updated in place.
 *   k_scale, v_scale  device, scales [N, H], updated in place (any alignment).
 *   k_fresh, v_fresh  device, [n_active, H, D] of dtype (HSA_BF16 or HSA_F32).
 *   idx               device, int32 [n_active], distinct values in [0, N).  For a
 *                     cache in pages [n_pages, page, H, D] that is N = n_pages * page
 *                     rows, idx[j] = page id * page + place in the page.
 *   table             device, fp32 [table_rows, D/2, 2] or NULL: K is first rotated
 *                     as hsa_rope_rows does (HSA_BF16 only), fresh row j by table row
 *                     table_idx[j], or idx[j] where table_idx is NULL.  The cache then
 *                     holds what hsa_kv_sync_scatter_rope would have written, in 8
 *                     bits.  table_idx needs a table.
 * An idx entry outside [0, N), or a table row outside [0, table_rows), skips its row
 * (HSA_ERR_INDEX).
 *
 * hsa_kv_dequant_gather: rows idx[j] of the cache (rows 0 .. n-1 where idx is NULL,
 * n <= N) as [n, H, D] of dtype (HSA_BF16 or HSA_F32), for the attention calls below;
 * one bf16 buffer of a layer's size then serves every layer.  An idx entry outside
 * [0, N) leaves its output rows untouched (HSA_ERR_INDEX).
 *
 * Both: D a multiple of 8 up to 256, H <= 2^24, n * H < 2^31, pointers but the scales
 * 16-byte aligned. */
int hsa_kv_quant_scatter(void *k_cache, void *v_cache, uint8_t *k_scale, uint8_t *v_scale,
                         const void *k_fresh, const void *v_fresh, const int32_t *idx,
                         int n_active, int N, int H, int D, hsa_dtype dtype,
                         const float *table, const int32_t *table_idx, int table_rows,
                         hsa_stream_t stream);
int hsa_kv_dequant_gather(const void *k_cache, const void *v_cache, const uint8_t *k_scale,
                          const uint8_t *v_scale, const int32_t *idx, int n, int N, int H,
                          int D, void *k_out, void *v_out, hsa_dtype dtype,
                          hsa_stream_t stream);

/* ------------------------------- attention over paged caches, packed prompts */

/* Attention of the n_new newest tokens of each of `batch` sequences over caches held
 * in pages, with grouped heads: query head h reads K/V head h / (Hq / Hkv), and
 *   out[b, i, h, :] = sum_j softmax_j(scale * <q[b,i,h], k_j>) v_j
 * over the keys j < seq_lens[b] - n_new + i + 1 of sequence b (so the newest tokens
 * are causal among themselves; their K/V are in the cache already).  A row without
 * keys is zero.  scale <= 0 selects 1/sqrt(D).
 *   q            device, bf16 [batch, n_new, Hq, D].
 *   k_pages,     device, [n_pages, page_size, Hkv, D] of cache_dtype: HSA_BF16, or
 *   v_pages      HSA_E4M3 as hsa_kv_quant_scatter writes it, with
 *   k_scale,     device, scales [n_pages, page_size, Hkv] (HSA_E4M3; else NULL), any
 *   v_scale      alignment; the aligned words of four bytes around those needed are read.
 *                A row as fresh memory holds it, all bytes zero, stands for zeros.
 *   page_table   device, int32 [batch, max_pages]: key j of sequence b is row
 *                j % page_size of page page_table[b, j / page_size].  Entries past a
 *                sequence's last page are not read, nor rows past its last key.
 *   seq_lens     device, int32 [batch], in [0, max_pages * page_size]; a value
 *                outside is taken as the nearer end and reported (HSA_ERR_INDEX).
 *   out          device, bf16 [batch, n_new, Hq, D], written.
 *   workspace    device, >= hsa_paged_attention_workspace_bytes(...) bytes, 16-byte
 *                aligned, overwritten; calls (and captured graphs) sharing one must
 *                not overlap on the GPU.  Its size depends on D and the device only.
 * D in {64, 128}; Hq < 2^16; page_size a power of two; max_pages * page_size < 2^31 - 256;
 * n_pages * page_size < 2^31; batch * Hkv * rows < 2^31 - 256 and batch * Hkv * ceil(rows / 8)
 * * max_pages * page_size / 64 < 2^31 with rows = n_new * Hq / Hkv.  A page id outside
 * [0, n_pages) reads as rows of zeros (HSA_ERR_INDEX).  Two launches; the result does not
 * depend on what else runs.  A flat cache of N rows is a cache of ceil(N / page_size) pages
 * with the identity as its table.
 * HSA_E4M3: a key's weight times the power of two of its value row is held to 2^-39 of the
 * row's largest such product; what lies further below adds nothing to out. */
int hsa_paged_attention(const void *q, int batch, int n_new, int Hq, const void *k_pages,
                        const void *v_pages, const uint8_t *k_scale, const uint8_t *v_scale,
                        int n_pages, int page_size, int Hkv, int D, hsa_dtype cache_dtype,
                        const int32_t *page_table, int max_pages, const int32_t *seq_lens,
                        float scale, void *out, void *workspace, size_t workspace_bytes,
                        hsa_stream_t stream);
size_t hsa_paged_attention_workspace_bytes(int batch, int n_new, int Hq, int Hkv, int D);

/* Attention of whole prompts: `batch` sequences packed one behind the other, with
 * grouped heads: query head h reads K/V head h / (Hq / Hkv).  Sequence b has the query
 * rows cu_q[b] .. cu_q[b+1]-1 and the key rows cu_k[b] .. cu_k[b+1]-1, Lq and Lk of
 * them; its query i stands at position p = i + Lk - Lq (its keys may begin before its
 * queries: a prompt continued) and sees
 *   mask == 0   all Lk keys;
 *   mask == F   the keys below (floor(p / F) + 1) * F: causal by frames of F tokens,
 *               plainly causal for F = 1.
 * A row that sees no key is zero.  What a row does not see does not reach it, NaN and
 * infinities included.  scale <= 0 selects 1/sqrt(D).
 *   q, k, v      device, bf16: token rows of Hq (Hkv, Hkv) heads x D values, q_row
 *                (k_row, v_row) elements from one token to the next: Hq * D where they
 *                are compact, more in a fused projection's output; multiples of 8.
 *   cu_q, cu_k   device, int32 [batch + 1], not falling, within [0, total_q] and
 *                [0, total_k]; other values are moved inside and reported
 *                (HSA_ERR_INDEX; what is computed is then unspecified).
 *   total_q,     rows that q and out (k and v) hold; those before cu[0] or from cu[batch]
 *   total_k      on, whatever they hold, do not reach the result, and are not written.
 *   out          device, bf16 [total_q, Hq, D] compact, written; overlaps no input.
 *   dtype        HSA_BF16.
 *   workspace    device, optional (NULL = none), >=
 *                hsa_packed_attention_workspace_bytes(...) bytes, 16-byte aligned: lets
 *                calls with few rows and long keys be cut along the keys and joined (a
 *                second launch).  Overwritten; calls (and captured graphs) sharing one
 *                must not overlap on the GPU.  Its size depends on D and the device.
 * D in {64, 128}; pointers but cu_q and cu_k 16-byte aligned; Hq * D <= 2^24; q_row, k_row,
 * v_row <= 2^31; batch * Hkv <= 2^23; total_k, total_q * Hq / Hkv and Hkv * (total_q * Hq /
 * Hkv / 256 + batch) < 2^31 - 1024.  A row that sees a score, scale * <q, k>, of magnitude
 * 2^30 or more is unspecified.  A NaN or infinity among values that some rows of a block of
 * 256 see and others do not is slow: those others are formed again, at 4 us a key, but where
 * they see NaN in the same dimensions themselves. */
int hsa_packed_attention(const void *q, long long q_row, const void *k, long long k_row,
                         const void *v, long long v_row, const int32_t *cu_q,
                         const int32_t *cu_k, int batch, int total_q, int total_k, int Hq,
                         int Hkv, int D, int mask, float scale, void *out, hsa_dtype dtype,
                         void *workspace, size_t workspace_bytes, hsa_stream_t stream);
size_t hsa_packed_attention_workspace_bytes(int Hq, int Hkv, int D);

/* ------------------------------------------------------- a6 cached Euler */

/* Cached Euler update (Sec. 2.4, Eq. 6) of all N tokens in one pass: when
 * pos[n] >= 0 the velocity cache takes the fresh velocity,
 * v_cache[n] = v_fresh[pos[n]]; then x[n] = fma(v_cache[n], dsigma, x[n])
 * (fp32, one rounding per element), dsigma = sigma_{i+1} - sigma_i.
 *   x, v_cache  device, fp32 [N, C], updated in place.
 *   v_fresh     device, fp32 [n_active, C] (velocities of A_i) or NULL.
 *   pos         device, int32 [N] (as written by hsa_partition_active) or
 *               NULL; both NULL = no refresh.
 *   n_fresh     rows of v_fresh; a pos value outside [-1, n_fresh) (above
 *               the range, or any negative value other than -1) is treated
 *               as -1 and reported as HSA_ERR_INDEX.
 * C must be a positive multiple of 4 and the pointers 16-byte aligned. */
int hsa_cached_euler(float *x, float *v_cache, const float *v_fresh,
                     const int32_t *pos, int n_fresh, int N, int C, float dsigma,
                     hsa_stream_t stream);

/* Cached Euler update fused with the velocity statistic of the dynamic token
 * selection (App. B, Eq. 7), for the initial full-budget iterations whose
 * velocities rank the tokens.  For every token with pos[n] >= 0 it first adds
 *   weight * ||v_fresh[pos[n]] - v_cache[n]||_1 / ||v_fresh[pos[n]]||_1
 * to stat[n] (v_cache[n] still holds the previous step's velocity; a zero
 * denominator adds 0 when the numerator is 0 and weight * FLT_MAX otherwise),
 * then performs exactly hsa_cached_euler.  With weight = 1/(number of steps
 * averaged) stat ends as the mean relative change, ready for hsa_partition.
 *   stat  device, fp32 [N], accumulated in place (fp32 fma).
 * pos and v_fresh are required; other arguments as for hsa_cached_euler. */
int hsa_cached_euler_l1rel(float *x, float *v_cache, const float *v_fresh,
                           const int32_t *pos, int n_fresh, int N, int C, float dsigma,
                           float *stat, float weight, hsa_stream_t stream);

/* ------------------------------------------------------------------ errors */

/* Waits for `stream`, then reports and clears the device-side errors recorded
 * on the current device since the last call: HSA_ERR_TIMEOUT if a bounded wait
 * ran out, else HSA_ERR_NONFINITE, else HSA_ERR_INDEX, else HSA_OK; or
 * HSA_ERR_CUDA if the wait itself failed.  The word is per device, shared by
 * every stream and thread. */
int hsa_get_device_error(hsa_stream_t stream);

/* Number of kernels this library has launched in this process, on any device
 * or stream, since it was loaded (a host-side counter, incremented when a
 * launch is enqueued; a call that fails its argument checks adds nothing).
 * A call captured into a CUDA graph counts once, at capture; replays of the
 * graph are not counted.  Never fails; takes no GPU. */
unsigned long long hsa_launch_count(void);

#ifdef __cplusplus
}
#endif

#endif /* HSA_H */
