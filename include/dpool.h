/*
 * dpool.h - C ABI of libdpool: MI355X (gfx950) paged decode attention for
 * dual-pool token-budget serving, plus the host-side pool sizing and router
 * that decide which pool (and so which decode shape) a request lands in.
 *
 * Paper: "Dual-Pool Token-Budget Routing for Cost-Efficient and Reliable LLM
 * Serving".  Citations below name its sections, equations and algorithm.
 *
 * Conventions (every entry point):
 *   - returns int status: DP_OK (0) or a negative errno-style code:
 *       DP_EINVAL  (-22) bad argument or shape
 *       DP_ENOMEM  (-12) block pool exhausted / workspace too small
 *       DP_ENOTSUP (-95) head_dim, block size, dtype or GQA group not supported
 *       DP_EIO     (-5)  a HIP runtime error (text via dp_last_error())
 *   - no exception, abort or exit crosses the ABI; on error, caller-visible
 *     state is left unchanged;
 *   - the caller owns every buffer it passes.  The library owns only the
 *     opaque dp_kv_pool handle (host memory);
 *   - device pointers are HIP device addresses on the current device; the
 *     decode call is asynchronous on the given stream and never synchronises.
 */
#ifndef DPOOL_H
#define DPOOL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DP_OK 0
#define DP_EIO (-5)
#define DP_ENOMEM (-12)
#define DP_EINVAL (-22)
#define DP_ENOTSUP (-95)

/* Text of the last error raised on the calling thread ("" if none). */
const char* dp_last_error(void);

/* Library version string. */
const char* dp_version(void);

/* ------------------------------------------------------------------------ */
/* KV-cache sizing and paged block pool (host only).                         */
/*                                                                           */
/* Sec. 1.1 Eq. 1: M_seq = 2 * n_layers * n_kv_heads * head_dim             */
/*                         * dtype_bytes * c_max   (bytes per sequence)      */
/* Sec. 1.1 Eq. 2: N_seq = floor((m_gpu_bytes * util - m_model_bytes)       */
/*                               / M_seq), clamped at 0                      */
/* The pool backs N_seq sequences of ceil(c_max / block_size) blocks each   */
/* (16-token PagedAttention blocks, pages handed out on demand: Sec. 3,     */
/* effects 1 and 3).  Free block ids are kept in a list shuffled once with  */
/* a seeded SplitMix64 stream (Steele, Lea & Flood 2014), so that a         */
/* sequence's blocks are scattered over the pool as in a long-running       */
/* server.                                                                   */
/* ------------------------------------------------------------------------ */
typedef struct {
  int32_t n_layers;     /* n_l: layers whose KV this GPU holds             */
  int32_t n_kv_heads;   /* n_h: KV heads on this GPU                        */
  int32_t head_dim;     /* d_h                                              */
  int32_t dtype_bytes;  /* b_dtype: 2 for bf16, 1 for fp8                   */
  int32_t block_size;   /* tokens per block (16)                            */
  int32_t reserved;     /* must be 0                                        */
  int64_t c_max;        /* C_max: tokens reserved per sequence              */
  double m_gpu_bytes;   /* M_gpu                                             */
  double util;          /* u, fraction of HBM usable (0, 1]                  */
  double m_model_bytes; /* M_model (weights + activations)                   */
} dp_pool_config;

typedef struct dp_kv_pool dp_kv_pool; /* opaque, host memory, owned by the library */

/* Size a pool (Eq. 1, Eq. 2) and build its shuffled free list.
 * DP_EINVAL on non-positive sizes, util outside (0,1] or reserved != 0;
 * DP_ENOMEM if the free list cannot be allocated.  *out is set only on success. */
int kv_pool_create(const dp_pool_config* cfg, uint64_t shuffle_seed, dp_kv_pool** out);

/* Sizing results: Eq. 1 M_seq, Eq. 2 N_seq, ceil(c_max/bs), N_seq*blocks_per_seq,
 * and the number of blocks currently free.  Any output pointer may be NULL. */
int kv_pool_info(const dp_kv_pool* pool, int64_t* m_seq_bytes, int64_t* n_seq,
                 int64_t* blocks_per_seq, int64_t* num_blocks, int64_t* free_blocks);

/* Hand out ceil(n_tokens / block_size) blocks for one sequence (on-demand
 * pages, Sec. 3 effect 1).  block_ids_out must hold that many int32.
 * DP_EINVAL if n_tokens < 0 or n_tokens > c_max; DP_ENOMEM if the pool has
 * too few free blocks (the OOM of Sec. 1.3), in which case nothing is taken. */
int kv_pool_alloc_seq(dp_kv_pool* pool, int64_t n_tokens, int32_t* block_ids_out);

/* Return blocks to the pool.  DP_EINVAL (nothing returned) if any id is out
 * of range or already free. */
int kv_pool_free_seq(dp_kv_pool* pool, const int32_t* block_ids, int64_t n_blocks);

void kv_pool_destroy(dp_kv_pool* pool);

/* ------------------------------------------------------------------------ */
/* Token-budget routing (host only): Sec. 2.1 Eq. 3-5, Sec. 2.2 Algorithm 1 */
/*                                                                           */
/* Route:  c* = c_hat_k - gamma * sigma_k (Eq. 5), clamped below at c_min;   */
/*         L_total = ceil(bytes / c*) + max_output_tokens (Eq. 3);           */
/*         step 1  L_total > C_max(short)           -> long                  */
/*         step 2  L_total <= b_short ? short : long                         */
/*         step 3  spill to the other pool if the chosen one is overloaded   */
/*                 (in_flight >= spill_theta * capacity) and the other can   */
/*                 take the request (L_total <= its C_max, not overloaded);  */
/*         final   L_total > C_max(chosen)          -> long.                 */
/*         The chosen pool's in_flight is incremented.                       */
/* OnResponse: c_obs = bytes / prompt_tokens;                                */
/*         c_hat = beta*c_hat + (1-beta)*c_obs (Eq. 4);                      */
/*         sigma = beta*sigma + (1-beta)*|c_obs - c_hat| (updated c_hat).    */
/* All arithmetic is IEEE double in exactly that order (no FMA contraction), */
/* so results are reproducible bit for bit by any IEEE-754 implementation.   */
/* ------------------------------------------------------------------------ */
typedef struct {
  double b_short;     /* B_short threshold in tokens (default 8192)        */
  double beta;        /* EMA decay (0.95)                                   */
  double gamma;       /* conservativeness (1.0)                             */
  double c0;          /* cold-start bytes/token (4.0)                       */
  double c_min;       /* floor of the conservative ratio (1.0)              */
  double spill_theta; /* overload fraction of capacity (1.0)                */
} dp_route_params;

typedef struct {
  double c_hat; /* calibrated bytes per token of the category */
  double sigma; /* EMA of |c_obs - c_hat|                      */
} dp_cat_state;

typedef struct {
  int64_t c_max;     /* longest total budget the pool can serve */
  int64_t capacity;  /* concurrent sequences (N_seq * instances) */
  int64_t in_flight; /* requests currently assigned             */
} dp_pool_state;      /* pools[0] = short pool, pools[1] = long pool */

/* Fill params with the paper's defaults. */
int route_default_params(dp_route_params* params);

/* Cold-start every category: c_hat = c0, sigma = 0. */
int route_init(const dp_route_params* params, dp_cat_state* cats, int32_t n_cats);

/* Route n requests in order (Algorithm 1, Route).  req_bytes[i] >= 0,
 * 0 <= req_cat[i] < n_cats, req_max_out[i] >= 0; otherwise DP_EINVAL and
 * nothing is written.  out_pool[i] = 0 (short) or 1 (long); out_l_total[i]
 * = the estimated budget (either output may be NULL).  pools[*].in_flight is
 * updated.  Host arrays, O(n), no allocation. */
int route_requests(const dp_route_params* params, const dp_cat_state* cats, int32_t n_cats,
                   dp_pool_state pools[2], const int64_t* req_bytes, const int32_t* req_cat,
                   const int64_t* req_max_out, int64_t n, int8_t* out_pool,
                   int64_t* out_l_total);

/* Algorithm 1, OnResponse.  DP_EINVAL (state unchanged) if cat is out of
 * range, req_bytes < 0 or prompt_tokens <= 0. */
int route_on_response(const dp_route_params* params, dp_cat_state* cats, int32_t n_cats,
                      int32_t cat, int64_t req_bytes, int64_t prompt_tokens);

/* ------------------------------------------------------------------------ */
/* Adaptive B_short (host only).  Sec. 7 names, as future work, a routing   */
/* threshold that adjusts itself from preemption rate, OOM events and        */
/* request rejections; Sec. 6 recommends alerting on a preemption rate above */
/* 1%, and Sec. 4.6 finds any B_short in 4K-16K within 80% of peak savings.  */
/* The paper gives no update rule; this is the library's, one call per       */
/* control interval:                                                         */
/*   e_i = w_preempt*preempted_i + w_oom*oom_i + w_reject*rejected_i         */
/*   x_i = e_i / max(admitted_i, 1) - target        (i = 0 short, 1 long)    */
/*   x_0 > 0 and x_0 > x_1:  b = b - step*b   (short pool under pressure:    */
/*                                             send borderline traffic long) */
/*   x_1 > 0 and x_1 > x_0:  b = b + step*b   (long pool under pressure)     */
/*   otherwise               b unchanged                                     */
/*   then b is clamped into [b_min, b_max].                                  */
/* IEEE double, in exactly that order, no FMA contraction.                   */
/* ------------------------------------------------------------------------ */
typedef struct {
  int64_t admitted;  /* requests routed to the pool during the interval */
  int64_t preempted; /* sequences preempted for want of KV cache         */
  int64_t oom;       /* out-of-memory events                             */
  int64_t rejected;  /* requests refused at admission                    */
} dp_pool_signals;   /* signals[0] = short pool, signals[1] = long pool  */

typedef struct {
  double w_preempt; /* weight of a preemption (1.0)                          */
  double w_oom;     /* weight of an OOM event (1.0)                          */
  double w_reject;  /* weight of a rejection (1.0)                           */
  double target;    /* tolerated events per admitted request (0.01)          */
  double step;      /* relative change of B_short per interval (0.05)        */
  double b_min;     /* lower bound of B_short in tokens (4096)               */
  double b_max;     /* upper bound (16384; no use above the short C_max)     */
} dp_adapt_params;

/* Fill ap with the defaults above. */
int route_adapt_default_params(dp_adapt_params* ap);

/* One control step on *b_short (in/out).  *action (may be NULL) = -1, 0 or
 * +1 for lowered, unchanged, raised (before the clamp).  DP_EINVAL, nothing
 * written, unless every count is >= 0, the weights and target are >= 0,
 * 0 < step < 1, 0 < b_min <= b_max and *b_short is finite and > 0. */
int route_adapt_threshold(const dp_adapt_params* ap, const dp_pool_signals signals[2], double* b_short,
                          int32_t* action);

/* ------------------------------------------------------------------------ */
/* Fleet cost model (host only): Sec. 3, "Cost Model: Why Splitting Always  */
/* Helps".                                                                   */
/*   G_homo = ceil(lambda / mu_long)                                         */
/*   G_dual = ceil(alpha * lambda / mu_short)                                */
/*          + ceil((1 - alpha) * lambda / mu_long)                           */
/*   rho = mu_short / mu_long;  savings_formula = alpha * (1 - 1 / rho)      */
/*   (the boxed equation);  savings_fleet = (G_homo - G_dual) / G_homo       */
/* lambda: request rate; alpha: fraction of traffic short; mu_*: per-GPU     */
/* throughput of each pool, same unit as lambda.  IEEE double, in that       */
/* order, no FMA contraction.  DP_EINVAL (nothing written) unless           */
/* lambda > 0, 0 <= alpha <= 1 and both throughputs are positive.           */
/* ------------------------------------------------------------------------ */
typedef struct {
  int64_t g_homo;         /* GPUs of the homogeneous fleet           */
  int64_t g_dual;         /* GPUs of the dual-pool fleet             */
  double rho;             /* throughput gain ratio                   */
  double savings_formula; /* alpha (1 - 1/rho)                       */
  double savings_fleet;   /* (G_homo - G_dual) / G_homo, with ceilings */
} dp_cost_result;

int dp_cost_model(double lambda, double alpha, double mu_short, double mu_long, dp_cost_result* out);

/* ------------------------------------------------------------------------ */
/* Paged decode attention (device, asynchronous).                           */
/*                                                                           */
/* The per-step KV read the paper's cost model calls memory-bandwidth bound */
/* (Sec. 3 effect 4; Sec. 4.4 "Why TPOT also improves"), over 16-token      */
/* PagedAttention blocks (Sec. 3 effect 3).  For sequence s with            */
/* T = context_lens[s] and query head h (KV head g = h / G, G = Hq / Hkv):  */
/*   K_t = k_scale[g] * k_blocks[block_tables[s][t/16], g, t%16, :]          */
/*   V_t = v_scale[g] * v_blocks[block_tables[s][t/16], g, :, t%16]          */
/*   out[s,h,:] = softmax_t(scale * q[s,h,:] . K_t) @ V                     */
/* T = 0 gives a zero row.                                                   */
/*                                                                           */
/* Layouts (row-major, device memory, 16-byte aligned):                      */
/*   q            [batch, n_q_heads, head_dim]            bf16               */
/*   k_blocks     [num_blocks, n_kv_heads, block_size, head_dim]             */
/*                (token-major: one token's dims are contiguous)             */
/*   v_blocks     [num_blocks, n_kv_heads, head_dim, block_size]             */
/*                (dims-major: one dim's 16 tokens are contiguous)           */
/*                both bf16 (DP_KV_BF16) or OCP e4m3 bytes (DP_KV_FP8_E4M3); */
/*                each (block, KV head) tile of K and of V is contiguous     */
/*   block_tables [batch, max_blocks_per_seq] int32; entries past            */
/*                ceil(T/16) are never read (may hold -1); ids outside       */
/*                [0, num_blocks) are clamped into range, never dereferenced */
/*   context_lens [batch] int32, each <= max_context_len (a caller promise;  */
/*                larger values are clamped, never read out of bounds).      */
/*                Cache slots at t >= T of a sequence's last block are never */
/*                used, whatever they hold                                   */
/*   k_scale,     [n_kv_heads] fp32 per-head dequantisation scales (fp8      */
/*   v_scale        only; must be NULL for bf16)                             */
/*   out          [batch, n_q_heads, head_dim] bf16 (DP_OUT_BF16) or fp32    */
/*   workspace    >= paged_decode_workspace_size(shape) bytes, 256-byte      */
/*                aligned, caller-owned.  It must be zero-filled before its  */
/*                first use; every completed call leaves its arrival         */
/*                counters at zero again, so one workspace serves any number */
/*                of later calls, of any shape, in stream order.  Calls that */
/*                share a workspace must not overlap in time.                */
/* Supported: head_dim 128, block_size 16, 1 <= Hq/Hkv <= 16, batch <= 4096. */
/* ------------------------------------------------------------------------ */
#define DP_KV_BF16 0
#define DP_KV_FP8_E4M3 1
#define DP_KV_FP8_E4M3_BLOCK 2 /* e4m3, a scale per block and head: only the entry points that name it */
#define DP_OUT_BF16 0
#define DP_OUT_FP32 1

typedef struct {
  int32_t batch;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t block_size;
  int32_t max_blocks_per_seq;
  int32_t max_context_len;
  int32_t kv_dtype;          /* DP_KV_*                                       */
  int32_t out_dtype;         /* DP_OUT_*                                      */
  int32_t partition_tokens;  /* minimum tokens of KV one wave processes (the  */
                             /* split-K granularity): a multiple of 32 (bf16) */
                             /* or 64 (fp8); 0 = library's choice             */
  int32_t workgroups_per_cu; /* resident workgroups per compute unit, 1..8    */
                             /* (capped by occupancy); 0 = library's choice   */
  int32_t reserved;          /* must be 0                                     */
  int64_t num_blocks;        /* blocks in k_blocks / v_blocks                  */
} dp_decode_shape;

/* Bytes of workspace paged_decode_attention needs for this shape (it depends
 * on the device's compute-unit count and the GQA group).  Returns 0 for
 * invalid shapes (the reason is in dp_last_error()). */
size_t paged_decode_workspace_size(const dp_decode_shape* shape);

/* The minimum tokens per wave slice the library uses for this shape
 * (0 for invalid shapes).  For a shape that paged_decode_attention gives one
 * workgroup per pair (below) it is the slice that cut pairs would have;
 * passed back as partition_tokens it asks for them. */
int32_t paged_decode_partition_tokens(const dp_decode_shape* shape);

/* Enqueue the decode attention on `stream` (a hipStream_t; NULL = default
 * stream) as one kernel launch.  Validates the shape and pointer alignment
 * on the host (DP_EINVAL / DP_ENOTSUP; DP_ENOMEM for a short workspace;
 * nothing is enqueued then); DP_EIO if the launch fails.
 *
 * Split-K over the context: the cached tokens of all (sequence, KV head)
 * pairs are cut into equal slices, one per wave; a pair cut by slice
 * boundaries leaves per-slice softmax partials (o_p, m_p, l_p), which are
 * merged with log-sum-exp weights M = max_p m_p, w_p = l_p * 2^(m_p - M),
 * out = sum_p w_p o_p / sum_p w_p: first inside each workgroup (through its
 * LDS), then, for pairs whose slices span several workgroups, the
 * workgroups' partials through the workspace, by the last to finish.
 * Calls of few, short sequences are not cut: each pair is one workgroup's,
 * and the workspace is neither read nor written (its size and alignment are
 * checked all the same).  That holds for partition_tokens and
 * workgroups_per_cu 0, max_context_len <= 512 (bf16) or 1,024 (e4m3) and at
 * most one pair per compute unit; either field other than 0 asks for slices.
 * Both ways round probabilities to bf16 against the maximum of their slice;
 * outputs differ by no more than that rounding.
 * The workspace also keeps, for each wave, the cache tiles its first unit
 * read; the next call starts loading those tiles before it has found its
 * own, and loads again where they differ.  A call with the context lengths
 * and block tables of the previous call on the workspace (every layer of a
 * decode step after the first) starts its reads earlier; results never
 * depend on what the workspace holds.
 * Results are deterministic: the same inputs and shape give the same bits. */
int paged_decode_attention(const void* q, const void* k_blocks, const void* v_blocks,
                           const int32_t* block_tables, const int32_t* context_lens,
                           float scale, const float* k_scale, const float* v_scale,
                           void* out, const dp_decode_shape* shape, void* workspace,
                           size_t workspace_bytes, void* stream);

/* paged_decode_attention for callers that cannot allocate device memory
 * (code under HIP graph capture, serving loops and harnesses that forbid
 * hipMalloc).  Same arguments, layouts, results and errors as
 * paged_decode_attention, without the workspace: the library keeps a fixed
 * 32 MiB device array per GPU (held until the process ends, its address
 * looked up and the array zero-filled by one small kernel on `stream` at
 * the first call made on that device) and uses it as the workspace.  Nothing
 * is allocated, on the first call or later.
 * DP_ENOMEM (nothing enqueued) if the shape needs more than 32 MiB (see
 * paged_decode_workspace_size): every GQA group up to 16 fits with one
 * workgroup per compute unit (workgroups_per_cu 0 or 1) on a 256-CU device.
 * Every call on a device shares its array: calls that overlap in time on
 * one device (different streams, host threads) race and must not be made. */
int paged_decode_attention_noalloc(const void* q, const void* k_blocks, const void* v_blocks,
                                   const int32_t* block_tables, const int32_t* context_lens,
                                   float scale, const float* k_scale, const float* v_scale,
                                   void* out, const dp_decode_shape* shape, void* stream);

/* ------------------------------------------------------------------------ */
/* Decode over a sliding window, and over block scales (device, asynchronous)*/
/*                                                                           */
/* Layers of long-context models that see a window read, for every           */
/* generated token, the window's part of the cache instead of all of it, and */
/* a few first tokens that stay visible.  For sequence s with                */
/* T = context_lens[s]:                                                       */
/*   out[s,h,:] = sum_t softmax_t(scale * q[s,h,:] . K_t) V_t                */
/*   over T - window <= t < T, and t < min(n_sink, T)                        */
/* T = 0 gives a zero row, and so does one whose scores are all -infinity.   */
/* A cached value of a token that is not seen never reaches the result,      */
/* finite or not, and table entries of blocks that hold no token that is     */
/* seen are never read (blocks that have left the window may go back to the  */
/* pool, their entries set below 0; kv_tables_step then ends such a sequence  */
/* with -2).  window >= 1; one of max_context_len or more hides nothing.      */
/* n_sink >= 0.                                                               */
/*                                                                           */
/* kv_dtype may also be DP_KV_FP8_E4M3_BLOCK: the cache holds e4m3 codes as  */
/* for DP_KV_FP8_E4M3, and k_scale, v_scale are [num_blocks, n_kv_heads]     */
/* bytes, the exponents of powers of two (OCP E8M0):                          */
/*   K_t = 2^(k_scale[blk][g] - 127) * k_blocks[blk, g, t%16, :]             */
/*   V_t = 2^(v_scale[blk][g] - 127) * v_blocks[blk, g, :, t%16]             */
/* with blk = block_tables[s][t/16]; 255 stands for NaN.  Such a cache needs */
/* no calibration: qk_norm_rope_append_scaled sets the scales.  Values are   */
/* taken as bf16, which holds them exactly but for those below 2^-126 (a few */
/* bits fewer) and above its largest (infinity).                              */
/*                                                                           */
/* Everything else, the shape, layouts, split, workspace and its rules,      */
/* limits and errors, is as for paged_decode_attention, and the two may      */
/* share a workspace; for DP_KV_FP8_E4M3 k_scale and v_scale are fp32        */
/* [n_kv_heads] and 4-byte aligned.  Calls whose windows and sinks hold few  */
/* tokens count as short whatever max_context_len is.  q, out and workspace  */
/* do not overlap (DP_EINVAL where they start together).  DP_EINVAL for      */
/* window < 1 or n_sink < 0; max_context_len <= 2^30.                         */
/* ------------------------------------------------------------------------ */
size_t window_decode_workspace_size(const dp_decode_shape* shape, int32_t window, int32_t n_sink);

int window_decode_attention(const void* q, const void* k_blocks, const void* v_blocks,
                            const int32_t* block_tables, const int32_t* context_lens, float scale,
                            int32_t window, int32_t n_sink, const void* k_scale, const void* v_scale,
                            void* out, const dp_decode_shape* shape, void* workspace,
                            size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* KV-cache append (device, asynchronous).                                   */
/*                                                                           */
/* Each decode step adds one token per sequence to the cache before the     */
/* attention reads it (Sec. 4.4: one KV-cache lookup per layer per          */
/* generated token); pages are 16-token blocks handed out on demand (Sec. 3 */
/* effects 1 and 3); the FP8 deployment of Sec. 4.7 stores 8-bit floats.   */
/* For sequence s, t = positions[s], KV head g:                             */
/*   blk = block_tables[s][t / 16], slot = t % 16                           */
/*   k_blocks[blk, g, slot, :] = enc(k_new[s, g, :] / k_scale[g])            */
/*   v_blocks[blk, g, :, slot] = enc(v_new[s, g, :] / v_scale[g])            */
/* enc() copies the bf16 bits for a bf16 cache (no scales); for an e4m3     */
/* cache it is a correctly rounded fp32 division, clamped to +-448 and      */
/* rounded to the nearest OCP E4M3FN value (ties to even).  Inputs are      */
/* finite (a caller promise).                                                */
/*                                                                           */
/*   k_new, v_new [batch, n_kv_heads, 128] bf16, 4-byte aligned             */
/*   k_blocks, v_blocks, block_tables: as for paged_decode_attention        */
/*   positions    [batch] int32: the slot index of the new token; a          */
/*                position outside [0, 16 * max_blocks_per_seq), or a block */
/*                id outside [0, num_blocks), writes nothing for that        */
/*                sequence                                                   */
/*   k_scale, v_scale [n_kv_heads] fp32 (e4m3 only; NULL for bf16)          */
/*   shape        uses batch, n_kv_heads, head_dim (128), block_size (16),   */
/*                max_blocks_per_seq, kv_dtype, num_blocks; the other        */
/*                fields are ignored except reserved (must be 0)            */
/* One launch on `stream`; DP_EINVAL / DP_ENOTSUP for bad arguments (nothing */
/* enqueued), DP_EIO if the launch fails.  Two sequences that name the same */
/* (block, slot) race.                                                       */
/* ------------------------------------------------------------------------ */
int kv_cache_append(const void* k_new, const void* v_new, void* k_blocks, void* v_blocks,
                    const int32_t* block_tables, const int32_t* positions,
                    const float* k_scale, const float* v_scale, const dp_decode_shape* shape,
                    void* stream);

/* ------------------------------------------------------------------------ */
/* Chunked-prefill attention (device, asynchronous).                        */
/*                                                                           */
/* Each pool runs chunked prefill internally (Sec. 1.2): a prompt is        */
/* attended in chunks (2,048 tokens by default) whose K and V are already   */
/* in the paged cache (kv_cache_append, or any writer of the same layout).  */
/* For sequence s with T = context_lens[s] cached tokens (the chunk         */
/* included) and n = q_start[s+1] - q_start[s] query rows, row              */
/* r = q_start[s] + i sits at position p = T - n + i and, for query head h  */
/* (KV head g = h / G):                                                      */
/*   out[r,h,:] = sum_{t <= p} softmax_t(scale * q[r,h,:] . K_t) V_t         */
/* with K_t, V_t gathered exactly as for paged_decode_attention.  Decode is */
/* the case n = 1.                                                           */
/*                                                                           */
/* Layouts: q and out [total_q, n_q_heads, 128] (bf16 / out_dtype), rows    */
/* packed sequence after sequence as q_start says; k_blocks, v_blocks,      */
/* block_tables, context_lens, k_scale, v_scale as for decode; q_start      */
/* [batch + 1] int32 on the device, non-decreasing, q_start[0] = 0,         */
/* q_start[batch] <= total_q.  A caller promise: n <= T for every sequence. */
/* Values that break it (or q_start out of order) are clamped: no access    */
/* leaves the buffers, rows past min(n, T) are left unwritten and rows of   */
/* overlapping ranges are unspecified.  No workspace; nothing is allocated. */
/* A cached V value that is not finite shows in its token's row and later    */
/* ones, and may show in rows up to 62 positions earlier, in none before.    */
/* Supported: head_dim 128, block_size 16, Hq a multiple of Hkv,            */
/* batch <= 4096, max_context_len <= 65536 (the long pool's C_max).          */
/* ------------------------------------------------------------------------ */
typedef struct {
  int32_t batch;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t block_size;
  int32_t max_blocks_per_seq;
  int32_t max_context_len;
  int32_t kv_dtype;   /* DP_KV_*                                             */
  int32_t out_dtype;  /* DP_OUT_*                                            */
  int32_t query_tile; /* 0 or 32; either way the library sizes its work items */
  int32_t reserved;   /* must be 0                                           */
  int64_t total_q;    /* rows of q and out                                   */
  int64_t num_blocks; /* blocks in k_blocks / v_blocks                       */
} dp_prefill_shape;

/* Enqueue the chunked-prefill attention on `stream` as one kernel launch.
 * Host-side validation as for decode (DP_EINVAL / DP_ENOTSUP, nothing
 * enqueued); DP_EIO if the launch fails. */
int chunked_prefill_attention(const void* q, const void* k_blocks, const void* v_blocks,
                              const int32_t* block_tables, const int32_t* context_lens,
                              const int32_t* q_start, float scale, const float* k_scale,
                              const float* v_scale, void* out, const dp_prefill_shape* shape,
                              void* stream);

/* Chunked prefill over a sliding window, and over block scales: row r at     */
/* position p (as above) sees p - window < t <= p, and t < n_sink.  Window,   */
/* sinks, kv_dtype DP_KV_FP8_E4M3_BLOCK and its k_scale and v_scale are as    */
/* for window_decode_attention; everything else is as for                     */
/* chunked_prefill_attention.  A row that sees only scores of -infinity gives */
/* zeros.  Table entries of blocks that hold no token that some row sees are  */
/* never read.  A cached V value that is not finite shows in the rows that    */
/* see its token, and may show in rows up to 62 positions from those, in none */
/* farther.  Supported: max_context_len <= 65536, or up to 2^30 where          */
/* window + n_sink <= 65024.                                                   */
/* q and out do not overlap (DP_EINVAL where they start together).            */
int window_prefill_attention(const void* q, const void* k_blocks, const void* v_blocks,
                             const int32_t* block_tables, const int32_t* context_lens,
                             const int32_t* q_start, float scale, int32_t window, int32_t n_sink,
                             const void* k_scale, const void* v_scale, void* out,
                             const dp_prefill_shape* shape, void* stream);

/* ------------------------------------------------------------------------ */
/* Block tables and slot maps on the device (asynchronous).                  */
/*                                                                           */
/* Blocks are handed out on demand (Sec. 3 effect 1).  kv_pool_alloc_seq    */
/* does it on the host; this call does it where the lengths already are,    */
/* for a whole batch and without a synchronisation: it gives every sequence */
/* the blocks its next tokens need, from a ring of free ids in device       */
/* memory, takes back the blocks of sequences that are over, and writes the */
/* block tables and, for every new token (a row), its cache slot and its    */
/* position.                                                                 */
/*   The ring: free_ids [num_blocks]; free_state_in = {head, count}: the    */
/* ids free_ids[(head + i) % num_blocks], i < count, are free (a new pool:  */
/* all ids of a kv_pool, head 0).                                            */
/*   Sequence s with c = context_lens[s] cached tokens (not counting the    */
/* new ones), b = n_owned[s] blocks in its table (at least ceil(c / 16),    */
/* which a smaller value is taken for) and x = new_tokens[s]:               */
/*     x < 0   the sequence is over: its b table entries go to the end of   */
/*             the ring, in table order, sequences in batch order; its      */
/*             context and owned count become 0 (they are free for the next */
/*             call, not for this one).  With x = -1 all b entries go, with  */
/*             x < -1 those that are not below 0: a sequence whose blocks    */
/*             left a window earlier, and went back to the ring then with    */
/*             their entries set below 0, ends with x = -2.  Such entries    */
/*             count as owned                                                */
/*     x >= 0  it needs max(0, ceil((c + x) / 16) - b) blocks.  In batch    */
/*             order, needs are met while the sum of all needs so far is at */
/*             most `count`; a sequence that needs none is always met.      */
/*             granted[s] = 1, context c + x, table entries b and up set to */
/*             the next ids of the ring.  Else granted[s] = 0 and the       */
/*             sequence stays as it was.  Refused too, and left out of the  */
/*             sum: c + x > 16 * max_blocks_per_seq, rows that end past     */
/*             total_rows, more than 64 * mask_words rows with parents.     */
/*   Rows: sequence s has rows q_start[s] .. q_start[s+1] (q_start = the    */
/* running sum of max(x, 0), whether granted or not, cut at total_rows).    */
/* The rows of a refused sequence have no tokens in the cache: attention's   */
/* results for them are of no use.                                           */
/* Row i of s is cached at t = c + i:                                        */
/*     slots = block_tables[s][t / 16] * 16 + t % 16 (-1 if not granted, or  */
/*     where that entry is below 0)                                           */
/*     positions = t, or with parents c + (number of ancestors)              */
/* Rows behind the last sequence (a batch padded to a fixed size) get slot  */
/* -1, position -1 and an empty mask.                                        */
/*   parents (may be NULL) makes each sequence's rows a tree of drafted     */
/* tokens: parents[row] is the index within the sequence of the row's       */
/* parent, which must come before it; -1 (as any other value) for a child   */
/* of the cached context.  tree_mask [total_rows, mask_words] 64-bit words, */
/* bit j % 64 of word j / 64 for row j of the sequence: set for the row and */
/* its ancestors.                                                            */
/*                                                                           */
/*   context_lens, n_owned, new_tokens, granted, context_lens_out,           */
/*   n_owned_out [batch] int32; free_ids [num_blocks] int32 (updated in      */
/*   place); free_state_in, free_state_out [2] int32; block_tables [batch,   */
/*   max_blocks_per_seq] int32 (updated in place; entries from the owned    */
/*   count on are of no meaning); q_start [batch + 1] int32; slots           */
/*   [total_rows] int64; positions, parents [total_rows] int32.              */
/* No output may be an input or another output (DP_EINVAL).  The updates in */
/* place leave what the call reads alone, so a call repeated on the same    */
/* inputs does the same.                                                     */
/* One launch; nothing is allocated.  batch <= 4096, block_size 16,         */
/* total_rows and num_blocks <= 2^30, mask_words 0 (no parents) to 4.       */
/* DP_EINVAL / DP_ENOTSUP for bad arguments (nothing enqueued), DP_EIO if   */
/* the launch fails.                                                         */
/* ------------------------------------------------------------------------ */
typedef struct {
  int32_t batch;
  int32_t block_size;
  int32_t max_blocks_per_seq;
  int32_t mask_words; /* 64-bit words of a row of tree_mask, 1..4; 0 without parents */
  int64_t total_rows; /* rows of slots, positions, parents and tree_mask             */
  int64_t num_blocks; /* ids of the pool: entries of free_ids                        */
  int64_t reserved;   /* must be 0                                                   */
} dp_tables_shape;

int kv_tables_step(const int32_t* context_lens, const int32_t* n_owned, const int32_t* new_tokens,
                   const int32_t* parents, int32_t* free_ids, const int32_t* free_state_in,
                   int32_t* block_tables, int32_t* context_lens_out, int32_t* n_owned_out,
                   int32_t* free_state_out, int32_t* q_start, int64_t* slots, int32_t* positions,
                   int32_t* granted, uint64_t* tree_mask, const dp_tables_shape* shape, void* stream);

/* ------------------------------------------------------------------------ */
/* Norm and rotation of queries and keys, with the cache write (device,      */
/* asynchronous).                                                            */
/*                                                                           */
/* What comes before the attention of a step, in one pass over the new      */
/* tokens' projections.  For row r at position p = positions[r], and each   */
/* head vector x of q and k:                                                 */
/*     y = x * w / sqrt(mean(x^2) + eps)     (q_weight or k_weight;          */
/*                                            y = x without that weight)     */
/*     the first rotary_dim dimensions of y are turned pair by pair, pair d  */
/*     = (d, d + rotary_dim / 2), or (2d, 2d + 1) if interleaved, by the     */
/*     angle whose cosine and sine are cos_sin[p][d] and                     */
/*     cos_sin[p][rotary_dim / 2 + d]:                                       */
/*         y_a' = y_a cos - y_b sin,  y_b' = y_b cos + y_a sin               */
/*     q_out[r, h, :] = y' rounded to bf16                                   */
/*     k_blocks[blk, g, slot, :] = enc(y' / k_scale[g])                      */
/*     v_blocks[blk, g, :, slot] = enc(v[r, g, :] / v_scale[g])              */
/* with blk = slots[r] / 16, slot = slots[r] % 16; enc() rounds to bf16, or */
/* as in kv_cache_append to e4m3.  Values need not be finite: a NaN, also    */
/* one that the norm of an infinity makes, is stored as NaN, an infinity as  */
/* +-448 in e4m3.  All arithmetic is fp32, rounded once.                     */
/* A row whose position is outside [0, n_positions) is left alone            */
/* altogether; one whose slot is outside [0, 16 * num_blocks) writes q_out   */
/* and no cache.  Two rows that name the same slot race.                     */
/*                                                                           */
/*   q [rows, n_q_heads, 128], k, v [rows, n_kv_heads, 128] bf16, heads      */
/*   contiguous, rows q_stride, k_stride, v_stride elements apart (slices    */
/*   of one projection's output, say); strides are multiples of 8            */
/*   q_weight, k_weight [128] bf16, either may be NULL                       */
/*   cos_sin [n_positions, rotary_dim] fp32; positions [rows] int32;         */
/*   slots [rows] int64                                                      */
/*   q_out [rows, n_q_heads, 128] bf16, contiguous; may be q itself where    */
/*   q_stride is n_q_heads * 128, and overlaps none of the inputs otherwise  */
/*   k_blocks, v_blocks, k_scale, v_scale: as for kv_cache_append            */
/* q, k, v, weights, cos_sin, q_out and the caches are 16-byte aligned.     */
/* rotary_dim is a multiple of 16 in [0, 128].  One launch; nothing is      */
/* allocated.  DP_EINVAL / DP_ENOTSUP for bad arguments (nothing enqueued), */
/* DP_EIO if the launch fails.                                               */
/* ------------------------------------------------------------------------ */
typedef struct {
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;    /* 128                                    */
  int32_t block_size;  /* 16                                     */
  int32_t kv_dtype;    /* DP_KV_*                                */
  int32_t rotary_dim;
  int32_t interleaved; /* 0: pairs (d, d + rotary_dim/2); 1: pairs (2d, 2d+1) */
  int32_t reserved;    /* must be 0                              */
  int64_t rows;
  int64_t num_blocks;
  int64_t n_positions; /* rows of cos_sin                        */
  int64_t q_stride;    /* elements from one row to the next      */
  int64_t k_stride;
  int64_t v_stride;
} dp_qk_shape;

int qk_norm_rope_append(const void* q, const void* k, const void* v, const void* q_weight,
                        const void* k_weight, float eps, const float* cos_sin,
                        const int32_t* positions, const int64_t* slots, void* q_out, void* k_blocks,
                        void* v_blocks, const float* k_scale, const float* v_scale,
                        const dp_qk_shape* shape, void* stream);

/* The same into a cache with block scales (DP_KV_FP8_E4M3_BLOCK, which      */
/* window_decode_attention and window_prefill_attention read).  k_scale and  */
/* v_scale are [num_blocks, n_kv_heads] exponent bytes, updated in place:     */
/* byte e stands for 2^(e - 127).  Rows that follow each other and go into   */
/* one block form a run.  For a run, head g, and y' (K) or v (V), with s0    */
/* the block's slot of its first row and a the largest finite magnitude      */
/* among its rows:                                                            */
/*     need = the smallest 2^(e - 127), 1 <= e <= 246, with a <= 448 * need  */
/*     new  = need if s0 = 0 (the block is begun; whatever it held before    */
/*            counts no more), else the larger of need and the block's scale */
/*     the run's codes   = y' / new, rounded once to e4m3, ties to even      */
/*     the slots before s0, where new is not the block's scale: their codes  */
/*            times (old / new), rounded to e4m3: the same values, but where */
/*            they fall below e4m3's normal range                             */
/* Values that are not finite are stored as NaN and do not count in a.       */
/* Slots of the block behind the run's are of no meaning.  Rows of one block */
/* lie next to each other in the call, at most 16 of them, their slots       */
/* rising, as kv_tables_step hands them out, and nothing else writes to the  */
/* block meanwhile; V tiles are written whole.  Rows that break this leave   */
/* unspecified values in their blocks, and no access leaves the buffers.     */
/* Chains of drafts that are refused are simply written over (a scale that   */
/* they raised stays raised for the block's earlier tokens); drafted trees,  */
/* whose accepted tokens move (kv_cache_accept), need one of the other       */
/* cache types.                                                               */
/* n_q_heads may be 0 (q, q_weight, q_out NULL): K and V only, which with     */
/* rotary_dim 0 and no k_weight is a plain append.  k_scale and v_scale, and  */
/* the two caches, are apart (DP_EINVAL where they start together).           */
/* Everything else, errors included, is as for qk_norm_rope_append.           */
int qk_norm_rope_append_scaled(const void* q, const void* k, const void* v, const void* q_weight,
                               const void* k_weight, float eps, const float* cos_sin,
                               const int32_t* positions, const int64_t* slots, void* q_out,
                               void* k_blocks, void* v_blocks, uint8_t* k_scale, uint8_t* v_scale,
                               const dp_qk_shape* shape, void* stream);

/* ------------------------------------------------------------------------ */
/* Attention of drafted trees over the paged cache (device, asynchronous).  */
/*                                                                           */
/* Speculative decoding checks several drafted tokens of a sequence in one  */
/* pass; they form a tree, and each may see the committed tokens, its       */
/* ancestors and itself.  For sequence s with T = context_lens[s] cached    */
/* tokens (the drafts included: K and V of draft j sit at token T - n + j)  */
/* and n = q_start[s+1] - q_start[s] drafts, row r = q_start[s] + i:        */
/*   out[r,h,:] = sum_t softmax_t(scale * q[r,h,:] . K_t) V_t               */
/*   over t < T - n, and t = T - n + j for every j < n whose bit j % 64 of  */
/*   tree_mask[r][j / 64] is set                                             */
/* with K_t, V_t gathered exactly as for paged_decode_attention.  Any bits  */
/* are allowed: a chain of drafts (bits 0..i), windows, rows that see no    */
/* draft.  A row that sees no token at all, or whose scores are all          */
/* -infinity, gives zeros.  A cached value of a token that a row does not    */
/* see never reaches it, finite or not.                                      */
/*                                                                           */
/* Layouts: q, out [total_q, n_q_heads, 128] bf16, rows packed as q_start   */
/* says; tree_mask [total_q, mask_words] 64-bit words, 8-byte aligned; the  */
/* rest as for chunked_prefill_attention.  A caller promise: n <= T and     */
/* n <= 64 * mask_words.  Values that break it are clamped: no access        */
/* leaves the buffers, rows past the clamped n are left unwritten.  An       */
/* offset of q_start below one before it counts as the largest so far, so    */
/* that no row belongs to two sequences.                                      */
/* Probabilities enter the second product as bf16 (the denominator sums the */
/* rounded ones); everything else is fp32 until out is rounded.              */
/*   workspace >= tree_decode_workspace_size(shape) bytes, 256-byte aligned, */
/*   of any content; calls that share one must not overlap in time.  q, out  */
/*   and workspace do not overlap (DP_EINVAL where they start together).      */
/* Results are deterministic.  At most two launches; nothing is allocated.  */
/* Supported: head_dim 128, block_size 16, Hq a multiple of Hkv,            */
/* batch <= 4096, mask_words 1..4, Hq / Hkv <= 1024.                        */
/* ------------------------------------------------------------------------ */
typedef struct {
  int32_t batch;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t block_size;
  int32_t max_blocks_per_seq;
  int32_t max_context_len;
  int32_t kv_dtype;   /* DP_KV_*                              */
  int32_t mask_words; /* 64-bit words of a row of tree_mask   */
  int32_t reserved;   /* must be 0                            */
  int64_t total_q;    /* rows of q, out and tree_mask         */
  int64_t num_blocks; /* blocks in k_blocks / v_blocks        */
} dp_tree_shape;

/* Bytes of workspace tree_decode_attention needs for this shape.  Returns 0
 * for invalid shapes (the reason is in dp_last_error()). */
size_t tree_decode_workspace_size(const dp_tree_shape* shape);

/* Enqueue the attention on `stream`.  DP_EINVAL / DP_ENOTSUP for bad
 * arguments, DP_ENOMEM for a short workspace (nothing enqueued); DP_EIO if a
 * launch fails. */
int tree_decode_attention(const void* q, const void* k_blocks, const void* v_blocks,
                          const int32_t* block_tables, const int32_t* context_lens,
                          const int32_t* q_start, const uint64_t* tree_mask, float scale,
                          const float* k_scale, const float* v_scale, void* out,
                          const dp_tree_shape* shape, void* workspace, size_t workspace_bytes,
                          void* stream);

/* ------------------------------------------------------------------------ */
/* Accepted drafts kept in the cache (device, asynchronous).                */
/*                                                                           */
/* After the model has checked a tree, one path of it is accepted.  Its     */
/* tokens lie scattered among the n drafted slots of the cache; this call   */
/* moves them to the front of those slots, in every layer's cache at once:  */
/* for sequence s (T, n as for tree_decode_attention) and j < a:            */
/*   K and V of token T - n + j = those of token T - n + accepted[s][j]     */
/*   context_lens_out[s] = T - n + a                                         */
/* a is n_accepted[s], cut at max_accept, at n, and at the first entry that */
/* is not larger than the one before it or not in [0, n).  n_accepted[s] < 0 */
/* leaves the sequence alone, context_lens_out[s] = T (for one that          */
/* kv_tables_step refused: it has rows, but no cached drafts).  Codes are    */
/* moved as they are.  A token whose block id is outside the pool is not     */
/* moved.  Offsets of q_start out of order, a broken promise, are clamped    */
/* pair by pair here: n may differ from the attention's then.                */
/*   k_layers, v_layers  host arrays of n_layers device pointers, caches as */
/*                       for kv_cache_append, all of one shape, no two the  */
/*                       same (DP_EINVAL); read during the call only         */
/*   accepted [batch, max_accept] int32, n_accepted [batch] int32;          */
/*   context_lens_out [batch] int32, none of the inputs (DP_EINVAL)          */
/*   shape  mask_words is not looked at                                      */
/* Blocks that hold drafts belong to one sequence, and nothing else writes  */
/* to them meanwhile: their V tiles are written whole.                       */
/* One launch per 64 layers (n_layers 1 to 1024); nothing is allocated.     */
/* DP_EINVAL / DP_ENOTSUP for bad arguments (nothing enqueued), DP_EIO if a */
/* launch fails.                                                             */
/* ------------------------------------------------------------------------ */
int kv_cache_accept(void* const* k_layers, void* const* v_layers, int32_t n_layers,
                    const int32_t* block_tables, const int32_t* context_lens, const int32_t* q_start,
                    const int32_t* accepted, const int32_t* n_accepted, int32_t max_accept,
                    int32_t* context_lens_out, const dp_tree_shape* shape, void* stream);

/* ------------------------------------------------------------------------ */
/* HBM read probe (device, asynchronous; measurement only).                 */
/*                                                                           */
/* Decode attention is bound by the rate at which the cached K and V can be */
/* read (Sec. 3 effect 4; Sec. 4.4).  This call reads device memory as a    */
/* plain read would, so that the decode kernel's bandwidth can be set       */
/* against what this device reaches, beside its published peak:             */
/*   tile_ids == NULL: every byte of buf[0, bytes) once, the grid sweeping   */
/*                     it front to back (n_tiles must be 0);                 */
/*   tile_ids != NULL: the 4 KiB tiles buf + 4096 * tile_ids[i],             */
/*                     i = 0 .. n_tiles-1, in list order (the decode's       */
/*                     (block, KV head) tile reads); ids are clamped into    */
/*                     [0, bytes / 4096).                                    */
/* buf and bytes are 16-byte multiples; workgroups (of 256 threads) sets    */
/* the launch width; sink holds at least `workgroups` int32 and is written   */
/* only in the practically impossible case that a workgroup's folded data   */
/* equals a fixed constant (it exists so the loads cannot be elided).       */
/* One launch on `stream`; DP_EINVAL for bad arguments (nothing enqueued),  */
/* DP_EIO if the launch fails.  The caller owns every buffer.               */
/* ------------------------------------------------------------------------ */
int dp_hbm_read_probe(const void* buf, size_t bytes, const int32_t* tile_ids, int64_t n_tiles,
                      int32_t workgroups, int32_t* sink, size_t sink_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DPOOL_H */
