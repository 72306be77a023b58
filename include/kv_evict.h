/*
 * kv_evict.h -- C ABI of the GB300 (sm_103a) diversified KV-eviction step.
 *
 * The step is the end-of-prefill token eviction of "Beyond Mean Attention:
 * Diversity-Aware, Layer-Wise Scoring for KV Cache Eviction" (Section 3). For every
 * (request, layer, KV head) -- a "unit" -- it
 *   1. scores every prefix token i by the attention A[q][i] it receives from the
 *      observation window, the last W query positions (Section 3.1, Eq. 1);
 *   2. reduces those scores over the window rows to the mean mu_i (Eq. 1) and the
 *      sample standard deviation sigma_i (Eq. 3);
 *   3. max-pools mu and sigma over the candidate tokens (Section 3.1 keeps the
 *      baselines' max-pooling), forms the base score s_i = mu_i + lambda1 * sigma_i
 *      (Eq. 2 without the redundancy term), restricts the candidates to the top
 *      4B tokens by s (Section 3.2), normalises s by its maximum (Eq. 5) and admits
 *      B tokens greedily by s~_i + lambda2 * corr(i, S) (Eq. 4, Eq. 5);
 *   4. gathers the kept key/value rows into a compact cache.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  * Symbols: N_L layers, Hq query heads, Hkv KV heads, G = Hq / Hkv (GQA group),
 *    d = head_dim, W = window, B = budget, n_req requests with prefix lengths L_r,
 *    SL = sum_r L_r, Lc_r = L_r - W candidate tokens of request r.
 *  * The window rows of unit (r, l, h) are the G query heads h*G .. h*G+G-1, each
 *    with its W window queries: n = G*W rows, row index g*W + w, at token position
 *    L_r - W + w. Causal masking: that row attends to keys 0 .. L_r - W + w.
 *  * All tensors are row-major, in device memory, allocated and owned by the
 *    caller; all but k and v are dense. bf16 tensors are passed as uint16_t bit
 *    patterns.
 *      q_win  [N_L][n_req][Hq][W][d]      bf16  window queries (after RoPE)
 *      k, v   [N_L][Hkv][SL][d]           bf16  prefix keys/values (after RoPE);
 *                                               request r occupies tokens
 *                                               off_r .. off_r + L_r - 1,
 *                                               off_r = L_0 + ... + L_{r-1}.
 *                                               Dense by default; any other
 *                                               strides between layers, heads and
 *                                               tokens through
 *                                               kv_evict_plan_set_kv_strides
 *      mu, sigma  packed per request: request r holds [N_L][Hkv][L_r] fp32 at
 *                 element offset N_L*Hkv*off_r
 *      indices    [n_req][N_L][Hkv][B] int32, kept candidate positions in
 *                 ascending order, -1 after the first min(B_l, Lc_r) entries
 *                 (B_l = B unless the plan has per-layer budgets, see
 *                 kv_evict_plan_layered)
 *      order      [n_req][N_L][Hkv][B] int32, the same positions in admission
 *                 order (optional)
 *      margins    [n_req][N_L][Hkv][B] fp32, per admission the gap between the
 *                 best and the second-best greedy value (optional)
 *      k_out, v_out [n_req][N_L][Hkv][B+W][d] bf16: rows 0 .. m-1 are the kept
 *                 candidates in ascending position (m = min(B_l, Lc_r)), rows
 *                 m .. m+W-1 the W window tokens, remaining rows zero.
 *  * Every pointer must be 16-byte aligned; q_win and k additionally 128-byte.
 *  * stream is a cudaStream_t passed as void*. Every device call is
 *    asynchronous on that stream and returns after the launches; device-side
 *    failures (a bounded wait that ran out) are reported by kv_evict_status.
 *  * Host validation failures return before any launch and write nothing.
 *  * A plan is immutable after kv_evict_plan and may be used from several host
 *    threads; a workspace must not be shared by calls that overlap on the GPU.
 */
#ifndef KV_EVICT_H
#define KV_EVICT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  KVE_OK = 0,
  KVE_EINVAL = 1,   /* invalid argument or unsupported shape (host check)     */
  KVE_ECUDA = 2,    /* a CUDA runtime/driver call failed                      */
  KVE_ETIMEOUT = 3, /* a device-side bounded wait ran out (kv_evict_status)   */
  KVE_ENOMEM = 4,   /* host allocation failed                                 */
  KVE_EPAGES = 5    /* too few free pages (kv_evict_cache_status)             */
} kve_status;

typedef struct {
  int32_t num_layers;       /* N_L >= 1                                        */
  int32_t num_q_heads;      /* Hq, a multiple of num_kv_heads                  */
  int32_t num_kv_heads;     /* Hkv >= 1                                        */
  int32_t head_dim;         /* d; this build supports d = 128                  */
  int32_t window;           /* W >= 1, with G*W <= 128                         */
  int32_t budget;           /* B >= 1 kept candidates per unit (the window is
                               kept in addition)                               */
  int32_t pool_kernel;      /* odd k, 1 <= k <= 255; max-pool of mu and sigma,
                               stride 1, window clipped to [0, Lc); 1 = none    */
  int32_t candidate_factor; /* greedy pool C = min(factor*B, Lc); Section 3.2
                               uses 4; 0 = every candidate                     */
  float norm_eps;           /* positive clamp of max_j s_j in Eq. 5            */
} kve_config;

typedef struct kve_plan kve_plan;

/* Validate cfg and the host array seq_lens[n_req] (every L_r > W), and build the
 * host-side schedule. *workspace_bytes receives the size of the device workspace
 * that kv_evict_score and kv_evict_select need (caller-allocated, 256-byte
 * aligned). The plan owns host memory only. Section 3 defines the shapes. */
kve_status kv_evict_plan(const kve_config* cfg, const int64_t* seq_lens,
                         int32_t n_req, kve_plan** plan_out,
                         size_t* workspace_bytes);

/* kv_evict_plan with a budget per layer: layer_budgets is a HOST array [N_L] with
 * 1 <= B_l <= cfg->budget; layer l keeps min(B_l, Lc_r) candidates (candidate pool
 * min(factor * B_l, Lc_r)). cfg->budget stays the row stride of indices, order,
 * margins (B) and of the compact cache (B + W). PyramidKV (Section 3.1) decreases
 * the budget with depth while keeping the total of the uniform allocation; see
 * kv_evict_budget_pyramid. layer_budgets = NULL is kv_evict_plan. */
kve_status kv_evict_plan_layered(const kve_config* cfg, const int64_t* seq_lens,
                                 int32_t n_req, const int32_t* layer_budgets,
                                 kve_plan** plan_out, size_t* workspace_bytes);

/* Flags of kv_evict_plan_ex. */
#define KVE_PLAN_PER_QUERY_HEAD 1

/* kv_evict_plan_layered with flags (0 = kv_evict_plan_layered).
 * KVE_PLAN_PER_QUERY_HEAD: every query head selects its own tokens. The paper leaves
 * the GQA grouping open; the default pools the G*W window rows of the query heads
 * that share a KV head into one unit (n = G*W rows, one selection per KV head).
 * With this flag a unit is (request, layer, query head): its n = W rows are that
 * head's window queries, its keys those of its KV head (query head hq reads KV head
 * hq / G), and the selection, the compact cache and every per-unit array are
 * indexed by query head: mu, sigma [n_req][N_L][Hq][L_r]; indices, order, margins
 * [n_req][N_L][Hq][B]; k_out, v_out [n_req][N_L][Hq][B+W][d]. Inputs keep their
 * layouts. Other flag bits: KVE_EINVAL. */
kve_status kv_evict_plan_ex(const kve_config* cfg, const int64_t* seq_lens,
                            int32_t n_req, const int32_t* layer_budgets,
                            int32_t flags, kve_plan** plan_out,
                            size_t* workspace_bytes);

void kv_evict_plan_destroy(kve_plan* plan);

/* Layout of k and v for later calls with this plan, so that a serving engine's cache
 * is read in place: strides[3] = element strides between layers, KV heads and
 * tokens (in that order) of the prefix keys (k_strides) and values (v_strides);
 * element (layer l, KV head h, token t, dim j) sits at l*s[0] + h*s[1] + t*s[2] + j,
 * with t = off_r + i for key i of request r (off_r as above). A row of d elements
 * stays contiguous. NULL is the dense default {Hkv*SL*d, SL*d, d}; a token-major
 * cache [N_L][SL][Hkv][d] is {SL*Hkv*d, d, Hkv*d}. Every stride must be a multiple
 * of 8 elements (16 bytes) and below 2^37, and the token stride at least d;
 * otherwise KVE_EINVAL and the plan is unchanged. Call it before the plan is used
 * on any stream; it changes the plan (not thread-safe with calls that use it). */
kve_status kv_evict_plan_set_kv_strides(kve_plan* plan, const int64_t* k_strides,
                                        const int64_t* v_strides);

/* Test hook: limit (ns) of every device-side bounded wait of later calls with this
 * plan (default 2e9), and a fault to inject on the host-chosen unit 0:
 * fault = 1 makes its row statistics never publish, so its column pass waits
 * out the limit and kv_evict_status reports KVE_ETIMEOUT. fault = 0 is normal. */
kve_status kv_evict_plan_set_debug(kve_plan* plan, uint64_t wait_limit_ns,
                                   int32_t fault);

/* Steps 1-2: window attention (Section 3.1 and Eq. 1 context: softmax of the
 * scaled window-query/key logits over the whole causal prefix, window keys
 * included), then per token mu (Eq. 1) and sigma (Eq. 3, divisor n - 1; sigma = 0
 * when n = 1) for every token 0 .. L_r - 1 of every unit. Reads q_win and k,
 * writes mu and sigma, uses ws as scratch. */
kve_status kv_evict_score(const kve_plan* plan, const uint16_t* q_win,
                          const uint16_t* k, float* mu, float* sigma, void* ws,
                          void* stream);

/* Steps 1-2 as kv_evict_score when the softmax normaliser of every window row is
 * already known -- a prefill attention kernel computes it for its own output (Section
 * 3.2 scores with the prefill's existing attention). lse [N_L][n_req][Hq][W] fp32 in
 * q_win's row order (device memory) holds, for the row at position L_r - W + w,
 *   lse = ln sum_{i <= L_r - W + w} exp(q . k_i / sqrt(d))   (natural log),
 * so that A[r][i] = exp(q . k_i / sqrt(d) - lse). The library then needs only the
 * column pass of Eq. 1 and Eq. 3 over the prefix: one pass of the score kernel
 * instead of two. mu and sigma are exactly as accurate as lse is; a row's lse that is
 * not finite makes its terms undefined. Reads q_win, k and lse; writes mu and sigma;
 * uses ws as scratch. */
kve_status kv_evict_score_lse(const kve_plan* plan, const uint16_t* q_win,
                              const uint16_t* k, const float* lse, float* mu,
                              float* sigma, void* ws, void* stream);

/* Steps 1-2 as kv_evict_score, together with the window rows' own attention output.
 * Section 3.2 scores the tokens with the prefill's existing attention; the window rows'
 * attention (the last W positions of every query head) is computed here anyway, so in
 * the same pass over the prefix the library also streams V and returns
 *   O[r] = sum_i A[r][i] * v_i      (A of Eq. 1: causal softmax over the prefix)
 * for every window row, and a caller's prefill can skip attention for those rows.
 * o_win has q_win's layout, [N_L][n_req][Hq][W][d] bf16 (with KVE_PLAN_PER_QUERY_HEAD
 * the same). v follows the plan's v strides. mu and sigma are those of kv_evict_score.
 * Precision: A enters the value product as bf16 (relative error <= 2^-8 per
 * probability), accumulated in fp32, and O is rounded to bf16 once, so
 * |O - O_exact| <= 2^-8 (sum_i A[r][i] |v_i| + |O|) elementwise. attn_ws is a
 * second scratch buffer (256-byte aligned) of kv_evict_score_attn_workspace bytes
 * (fp32 partial outputs, 64 KB per score work item). v must be 128-byte aligned. */
kve_status kv_evict_score_attn(const kve_plan* plan, const uint16_t* q_win,
                               const uint16_t* k, const uint16_t* v, float* mu,
                               float* sigma, uint16_t* o_win, void* ws,
                               void* attn_ws, void* stream);

/* *bytes = the attn_ws size of kv_evict_score_attn for this plan. */
kve_status kv_evict_score_attn_workspace(const kve_plan* plan, size_t* bytes);

/* Step 3: pooling (Section 3.1), base score (Eq. 2), top factor*B candidate pool
 * (Section 3.2), normalisation (Eq. 5, denominator clamped to norm_eps), greedy
 * admission by s~ + lambda2 * corr(i, S) (Eq. 4, Eq. 5) with ties broken towards
 * the lower token position. lambda1 and lambda2 are HOST arrays [N_L] (the
 * layer-wise coefficients of Section 3.3). Writes indices; order and margins may
 * be NULL. Uses ws as scratch. */
kve_status kv_evict_select(const kve_plan* plan, const float* mu,
                           const float* sigma, const uint16_t* k,
                           const float* lambda1, const float* lambda2,
                           int32_t* indices, int32_t* order, float* margins,
                           void* ws, void* stream);

/* Steps 3 and 4 in one launch: exactly what kv_evict_select followed by
 * kv_evict_gather writes (indices, order, margins, k_out, v_out; the same arguments
 * and the same layouts), with the compact cache written by the selection's own CTA
 * for each unit. Beside the values and the window rows it reads the kept key rows a
 * second time where the candidate pool is 256 at most (they are in L2, just read for
 * the cosines of Eq. 4; larger pools still hold them in shared memory). v may be
 * page-locked host memory as for kv_evict_gather (and k as well: its pool's rows, its
 * kept rows and its window rows then cross the host link). Returns KVE_EINVAL
 * on the conditions of either call. For a plan whose selection runs over every
 * candidate (candidate_factor 0 beyond 512 prefix tokens) the two steps stay two
 * launches. */
kve_status kv_evict_select_gather(const kve_plan* plan, const float* mu,
                                  const float* sigma, const uint16_t* k,
                                  const uint16_t* v, const float* lambda1,
                                  const float* lambda2, int32_t* indices,
                                  int32_t* order, float* margins,
                                  uint16_t* k_out, uint16_t* v_out, void* ws,
                                  void* stream);

/* Step 3 for n_profiles profiles of the layer-wise coefficients in one pass over
 * the units (Section 3.3 searches over profiles and re-selects for each; mu and
 * sigma do not depend on the coefficients, so one kv_evict_score serves them all).
 * lambda1 and lambda2 are HOST arrays [n_profiles][N_L]; profile p selects exactly
 * what kv_evict_select selects with lambda1 + p*N_L and lambda2 + p*N_L. Outputs are
 * stacked by profile: indices [n_profiles][n_units][B]; order and margins likewise
 * (either may be NULL). ws is a separate scratch buffer (256-byte aligned) of
 * kv_evict_select_profiles_workspace bytes, not the plan's workspace; its first word
 * is this call's error word (cleared by the call, read by kv_evict_status(plan, ws,
 * stream)). One launch
 * carries 6144 / (2 N_L) profiles (96 for N_L = 32); more go to further launches on
 * stream. Returns KVE_EINVAL for n_profiles < 1 or a non-finite coefficient, before
 * any launch. */
kve_status kv_evict_select_profiles(const kve_plan* plan, int32_t n_profiles,
                                    const float* mu, const float* sigma,
                                    const uint16_t* k, const float* lambda1,
                                    const float* lambda2, int32_t* indices,
                                    int32_t* order, float* margins, void* ws,
                                    void* stream);

/* *bytes = scratch of kv_evict_select_profiles for n_profiles profiles: a 256-byte
 * header holding the error word, then 4 bytes per prefix token per unit per profile. */
kve_status kv_evict_select_profiles_workspace(const kve_plan* plan,
                                              int32_t n_profiles, size_t* bytes);

/* Step 3 without a workspace. The paper has no counterpart: this entry point
 * exists for callers that cannot allocate device memory at eviction time --
 * serving engines that reserve nearly all of HBM for their own KV-cache pool and
 * hand kernels only pointers into it, or plugin hosts that give a kernel nothing
 * but its inputs and outputs. It computes exactly what kv_evict_select computes,
 * with the same arguments except ws; its scratch (4 bytes per prefix token per
 * unit) is a 16 MiB array compiled into the library, which every GPU that loads
 * the library keeps reserved until the process exits. It allocates nothing.
 *  * Returns KVE_EINVAL when N_L * U * SL exceeds 4194304 (16 MiB / 4 B), where U
 *    is the number of units per layer: Hkv, or Hq for a KVE_PLAN_PER_QUERY_HEAD
 *    plan. E.g. a 32-layer, 8-KV-head request of more than 16384 tokens, or a
 *    per-query-head plan with 32 layers and 32 query heads beyond 4096 tokens.
 *  * Device-side check failures go to an error word that the library keeps beside
 *    the array: kv_evict_status(plan, NULL, stream) reads and clears it.
 *  * The first call on a device looks up the array's device address on that
 *    device (cudaGetSymbolAddress); make that first call before any stream
 *    capture on the device.
 *  * All calls share the one array and each call overwrites it before reading it.
 *    Calls whose executions overlap on the GPU (for example on two streams at
 *    once) race on it and give undefined results; serialise them. */
kve_status kv_evict_select_noalloc(const kve_plan* plan, const float* mu,
                                   const float* sigma, const uint16_t* k,
                                   const float* lambda1, const float* lambda2,
                                   int32_t* indices, int32_t* order,
                                   float* margins, void* stream);

/* Step 4: compact cache (Section 1: each layer keeps B entries after prefill;
 * the window tokens are kept as well). Copies key/value rows bit-exactly.
 * Exception to the device-memory convention: k and v may also be page-locked
 * host memory of the CUDA runtime (cudaHostAlloc, cudaMallocHost, or host memory
 * registered with cudaHostRegister). Under unified addressing the kernel reads
 * such memory in place, and only the kept rows (min(B_l, Lc_r) + W per unit)
 * cross the host link. k_out and v_out stay in device memory. Returns KVE_EINVAL
 * for host memory the runtime does not know (pageable memory) or a pointer the
 * runtime cannot classify. */
kve_status kv_evict_gather(const kve_plan* plan, const uint16_t* k,
                           const uint16_t* v, const int32_t* indices,
                           uint16_t* k_out, uint16_t* v_out, void* stream);

/* Synchronise the stream, read the device error word of ws and clear it. ws is the
 * plan's workspace, the scratch of kv_evict_select_profiles, or NULL for the error
 * word of kv_evict_select_noalloc on the current device.
 * Returns KVE_OK, KVE_ETIMEOUT (a bounded wait ran out) or KVE_ECUDA (a CUDA call
 * failed, or a device-side consistency check of the selection failed: a candidate
 * pool that did not hold exactly C positions -- that unit then reports no
 * selection, indices -1 -- or a pool position outside the unit, whose key row is
 * then not read). */
kve_status kv_evict_status(const kve_plan* plan, void* ws, void* stream);

/* Depth profile of Eq. 6 on the host: kind 0 Global (lambda = sinh(c[0]) on every
 * layer), 1 Segments (sinh(c[0]), sinh(c[1]), sinh(c[2]) on layers
 * [0, b0), [b0, b1), [b1, N_L), with seg_bounds = {b0, b1}, or thirds when
 * seg_bounds is NULL), 2 Curve (sinh(c0 + c1 t + c2 t^2), t = l / (N_L - 1)).
 * Writes lambda_out[num_layers]. */
kve_status kv_evict_profile(int32_t kind, const float* c, int32_t num_layers,
                            const int32_t* seg_bounds, float* lambda_out);

/* A depth-decreasing budget schedule with the total of the uniform one (Section 3.1
 * states only these two properties of PyramidKV's allocation; this function is a
 * reading of it): budgets_out[l] (HOST, [num_layers]) falls linearly with depth
 * from 2B - b to b, b = max(1, floor(last_ratio * B)), rounded down and the
 * remainder given one each to the shallowest layers, so that the budgets are
 * non-increasing and sum to num_layers * B. last_ratio = 1 is uniform. The
 * largest budget is budgets_out[0]: pass it as cfg->budget. Returns KVE_EINVAL
 * unless B >= 1, num_layers >= 1 and 0 < last_ratio <= 1. */
kve_status kv_evict_budget_pyramid(int32_t budget, int32_t num_layers,
                                   float last_ratio, int32_t* budgets_out);

/* ------------------------------------------------------------------------------------
 * The paged 8-bit cache: what a serving program decodes from after an eviction.
 *
 * A sequence's compact cache is kept in 8 bits, in pages of P tokens that a block table
 * names, and grows as the model answers. Four calls work on it:
 *   kv_evict_cache_pages   pages taken and released, and the slots of new tokens, from
 *                          the sequences' old and new lengths (on the GPU);
 *   kv_evict_cache_gather  step 4 into the cache: the kept and the window rows;
 *   kv_evict_cache_store   new tokens' key and value rows, written by slot;
 *   kv_evict_cache_attend  attention of new tokens' queries over one layer's sequences.
 *
 *  * H = num_kv_heads is the number of heads whose rows the cache holds: the KV heads,
 *    or the query heads for a KVE_PLAN_PER_QUERY_HEAD plan (then num_q_heads = H).
 *    Query head hq reads cache head hq / G, G = num_q_heads / H. S = max_seqs.
 *  * Pages:  k, v [num_pages][H][P][d] uint8, e4m3 codes (1 sign, 4 exponent, 3 fraction
 *    bits, largest 448, no infinities); k_scale, v_scale [num_pages][H] fp32. A cached
 *    value is its code's value times the scale of its page and head. The pages are shared
 *    by all layers.
 *  * Scales are powers of two: need(a) is the smallest 2^e, e >= -126, with a <= 448 * 2^e
 *    for the largest finite magnitude a of the rows that share it. A code is the value
 *    divided by the scale, rounded to the nearest (ties to even); infinities become the
 *    largest code of their sign, NaN stays NaN. A power of two loses at most one of the 18
 *    binades that a code spans and none of its fraction bits, and a page whose scale grows
 *    keeps its older codes exactly, but for those that become subnormal.
 *  * table [N_L][S][max_pages] int32: page j of a sequence holds its tokens j*P ..
 *    j*P + P - 1. Entries at and behind ceil(len / P) are not read. Position i of a
 *    sequence is slot table[i / P] * P + i % P.
 *  * lens [N_L][S] int32: tokens in the cache, 0 .. max_pages * P; budgets may differ by
 *    layer, so lengths do.
 *  * The workspace ws (256-byte aligned) belongs to one cache and is cleared once by
 *    kv_evict_cache_reset; calls that use it must not overlap on the GPU. Page numbers and
 *    slots outside the pool are never followed: the call leaves those tokens out and
 *    reports KVE_ECUDA through kv_evict_cache_status.
 *  * The handle holds the addresses of k, v, k_scale and v_scale; it is immutable. A call
 *    made while another device than theirs is current returns KVE_EINVAL.
 * ---------------------------------------------------------------------------------- */
typedef struct {
  int32_t num_layers;       /* N_L, 1 .. 256                                   */
  int32_t num_q_heads;      /* a multiple of num_kv_heads, G <= 128            */
  int32_t num_kv_heads;     /* H, 1 .. 1024                                    */
  int32_t head_dim;         /* d; this build supports d = 128                  */
  int32_t page_tokens;      /* P: 16, 32, 64 or 128                            */
  int32_t num_pages;        /* pages in the pool, num_pages * H * P < 2^31     */
  int32_t max_pages;        /* pages of one sequence, 1 .. num_pages           */
  int32_t max_seqs;         /* S, 1 .. 1024                                    */
} kve_cache_config;

typedef struct kve_cache kve_cache;

/* A cache of cfg over device buffers of one device that the caller owns (k and v 128-byte,
 * the scales 16-byte aligned; nothing is written; KVE_EINVAL where one of them is host
 * memory or another device's; where the CUDA runtime knows none of them, they are taken
 * as they are). The handle owns host memory only.
 * *workspace_bytes receives the size of ws. */
kve_status kv_evict_cache_create(const kve_cache_config* cfg, uint8_t* k, uint8_t* v,
                                 float* k_scale, float* v_scale, kve_cache** cache_out,
                                 size_t* workspace_bytes);

void kv_evict_cache_destroy(kve_cache* cache);

/* Clears ws, and where free_pages and ring are given makes every page free:
 * free_pages [num_pages] = 0, 1, .., ring [2] = {0, num_pages}. Both or neither. */
kve_status kv_evict_cache_reset(const kve_cache* cache, int32_t* free_pages, int32_t* ring,
                                void* ws, void* stream);

/* Pages and slots of every sequence, from lens_from to lens_to (each [N_L][S], device
 * memory). free_pages [num_pages] is a ring of page numbers, ring_in = {head, count}: the
 * free pages are entries head .. head + count - 1 modulo num_pages. In the order (layer,
 * sequence, page), a sequence that grows takes ceil(to / P) - ceil(from / P) pages from the
 * ring's head into its table row, one that shrinks gives its last pages to the ring's tail
 * (their table entries stay as they were). ring_out and lens_out (= lens_to) receive the
 * state after the call. Pages released here can be taken from the next call on.
 * slots (or NULL) [N_L][slot_stride] receives per layer the slots of the new tokens
 * (positions from .. to - 1 where to > from), packed in sequence order, -1 behind them: the
 * slots argument of kv_evict_cache_store for that layer.
 * All or nothing: if the free pages do not suffice (KVE_EPAGES), or a length or the ring is
 * out of range, or a layer has more than slot_stride new tokens (KVE_ECUDA), no page moves,
 * lens_out = lens_from, ring_out = ring_in, every slot is -1, and kv_evict_cache_status
 * tells. ring_out may be ring_in, and lens_out may be lens_from or lens_to, so that one
 * captured graph can advance its own state. Tables are int32 throughout and the call
 * neither synchronises nor allocates. */
kve_status kv_evict_cache_pages(const kve_cache* cache, const int32_t* lens_from,
                                const int32_t* lens_to, int32_t* table, int32_t* free_pages,
                                const int32_t* ring_in, int32_t* ring_out, int32_t* lens_out,
                                int32_t* slots, int64_t slot_stride, void* ws, void* stream);

/* Step 4 into the cache: the rows that kv_evict_gather would copy for the plan's request r,
 * in its order (kept candidates ascending, then the window rows), become positions 0 ..
 * m + W - 1 of sequence first_seq + r of every layer, in 8 bits. The table rows of those
 * sequences hold the pages (kv_evict_cache_pages with lens_to = m + W). Rows of the last
 * page behind the sequence are left as they were. A kept index outside 0 .. Lc_r - 1 (a
 * selection that gave up leaves -1) becomes a row of zeros, and kv_evict_cache_status
 * returns KVE_ECUDA. Nothing is written where the last
 * kv_evict_cache_pages call on ws moved no page: what the table then names can be another
 * sequence's. k, v and indices as for kv_evict_gather
 * (pinned host memory too); the plan and the cache have the same layers and heads. */
kve_status kv_evict_cache_gather(const kve_cache* cache, const kve_plan* plan,
                                 const uint16_t* k, const uint16_t* v, const int32_t* indices,
                                 int32_t first_seq, const int32_t* table, void* ws,
                                 void* stream);

/* Key and value rows of n_tokens new tokens of one layer, written by slot: token t's rows
 * go to slots[t]; a negative slot (a padded batch) writes nothing. k_new, v_new [n_tokens]
 * [H][d] bf16, 16-byte aligned, with element strides {token, head} (multiples of 8, not
 * negative; NULL is dense). Tokens of one page that the call writes stand together in
 * ascending order (as kv_evict_cache_pages packs them); a page written from two places of
 * the call gets undefined codes. A run of tokens that starts at row 0 of a page sets its scale to
 * need of its rows; one that starts later keeps the larger of need and the page's scale,
 * and where that grows, the page's older rows are rounded to it once more. Making the same
 * call again changes nothing. n_tokens < 2^20; with 0 of them nothing is done. */
kve_status kv_evict_cache_store(const kve_cache* cache, const uint16_t* k_new,
                                const uint16_t* v_new, const int64_t* k_strides,
                                const int64_t* v_strides, const int32_t* slots,
                                int64_t n_tokens, void* ws, void* stream);

/* Attention of layer `layer`: q_tokens (T >= 1, G * T <= 128) queries of each of the
 * sequences 0 .. n_seq - 1, whose keys and values are in the cache already. Query t of a
 * sequence of length len stands at position len - T + t and sees the positions up to its
 * own:  out = sum_i softmax(q . k_i / sqrt(d)) v_i.  A query that sees nothing (len < T - t, an
 * empty sequence) gets zeros and lse = -inf. Rows of sequences behind n_seq are left as
 * they were. q, out [n_seq * T][Hq][d] bf16, 16-byte aligned, element strides {token, head}
 * (multiples of 8, not negative; NULL is dense; out's rows must not overlap; out may be q
 * with the same strides). lse (or NULL)
 * [n_seq * T][Hq] fp32: ln sum_i exp(q . k_i / sqrt(d)). The table and lens of every layer
 * are passed; layer picks. What the pages hold behind a sequence, NaN codes included, has
 * no part in its rows. A query row with an infinity or a NaN gives NaN.
 * Statistics and sums are fp32. What is held in fewer bits: a query element below 2^-13 of
 * its row's largest to 2^-21 of that; a probability times its page's value scale to 2^-12
 * of itself, or to 2^-26 of the largest such product among the tokens of its tile
 * (positions 128 j .. 128 j + 127) that the row sees, whichever is more; an output to
 * len * 2^-133. */
kve_status kv_evict_cache_attend(const kve_cache* cache, int32_t layer, int32_t n_seq,
                                 int32_t q_tokens, const uint16_t* q, const int64_t* q_strides,
                                 const int32_t* table, const int32_t* lens, uint16_t* out,
                                 const int64_t* out_strides, float* lse, void* ws,
                                 void* stream);

/* ------------------------------------------------------------------------------------
 * Rotary positions: the rotation that the queries and keys of this library have behind them ("after
 * RoPE"), and that new ones still need. Behind an eviction a token's position is no longer its
 * place in the cache, so positions are an input of every call.
 *
 *  * Pair j = 0 .. n/2 - 1 of the first n = rotary_dim elements of a row, (x_j, x_{j + n/2}), or
 *    (x_2j, x_{2j+1}) where interleaved, becomes
 *      A (a cos t - b sin t),  A (b cos t + a sin t),  t = position * frequencies[j];
 *    the elements behind n stay as they are. For frequencies below 2^62 in magnitude angles are exact
 *    to 2^-31 of a turn at every int32 position (negative ones too); cos and sin to 2^-23 beside that;
 *    results are rounded once to bf16.
 *  * The transpose, A (a cos t + b sin t), A (b cos t - a sin t), is the gradient of that, and with
 *    A = 1 takes it out again.
 * ---------------------------------------------------------------------------------- */
#define KVE_ROTARY_NONE 0     /* base^(-2j/n)                                                    */
#define KVE_ROTARY_LINEAR 1   /* that over factor                                                */
#define KVE_ROTARY_NTK 2      /* with base * factor^(n/(n-2)): the slowest pair factor times slower */
#define KVE_ROTARY_PARTS 3    /* pairs of low_turns or fewer turns within original_length over factor,
                                 those of high_turns or more as they are, linear in the turns between */
#define KVE_ROTARY_YARN 4     /* the same, linear in j between the pairs that make high_turns (rounded
                                 down) and low_turns (up); A = 1 + 0.1 ln factor                 */

typedef struct kve_rotary kve_rotary;

/* Frequencies [rotary_dim / 2] in radians a position, and A, of one of the forms above (host). base > 1;
 * factor >= 1 (but for NONE); original_length >= 1 and 0 < low_turns < high_turns for PARTS and
 * YARN, else not read. */
kve_status kv_evict_rotary_frequencies(int32_t kind, int32_t rotary_dim, double base, double factor,
                                       double original_length, double low_turns, double high_turns,
                                       double* frequencies, double* amplitude);

/* A rotation of rows of head_dim = 128 elements whose first rotary_dim (a multiple of 16, 16 .. 128)
 * turn, by the given finite frequencies (host), A = amplitude (|A| <= 1e30). The handle owns host
 * memory only, is immutable, and serves every device and stream; calls copy what they need of it. */
kve_status kv_evict_rotary_create(int32_t head_dim, int32_t rotary_dim, int32_t interleaved,
                                  const double* frequencies, double amplitude, kve_rotary** rotary_out);

void kv_evict_rotary_destroy(kve_rotary* rotary);

/* x, out [n_tokens][heads][d] bf16, 16-byte aligned, with element strides {token, head} (multiples of 8,
 * not negative; NULL is dense; out's rows must not overlap): row (t, h) of out is that of x turned
 * by positions[t] (int32). x and positions may be pinned host memory. out may be x with the same
 * strides, or shares nothing with it. transpose: 0 or 1. n_tokens * heads < 2^31; with 0 tokens
 * nothing is done. KVE_EINVAL where out is host memory or another device's than the current one. */
kve_status kv_evict_rotary_apply(const kve_rotary* rotary, const uint16_t* x, const int64_t* x_strides,
                                 uint16_t* out, const int64_t* out_strides, int32_t heads,
                                 const int32_t* positions, int64_t n_tokens, int32_t transpose,
                                 void* stream);

/* kv_evict_cache_store with the rotation on the way, in one launch: the keys are turned by
 * positions [n_tokens] and rounded to bf16 before they are written, bit for bit as
 * kv_evict_rotary_apply and kv_evict_cache_store would one after the other; the values are written as
 * they are. With q and q_out (both or neither; [n_tokens][Hq][d], conditions as for
 * kv_evict_rotary_apply) the tokens' queries are turned too, those of negative slots among them.
 * q_out shares nothing with k_new and v_new. Works on 8-bit and 4-bit caches. */
kve_status kv_evict_cache_append(const kve_cache* cache, const kve_rotary* rotary, const int32_t* positions,
                                 const uint16_t* q, const int64_t* q_strides, uint16_t* q_out,
                                 const int64_t* q_out_strides, const uint16_t* k_new,
                                 const uint16_t* v_new, const int64_t* k_strides,
                                 const int64_t* v_strides, const int32_t* slots, int64_t n_tokens,
                                 void* ws, void* stream);

/* ------------------------------------------------------------------------------------
 * The paged cache in 4 bits: 68 bytes a row where the 8-bit cache has 128.
 *
 * A handle of kv_evict_cache4_create serves the calls of the 8-bit cache (kv_evict_cache_reset, _pages,
 * _gather, _store, _append, _attend, _status, _destroy), with the same tables, lengths, slots and
 * workspace, and these differences:
 *
 *  * Pages:  k, v [num_pages][H][P][d / 2] uint8: codes c in 0 .. 15, element 2i in the low and
 *    2i + 1 in the high half of byte i; k_param, v_param [num_pages][H][P][2] bf16: s and z of each
 *    row, an element being s c + z. (128-byte and 16-byte aligned.)
 *  * A row x is written as z = min x, s = RN_bf16(fl(fl((max x - min x) / 16) * fl(16 / 15))),
 *    c = fl(fl((x - z) / 16) / (s / 16)) rounded to the nearest integer (ties to even), fl to fp32;
 *    s = 0 and c = 0 where s would be below 2^-120. An element is off by at most 0.53 of a step s. A
 *    row with an infinity or a NaN becomes s = z = NaN, c = 0, and so NaN wherever it is seen.
 *  * Rows share nothing: a page may be written in any order, and a slot that a call names twice gets
 *    undefined codes (its row only).
 *  * Attention: l = (s (q . c) + z sum q) / sqrt(d), out = sum p s c + sum p z, statistics and sums in
 *    fp32. What is held in fewer bits: a query element below 2^-27 of its row's largest to 2^-35
 *    of that; p s to 2^-12 of itself, or to 2^-31 of the largest p s so far, whichever is more; the sum
 *    of p z to len * 2^-149. A p below 2^-126 of its row's largest may count as 0. A query row with an
 *    infinity, a NaN or a magnitude of 2^112 or more gives NaN.
 * ---------------------------------------------------------------------------------- */
kve_status kv_evict_cache4_create(const kve_cache_config* cfg, uint8_t* k, uint8_t* v, uint16_t* k_param,
                                  uint16_t* v_param, kve_cache** cache_out, size_t* workspace_bytes);

/* Synchronise the stream, read the error word of ws and clear it: KVE_OK, KVE_EPAGES (too
 * few free pages), KVE_ETIMEOUT (a bounded wait ran out) or KVE_ECUDA (a length, page, slot
 * or ring entry out of range, or a CUDA call failed). */
kve_status kv_evict_cache_status(const kve_cache* cache, void* ws, void* stream);

const char* kv_evict_strerror(kve_status status);

#ifdef __cplusplus
}
#endif

#endif /* KV_EVICT_H */
