/*
 * libseer -- C ABI of the Seer hot path on one GB300 (sm_103a).
 *
 * Seer (arXiv 2607.14557) detects, at denoising step 0, where the valid text
 * response of a diffusion multimodal LLM ends (Sec. 3.2-3.3), truncates the
 * padded suffix once, and runs every later layer and step over the ragged
 * sequences [visual prefix + prompt + truncated response] (Sec. 3.4-3.6).
 *
 * Conventions shared by every entry point:
 *  - Pointers marked "device" are CUDA device pointers owned by the caller.
 *    The library never allocates, frees or synchronises device memory except
 *    where an entry point says so (seer_check_device, seer_profile_read).
 *  - `stream` is a cudaStream_t passed as void*; all work is enqueued on it.
 *  - Matrices are row-major.  Weight matrices use the nn.Linear layout
 *    [out_features, in_features] (K-major for the tensor cores).
 *  - Argument checks that need only host values run before any launch and
 *    return SEER_ERR_INVALID_ARG / SEER_ERR_UNSUPPORTED with a message in
 *    seer_last_error().  Values that live on the device (row counts,
 *    cu_seqlens) are checked by the kernels, which record a code that
 *    seer_check_device() reports; a kernel never traps.
 *  - 16-bit work (bf16 / f16) runs on hand-written tcgen05/TMEM/TMA kernels
 *    and needs d_model % 256 == 0, d_ff % 128 == 0, head_dim == 128 and
 *    16-byte aligned pointers.  fp32 work (small shapes) runs on CUDA-core
 *    kernels and needs d_model % 8 == 0, head_dim <= 128, head_dim % 4 == 0.
 *  - Precision of a bf16 layer: its input x and output y are bf16, but its
 *    weights and every intermediate tensor are f16 (same tensor-core rate,
 *    three more mantissa bits) with fp32 accumulation.  A layer that stored
 *    its intermediates in bf16 misses |err| <= 1e-2 + 1e-2|ref| against the
 *    exact result on a few percent of outputs at d = 4096, F = 12288; with
 *    f16 intermediates it meets it.  Values must stay within the f16 range
 *    (|v| <= 65504): every 16-bit store of the GEMM, attention and RMSNorm
 *    kernels passes a range guard, and a value that overflowed to infinity
 *    (or is NaN) records device error code 6, which seer_check_device reports.
 *  - There is no CPU fallback: without a usable GPU every call fails with
 *    SEER_ERR_CUDA.
 */
#ifndef SEER_H
#define SEER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SEER_OK = 0,
  SEER_ERR_INVALID_ARG = 1,   /* a host-side argument is out of range or null */
  SEER_ERR_UNSUPPORTED = 2,   /* shape/alignment the kernels do not handle */
  SEER_ERR_WORKSPACE = 3,     /* workspace missing or smaller than required */
  SEER_ERR_CUDA = 4,          /* a CUDA runtime call failed (see seer_last_error) */
  SEER_ERR_TIMEOUT = 5,       /* seer_poll_ctrl gave up waiting */
  SEER_ERR_DEVICE = 6         /* a kernel recorded a device-side error */
} seer_status;

typedef enum { SEER_F32 = 0, SEER_BF16 = 1, SEER_F16 = 2 } seer_dtype;

/* Layer geometry.  A pre-norm block: RMSNorm -> QKV -> bidirectional MHA ->
 * O projection + residual -> RMSNorm -> SwiGLU MLP + residual.  The paper
 * does not spell out the block (it evaluates LLaDA-style backbones); this
 * LLaMA-style reading uses no biases.  The paper names no positional scheme:
 * rope_theta > 0 turns on a rotary embedding of q and k (half-split pairs
 * (i, i + dh/2) rotated by pos * rope_theta^(-2i/dh), pos = the row's index
 * in its sequence, restarting at 0 in every segment); 0 leaves it off. */
typedef struct {
  int d_model;
  int n_heads;
  int head_dim;      /* d_model == n_heads * head_dim */
  int d_ff;          /* SwiGLU intermediate width F */
  float rms_eps;     /* 1e-5 */
  float rope_theta;  /* 0 = no rotation; > 0 = rotary base (e.g. 10000) */
} seer_dims;

/* Detector and routing parameters (Sec. 3.3-3.4; defaults in brackets). */
typedef struct {
  float act_eps;         /* |a| < act_eps counts as a near-zero activation; the paper
                            uses an absolute threshold whose value it does not print */
  double tau_jump;       /* minimum sparsity jump [0.03] */
  double gamma;          /* plateau tolerance: noise <= gamma * jump [0.6] */
  int window;            /* look-ahead window size w [3] */
  double tau_pad;        /* padding waste threshold for the static path [0.2] */
  int eager_max_bucket;  /* buckets <= this go to the eager path [4] */
  int bucket_min;        /* smallest micro-bucket; the set doubles from it up to N [8] */
} seer_params;

/* Device pointers of one block's weights: f16 for a bf16 or f16 layer (make
 * them once with seer_convert), fp32 for an fp32 layer.
 * w_qkv [3*d, d] = rows of Wq, then Wk, then Wv;  w_o [d, d];
 * w_gate, w_up [F, d];  w_down [d, F];  g_attn, g_mlp [d] RMSNorm gains. */
typedef struct {
  const void* w_qkv;
  const void* w_o;
  const void* w_gate;
  const void* w_up;
  const void* w_down;
  const void* g_attn;
  const void* g_mlp;
} seer_layer_weights;

/* Execution paths of the hybrid router (Sec. 3.4). */
enum { SEER_PATH_STATIC = 0, SEER_PATH_VARLEN = 1, SEER_PATH_EAGER = 2 };

/* Control word written by seer_pack_ragged to pinned host memory (Sec. 3.5:
 * the CPU polls a small signal instead of waiting for the tensors).
 * int32 words:
 *   [0] epoch (written last; equals the `epoch` argument once ready)
 *   [1] total packed rows            [2] longest segment (rows)
 *   [3] graph capacity (rows): the smallest m * 2^e >= total, m in 8..15
 *   [4] number of groups              [5] bit mask of the paths in use
 *   [6] rows of bucket padding added by static groups   [7] reserved
 *   then per group g < SEER_MAX_GROUPS, 4 words at 8 + 4g:
 *   bucket, member count, path, rho in parts per million (rounded down). */
#define SEER_MAX_GROUPS 32
#define SEER_CTRL_WORDS (8 + 4 * SEER_MAX_GROUPS)

/* ---------------------------------------------------------------------------
 * Step-0 boundary detector (Sec. 3.2-3.3).
 *
 * For each sequence b the response rows x[resp_start[b] + t], t < N, go
 * through the SwiGLU MLP a = SiLU(x Wg^T) * (x Wu^T) on the tensor cores; the
 * epilogue counts |a| < act_eps per row (never storing a), giving
 * counts_out[b*N + t] (the sparsity s_t = counts/F).  The SNR scan then finds
 * the first 0-based i in [1, N-w] with jump = min(s_i..s_{i+w-1}) - s_{i-1}
 * >= tau_jump and max(..) - min(..) <= gamma * jump, evaluated in fp64 in that
 * order; L* = i* + 1, or L* = N and i* = -1 when nothing passes.
 *
 * x          device [T_rows, d] rows of the full windows (dtype dt)
 * resp_start device int32 [B]: first response row of each sequence; every
 *            resp_start[b] + N must be <= T_rows (checked on the device)
 * w_gate, w_up  device [F, d], same dtype as x (bf16 operands feed the
 *            tensor cores directly; the counts need no intermediate storage)
 * counts_out device int32 [B*N] (overwritten)
 * L_star_out, i_star_out  device int32 [B] (i_star_out may be NULL)
 * Requires B >= 1, N >= 1.  No workspace.
 * ------------------------------------------------------------------------- */
seer_status seer_detect_boundary(const void* x, seer_dtype dt, int T_rows, const int32_t* resp_start,
                                 int B, int N, const void* w_gate, const void* w_up,
                                 const seer_dims* dims, const seer_params* params,
                                 int32_t* counts_out, int32_t* L_star_out, int32_t* i_star_out,
                                 void* stream);

/* The sparsity counts alone (Sec. 3.2; S1 of seer_detect_boundary): for each
 * response row t of each sequence, the number of |a_j| < act_eps over the F
 * SwiGLU activations of that row with the given gate/up weights.  With
 * accumulate != 0 the counts are added to counts_inout instead of replacing
 * it, so several layers' gate/up weights can be tapped (a multi-layer
 * sparsity signal, Sec. 4.5 / Table 12): the sum is then a count out of
 * k * F for seer_snr_scan.  Arguments as for seer_detect_boundary. */
seer_status seer_sparsity_counts(const void* x, seer_dtype dt, int T_rows, const int32_t* resp_start, int B, int N,
                                 const void* w_gate, const void* w_up, const seer_dims* dims, float act_eps,
                                 int accumulate, int32_t* counts_inout, void* stream);

/* The SNR scan alone (Sec. 3.3) over precomputed counts: counts device int32
 * [B*N] of near-zero activations out of F; writes L_star_out (and i_star_out
 * when not NULL), device int32 [B].  Same fp64 evaluation as above.  Any
 * look-ahead window 1 <= window <= N - 1 (params->window). */
seer_status seer_snr_scan(const int32_t* counts, int B, int N, int F, const seer_params* params,
                          int32_t* L_star_out, int32_t* i_star_out, void* stream);

/* ---------------------------------------------------------------------------
 * Routing + device-resident compaction (Sec. 3.4-3.5), one fused kernel.
 *
 * Groups the sequences by micro-bucket (smallest of {m, 2m, 4m, ..., <N} U {N}
 * that holds L*_b, m = params->bucket_min, 8 in the paper), computes each group's padding waste ratio (Eq. 4) and path:
 * eager if bucket <= eager_max_bucket or the group has one member, else
 * static if rho <= tau_pad, else varlen.  Static members keep ctx_b + bucket
 * rows (the rows past ctx_b + L*_b are padding, masked as keys), the others
 * keep ctx_b + L*_b rows.  Rows are copied from the full-window layout into
 * x_packed back to back with 16-byte vector copies.
 *
 * x_full        device [cu_full[B], d] full-window rows (ctx_b + N per sequence)
 * cu_full       device int32 [B+1]
 * ctx_len       device int32 [B]: visual + prompt rows of each sequence
 * L_star        device int32 [B] (1 <= L* <= N; checked on the device)
 * N             generation window (for the bucket set)
 * T_capacity    rows available in x_packed; the packed total must fit
 * x_packed      device [T_capacity, d] (rows past the total are untouched)
 * cu_out        device int32 [B+1] segment offsets;  kv_len_out device int32 [B]
 * meta_out      device int32 [SEER_CTRL_WORDS]: the same words as the control word
 * host_ctrl     pinned, device-mapped host memory of SEER_CTRL_WORDS int32, or
 *               NULL; receives the control word with word 0 = epoch written last
 * ------------------------------------------------------------------------- */
seer_status seer_pack_ragged(const void* x_full, seer_dtype dt, const int32_t* cu_full,
                             const int32_t* ctx_len, const int32_t* L_star, int B, int d, int N,
                             int T_capacity, const seer_params* params, void* x_packed,
                             int32_t* cu_out, int32_t* kv_len_out, int32_t* meta_out,
                             int32_t* host_ctrl, int32_t epoch, void* stream);

/* Spin on the host control word until word 0 equals `epoch` (acquire), then
 * copy SEER_CTRL_WORDS words to ctrl_copy.  Never touches the GPU.  Returns
 * SEER_ERR_TIMEOUT after timeout_us microseconds. */
seer_status seer_poll_ctrl(const int32_t* host_ctrl, int32_t epoch, int timeout_us, int32_t* ctrl_copy);

/* ---------------------------------------------------------------------------
 * One truncated denoising layer over packed ragged sequences (Sec. 3.1 Eq. 2,
 * Sec. 3.6 Eqs. 9-10): every segment attends bidirectionally to its own first
 * kv_len[b] rows only.
 *
 *   xn = RMSNorm(x); [q k v] = xn Wqkv^T; o = MHA(q, k, v); h = x + o Wo^T;
 *   hn = RMSNorm(h); a = SiLU(hn Wg^T) * (hn Wu^T); y = h + a Wd^T
 * x and y have the layer dtype dt; every tensor between ops is f16 for a
 * 16-bit layer and fp32 for an fp32 layer (see the precision note above).
 *
 * x, y          device [T_capacity, d]; y must not alias x
 * cu_seqlens    device int32 [B+1]; total rows cu_seqlens[B] <= T_capacity is
 *               read on the device, so one captured CUDA graph serves any
 *               total up to the capacity
 * kv_len        device int32 [B] valid keys per segment, or NULL (= segment length)
 * count_resp_start  optional device int32 [B] (NULL disables): packed row of
 *               each sequence's first response token; the SwiGLU epilogue then
 *               adds |a| < act_eps counts of rows [start, start+N) (inside the
 *               segment) into counts_out[b*N + t] (device int32 [B*N], zeroed
 *               by this call) -- the step-0 detection layer hook
 * ws, ws_bytes  device workspace of at least seer_layer_workspace_size() bytes
 * ------------------------------------------------------------------------- */
seer_status seer_layer_forward(const seer_layer_weights* w, const seer_dims* dims, seer_dtype dt,
                               const void* x, void* y, const int32_t* cu_seqlens,
                               const int32_t* kv_len, int B, int T_capacity,
                               const int32_t* count_resp_start, int N, float act_eps,
                               int32_t* counts_out, void* ws, size_t ws_bytes, void* stream);

seer_status seer_layer_workspace_size(const seer_dims* dims, seer_dtype dt, int T_capacity, int B,
                                      size_t* bytes);

/* ---------------------------------------------------------------------------
 * The layer's steps one at a time (same kernels as seer_layer_forward).
 * Row counts: M_dev (device int32, may be NULL) overrides M_cap when set.
 * ------------------------------------------------------------------------- */

/* y[M, d] = x * rsqrt(mean(x^2) + eps) * g, fp32 arithmetic.  g has y's
 * dtype.  Type pairs: bf16->f16, bf16->bf16, f16->f16, f32->f32; d % 8 == 0. */
seer_status seer_rmsnorm(const void* x, seer_dtype x_dt, const void* g, void* y, seer_dtype y_dt, int M_cap,
                         const int32_t* M_dev, int d, float eps, void* stream);

/* c[M, N] = a[M, K] w[N, K]^T (+ r[M, N] when r != NULL), fp32 accumulation.
 * a and w share op_dt; with 16-bit operands r and c may each be bf16 or f16
 * (N % 256 == 0, K % 64 == 0); with fp32 operands everything is fp32. */
seer_status seer_linear(const void* a, const void* w, seer_dtype op_dt, const void* r, seer_dtype r_dt, void* c,
                        seer_dtype c_dt, int M_cap, const int32_t* M_dev, int N, int K, void* stream);

/* In-place rotary embedding of the q and k heads of qkv [T, 3*H*dh]
 * (q | k | v column blocks, any dtype), as seer_layer_forward applies it when
 * rope_theta > 0 (there fused into the QKV projection's epilogue for 16-bit
 * layers): pair (i, i + dh/2) of a head turns by pos * theta^(-2i/dh), pos =
 * row - cu_seqlens[b] for the segment b holding the row.  Rows past
 * cu_seqlens[B] (device) are untouched.  theta > 0, head_dim even and <= 128.
 * Not from the paper (which names no positional scheme). */
seer_status seer_rope(void* qkv, seer_dtype dt, const int32_t* cu_seqlens, int B, int T_capacity, int n_heads,
                      int head_dim, float theta, void* stream);

/* act[M, F] = SiLU(a w_gate^T) * (a w_up^T) (F % 128 == 0 for 16-bit
 * operands); near-zero counts as in seer_layer_forward. */
seer_status seer_swiglu(const void* a, const void* w_gate, const void* w_up, seer_dtype op_dt, void* act,
                        seer_dtype act_dt, int M_cap, const int32_t* M_dev, int F, int K, const int32_t* cu_seqlens,
                        int B, const int32_t* count_resp_start, int N, float act_eps, int32_t* counts_out,
                        void* stream);

/* seer_attention for callers that cannot allocate device memory, such as code
 * whose device memory is owned by another allocator (an engine's pool, a
 * plugin without cudaMalloc) or that must not allocate on its hot path.  The
 * paper has no counterpart; this is a service of the library.
 * Same arguments and results as seer_attention, minus the workspace: the
 * schedule lives in a fixed 1 MiB __device__ array compiled into libseer,
 * held by every GPU that loads the library until the process exits.
 * For 16-bit attention n_heads * (ceil(T_capacity/128) + B) must stay
 * <= 65520 (the work units whose schedule fits the array), else the call
 * returns SEER_ERR_WORKSPACE; fp32 attention uses no schedule and has no such
 * limit.  The first call on a device looks up the array's device address
 * (cudaGetSymbolAddress) with that device current, so make it before any
 * stream capture; the address is kept for the process, so resetting the
 * device (cudaDeviceReset) while libseer is loaded is not supported.
 * Allocates nothing.  Every call reuses the same array: calls whose kernels
 * overlap on the GPU race and must not be issued (nothing in the array needs
 * to start at zero). */
seer_status seer_attention_noalloc(const void* qkv, void* o, seer_dtype dt, const int32_t* cu_seqlens,
                                   const int32_t* kv_len, int B, int T_capacity, int n_heads, int head_dim,
                                   void* stream);

/* dst[i] = src[i] converted (round to nearest even) for i < n; n % 8 == 0.
 * bf16 -> f16 is exact for |v| >= 2^-14 and below 65504 (f16's normal range);
 * a 16-bit result that is infinite or NaN records device error code 6.
 * Used once per model to make the f16 weight copies of bf16 layers. */
seer_status seer_convert(const void* src, seer_dtype src_dt, void* dst, seer_dtype dst_dt, size_t n, void* stream);

/* o[T, H*dh]: per segment b and head h, softmax(q k^T / sqrt(dh)) v over the
 * segment's first kv_len[b] keys (Eqs. 6-7, no causal mask).  qkv [T, 3*H*dh]
 * holds q | k | v.  ws as for seer_layer_forward (only the scheduling part:
 * the work units, their count and the counter from which the attention
 * kernel's persistent CTAs take units; rewritten by every call that does not
 * make its schedule inside the kernel, so calls that share a workspace must
 * not overlap on the GPU).  Where a call has few units (segment, head, 256
 * query rows) and many keys, each unit's keys are shared by a cluster of CTAs
 * and the shares merged in fp32: such a call's results differ from those of a
 * call that keeps them together by fp32 rounding before the 16-bit store.
 * Which of the two a 16-bit call does follows from n_heads, B and the
 * capacities it is given, so the same rows may be rounded otherwise in another
 * batch or in buffers of another capacity.  A layer with the count hook always
 * keeps them together: for the same input rows its counts are the same in any
 * batch and at any capacity, and its y may differ from the same call without
 * the hook by that rounding.  Layers before a hooked one do share keys, so the
 * counts of a stack may still differ between batches where an activation lies
 * within a rounding of the threshold. */
seer_status seer_attention(const void* qkv, void* o, seer_dtype dt, const int32_t* cu_seqlens,
                           const int32_t* kv_len, int B, int T_capacity, int n_heads, int head_dim,
                           void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Prefix key/value caching combined with truncation (the paper reports that
 * Seer composes with KV caching of the visual + prompt prefix, Table 7).
 * A K/V cache of one layer is a [T_kv_cap, 2*H*dh] matrix (K | V per row, the
 * layer's intermediate type: f16 for 16-bit layers, f32 for f32 ones) laid
 * out like the packed truncated sequences: segment b owns rows
 * [cu_kv[b], cu_kv[b+1]), its first ctx_len[b] rows hold the prefix's keys
 * and values (seer_kv_prefill) and the rest the response rows' own, which
 * seer_layer_forward_cached writes on every call.  cu_kv is the cu_seqlens of
 * seer_pack_ragged.  Rotary embeddings are not supported on this path.
 * ------------------------------------------------------------------------- */

/* Fills the prefix part of a layer's K/V cache: for each segment b, the rows
 * [cu_x[b], cu_x[b] + ctx_len[b]) of x (the layer's input hidden states, any
 * row layout, dtype dt) are normalised and projected with the K and V rows of
 * w->w_qkv, and the results stored at cache rows [cu_kv[b], cu_kv[b] +
 * ctx_len[b]).  ws: seer_layer_workspace_size(dims, dt, T_x_cap, B) bytes.
 * Row counts are read on the device; segments that would fall outside x or
 * the cache are skipped and recorded (seer_check_device). */
seer_status seer_kv_prefill(const seer_layer_weights* w, const seer_dims* dims, seer_dtype dt, const void* x,
                            const int32_t* cu_x, const int32_t* ctx_len, int B, int T_x_cap, void* kv_cache,
                            const int32_t* cu_kv, int T_kv_cap, void* ws, size_t ws_bytes, void* stream);

/* The block over the response rows only (packed by cu_resp, dtype dt in and
 * out, as from seer_gather_response): queries are the response rows, keys and
 * values the segment's cached prefix rows followed by its response rows (the
 * first kv_len[b] rows of the segment in all, kv_len as from
 * seer_pack_ragged; NULL = the whole segment).  Writes the response rows'
 * K and V into the cache first.  y_resp must not alias x_resp.  ws:
 * seer_layer_workspace_size(dims, dt, T_resp_cap, B) bytes. */
seer_status seer_layer_forward_cached(const seer_layer_weights* w, const seer_dims* dims, seer_dtype dt,
                                      const void* x_resp, void* y_resp, const int32_t* cu_resp, const int32_t* ctx_len,
                                      int B, int T_resp_cap, void* kv_cache, const int32_t* cu_kv,
                                      const int32_t* kv_len, int T_kv_cap, void* ws, size_t ws_bytes, void* stream);

/* Response rows of packed sequences: cu_resp_out[b] = cu[b] - (ctx_len[0] +
 * ... + ctx_len[b-1]) (device int32 [B+1]) and x_resp rows [cu_resp_out[b],
 * cu_resp_out[b+1]) = x_packed rows [cu[b] + ctx_len[b], cu[b+1]).  d * size
 * of dt must be a multiple of 16 bytes. */
seer_status seer_gather_response(const void* x_packed, seer_dtype dt, const int32_t* cu, const int32_t* ctx_len, int B,
                                 int d, int T_cap, void* x_resp, int32_t* cu_resp_out, void* stream);

/* ---------------------------------------------------------------------------
 * Paged key/value cache with grouped heads: for servers that admit prompts,
 * draft or refine a few rows per step and keep the accepted ones, over caches
 * whose lengths change.  The paper has no counterpart; the contiguous cache
 * above is laid out once per truncated batch.
 * A pool of pages holds one layer's keys and values: page p owns rows
 * [p * page_size, (p + 1) * page_size) of kv, each row K | V of n_kv_heads heads
 * in the call's dtype; row t of request b is row t % page_size of page
 * table[b * max_pages + t / page_size].  One table serves every layer's pool.
 * Query head h reads key/value head h / (n_heads / n_kv_heads).
 * What the device finds inconsistent (lengths outside the buffers, pages outside
 * the pool, too few free pages) is recorded (seer_check_device) and that
 * request's or row's part left out; no access leaves the buffers named.  T_cap is at
 * most 2^30, and where it is 0 row buffers may be NULL; masks are 8-byte aligned.
 * Attention of 16-bit types rounds each probability to the type before the product
 * with its value (the row's sum adds the rounded ones); scores, sums and maxima are
 * fp32.  Where a request's keys are split over CTAs and joined in fp32 follows from all
 * requests' lengths (tree attention) or from B, T_cap and max_draft (fp32), so the same
 * rows may be rounded otherwise in another batch.  A call repeats itself bit by bit.
 * A value that is infinite or NaN and lies among keys that some row of its tile does
 * not see costs time: those rows are taken one by one (one such value late in a prompt
 * of 11792 rows: 0.7 ms become 47).
 * ------------------------------------------------------------------------- */
#define SEER_MAX_DRAFT 64          /* new rows of a request that a tree can hold */
#define SEER_MAX_REQUESTS 16384    /* requests of a call */

typedef struct {
  void* kv;               /* device [n_pages * page_size, 2 * n_kv_heads * head_dim] */
  const int32_t* table;   /* device [B, max_pages] */
  int n_pages;
  int page_size;          /* a power of two from 8 to 1024; n_pages * page_size < 2^31 - 1024 */
  int max_pages;          /* pages of the longest request that the table holds */
  int n_kv_heads;
  int head_dim;           /* <= 128, a multiple of 16 (fp32: of 8) */
} seer_pages;

/* Pages, slots and positions of a step's new rows, from the requests' lengths.
 * Request b has cached_len[b] rows in the cache and adds new_len[b]; its new rows
 * are packed, rows cu_new_out[b] .. cu_new_out[b+1] - 1.  It owns the first
 * ceil(cached_len / page_size) entries of its table row; the entries up to
 * ceil((cached_len + new_len) / page_size) are taken from the free list, requests in
 * order, from free_pages[*free_head] on, and written to the table.  A request holds
 * at most max_pages * page_size rows, and at most 2^31 - 1025.
 *   kv_len_out[b]   = cached_len[b] + new_len[b]      (device int32 [B])
 *   slot_out[r]     = the pool row of new row r, -1 where it has none
 *   position_out[r] = cached_len[b] + i of the request's i-th new row, or, with
 *                     parent, cached_len[b] + its depth
 *   mask_out[r]     = bit j set where new row j of the request is the row itself or
 *                     an ancestor (without parent: j <= i); may be NULL
 *   *free_head_out  = *free_head + the pages taken (not the same address)
 * parent          device int32 [T_cap] or NULL: new row i's parent among the
 *                 request's new rows, -1 for a child of the last cached row; a
 *                 parent comes before its children
 * T_cap           rows of slot_out, position_out, mask_out and parent; rows past
 *                 cu_new_out[B] are untouched
 * With parent or mask_out a request has at most SEER_MAX_DRAFT new rows.  Table
 * entries of taken pages beyond the free list become -1.  No output is an input.
 * Every output depends on the inputs alone, so a call may be repeated.
 * Entries from ceil(cached_len / page_size) on are written over, whatever they hold:
 * the pages of rows that the caller drops (rejected drafts, ended requests) are the
 * caller's to put back, see seer_kv_accept. */
seer_status seer_page_tables(const int32_t* cached_len, const int32_t* new_len, int B, int page_size, int n_pages,
                             const int32_t* free_pages, int n_free, const int32_t* free_head, int32_t* table,
                             int max_pages, int T_cap, const int32_t* parent, int32_t* cu_new_out, int32_t* kv_len_out,
                             int32_t* slot_out, int32_t* position_out, uint64_t* mask_out, int32_t* free_head_out,
                             void* stream);

/* Stores the K | V part of packed rows q | k | v (n_heads query heads, then
 * pages->n_kv_heads key and as many value heads; ld_qkv values per row) at their
 * slots, the keys turned by their position as in seer_rope (theta 0: as they are).
 * rotated, when not NULL, receives the turned q | k of every row (ld_rotated values
 * per row); it may be qkv itself with its ld.  Rows: M_dev (device int32, may be
 * NULL) overrides T_cap.  slot -1: nothing is stored for the row; slots of a call
 * are distinct (two rows with one leave pieces of either there).  position: device
 * int32 [T_cap], NULL when theta is 0; theta is 0 or at least 1.  An angle is off by
 * at most 2^-21 rad up to position 2^29 and 2^-20 up to the last; one rounding per
 * value. */
seer_status seer_kv_append(const void* qkv, int ld_qkv, seer_dtype dt, int n_heads, int T_cap, const int32_t* M_dev,
                           const int32_t* slot, const int32_t* position, float theta, void* rotated, int ld_rotated,
                           const seer_pages* pages, void* stream);

/* Keeps the accepted rows of each request's draft: row cached_len[b] + k of request
 * b becomes its row cached_len[b] + accepted[b * max_draft + k], k < n_accepted[b]
 * (accepted ascends strictly, as the rows of a path from the root do), and
 * len_out[b] = cached_len[b] + n_accepted[b] is its next cached_len.  A request with
 * a list that does not ascend, leaves the draft or meets a page outside the pool
 * keeps nothing and is recorded.  One call per layer's pool.
 * The table is as before: its entries from ceil(len_out[b] / page_size) up to
 * ceil(kv_len[b] / page_size) are pages that only rejected rows filled.  Before the
 * next seer_page_tables, which writes over them, the caller puts these k pages back,
 * e.g. into free_pages[head - k .. head - 1], those already taken, and lowers the free
 * list's head by k. */
seer_status seer_kv_accept(seer_dtype dt, const int32_t* cached_len, const int32_t* accepted, const int32_t* n_accepted,
                           int B, int max_draft, const seer_pages* pages, int32_t* len_out, void* stream);

/* Causal attention over whole packed prompts with grouped heads: per sequence,
 * row i attends to rows 0 .. i, scores divided by sqrt(head_dim).  q, k, v and o are
 * rows of n_heads or n_kv_heads heads, ld_* values apart (column blocks of one
 * packed buffer, or buffers of their own), 16-byte aligned.  cu_seqlens device
 * int32 [B+1], read on the device; rows past cu_seqlens[B] are untouched.  head_dim:
 * 64 or 128 for 16-bit types, a multiple of 4 up to 128 for fp32.  o must not
 * overlap the inputs.  A key that a row does not see never reaches its result, not
 * even an infinite or NaN one.  Where an offset is below the one before it, that
 * sequence is left out and recorded, and rows of sequences that then overlap hold
 * either's result.  No workspace. */
seer_status seer_attention_causal(const void* q, int ld_q, const void* k, int ld_k, const void* v, int ld_v, void* o,
                                  int ld_o, seer_dtype dt, const int32_t* cu_seqlens, int B, int T_cap, int n_heads,
                                  int n_kv_heads, int head_dim, void* stream);

/* Attention of each request's new rows over its pages (their own keys stored there
 * before, seer_kv_append): new row i sees the kv_len[b] - n cached rows, n =
 * cu_new[b+1] - cu_new[b], and the new rows j with bit j of mask[row] set (mask
 * NULL: j <= i).  n <= max_draft <= SEER_MAX_DRAFT; n = 1 decodes single tokens.  A
 * row that sees no key is 0.  A page outside the pool reads as zeros and is
 * recorded.  head_dim, scaling and hidden keys as above.
 * ws: seer_attention_tree_workspace_size() bytes; calls that share one must not
 * overlap on the GPU; nothing in it needs to start at zero. */
seer_status seer_attention_tree(const void* q, int ld_q, void* o, int ld_o, seer_dtype dt, const int32_t* cu_new,
                                const int32_t* kv_len, const uint64_t* mask, int B, int T_cap, int n_heads,
                                int max_draft, const seer_pages* pages, void* ws, size_t ws_bytes, void* stream);
seer_status seer_attention_tree_workspace_size(seer_dtype dt, int B, int n_heads, int n_kv_heads, int head_dim,
                                               int max_draft, size_t* bytes);

/* ---------------------------------------------------------------------------
 * A paged cache under a budget, for servers whose prompts outgrow the positions that a
 * model was trained on and the memory that a request may hold: positions scaled for
 * long contexts, and the cached rows dropped that the queries look at least.  A step:
 *   seer_page_tables, seer_kv_append_rotary (positions count the rows dropped so far),
 *   attention, seer_attention_mass, and for requests past their budget
 *   seer_evict_select and seer_kv_evict.
 * Attention does not depend on the order of cached rows (a key carries its position), so
 * an evicted row's place is taken by a row from the cache's end and nothing else moves.
 * Two numbers are kept for row t of request b, at [b * ld_mass + t]: mass (fp32), the
 * attention weight it has gathered, and birth (int32), its position.  gone[b] counts the
 * rows that the request has lost: kv_len[b] + gone[b] is its next position.  Lengths are
 * the same in every layer, so one page table goes on serving all; mass, birth and the
 * choice of rows may be each layer's own or shared.
 * What the device finds inconsistent is recorded (seer_check_device) and that request
 * left out; no access leaves the buffers named.  A call repeats itself bit by bit.
 * ------------------------------------------------------------------------- */
typedef enum {
  SEER_ROTARY_PLAIN = 0,
  SEER_ROTARY_LINEAR = 1,   /* every rate divided by factor */
  SEER_ROTARY_TURNS = 2,    /* by the turns n a pair makes over original_len: as it is from
                               high turns on, divided by factor up to low, between them
                               rate * (g + (1 - g) / factor), g = (n - low) / (high - low) */
  SEER_ROTARY_PAIRS = 3     /* by the pair's number i: rate * (1 - t + t / factor), t rising
                               from 0 at pair first to 1 at pair last, the (floored, ceiled)
                               pairs that make high and low turns over original_len; first
                               at least 0, last at most rotary_dim - 1 and above first by
                               0.001 where it would not be */
} seer_rotary_scaling;

typedef struct {
  double theta;             /* pair i turns by theta^(-2i / rotary_dim) per position; >= 1 */
  double factor;            /* scalings: >= 1 */
  double low, high;         /* TURNS, PAIRS: 0 < low < high */
  double magnitude;         /* cosines and sines are multiplied by it (1: a rotation); finite in fp32 */
  int original_len;         /* TURNS, PAIRS: > 0 */
  int rotary_dim;           /* the head's first values that turn: even, from 2 to head_dim */
  int interleaved;          /* 0: pairs (i, i + rotary_dim / 2); 1: pairs (2i, 2i + 1) */
  int scaling;              /* seer_rotary_scaling */
} seer_rotary;

/* out[r] = the n_heads heads of x[r] turned by position[r] (device int32 [T_cap], may be
 * negative): (a, b) of a pair becomes magnitude * (a cos - b sin, b cos + a sin); values
 * from rotary_dim on are copied as they are.  Rows of x and out are ld_* values apart;
 * out may be x itself with its ld, else they must not overlap.  M_dev (device int32, may
 * be NULL) overrides T_cap; rows past it are untouched.  head_dim: a multiple of 16 (fp32:
 * of 8) up to 128; without interleaving rotary_dim is a multiple of 4 (fp32: of 2).  An
 * angle is off by at most 2^-20 rad up to position 2^29 and 2^-18 up to the last; one
 * rounding per value. */
seer_status seer_rotate(const void* x, int ld_x, seer_dtype dt, int n_heads, int head_dim, int T_cap,
                        const int32_t* M_dev, const int32_t* position, const seer_rotary* rotary, void* out, int ld_out,
                        void* stream);

/* seer_kv_append with the rotation that `rotary` describes (NULL: none), each row turned
 * by its position + shift of its request: row r of request b, cu_new[b] <= r <
 * cu_new[b+1], by position[r] + shift[b] (shift NULL: by position[r], cu_new may then be
 * NULL; rows outside the requests are not shifted).  shift is the gone of a cache that
 * has lost rows and position what seer_page_tables gives. */
seer_status seer_kv_append_rotary(const void* qkv, int ld_qkv, seer_dtype dt, int n_heads, int T_cap,
                                  const int32_t* M_dev, const int32_t* slot, const int32_t* position,
                                  const int32_t* cu_new, const int32_t* shift, int B, const seer_rotary* rotary,
                                  void* rotated, int ld_rotated, const seer_pages* pages, void* stream);

/* Attention weight that each cached row receives from the request's last new rows, summed
 * over them and over all query heads:
 *   mass_out[b, t] = (t < c ? keep * mass_in[b, t] : 0) + sum_h sum_i p_h(i, t), t < kv_len[b]
 * with c = kv_len[b] - n rows from before the step, n new rows (their keys stored), of which
 * the last w = min(n, window) look: new row i sees rows t <= c + i, and p_h(i, .) is the
 * softmax of q_h(i) k_t / sqrt(head_dim) over them.  The sum over a softmax's row is 1, so
 * the new weight of a request adds up to w * n_heads.  Also birth[b, c + i] = c + i +
 * gone[b] of all new rows (birth NULL: not kept; gone NULL: zeros).
 * q               rows of n_heads heads, turned as the keys are; request b's new rows are
 *                 rows cu_new[b] .. cu_new[b+1] - 1
 * accepted        NULL: n = cu_new[b+1] - cu_new[b].  Else, after seer_kv_accept with the
 *                 same lists: n = n_accepted[b], and new row i's query is row cu_new[b] +
 *                 accepted[b * max_draft + i]; kv_len is then seer_kv_accept's len_out.  A
 *                 row whose entry is outside its draft is recorded and does not look
 * window          rows that look at most, 1 .. SEER_MAX_DRAFT.  For the weight from all rows
 *                 of a prompt make a call per window of them with keep 1, their numbers as
 *                 accepted and kv_len up to the last of them; each goes through the keys up
 *                 to there once (scores kept, see ws) or twice
 * T_kv_cap        the requests' kv_len add up to at most this; requests past it are left
 *                 out and recorded
 * mass_in         may be mass_out itself (not overlap it otherwise); NULL where keep is 0
 * Entries from kv_len[b] to ld_mass are untouched.  A request without new rows keeps
 * keep * mass_in.  A score of minus infinity weighs nothing; one of plus infinity or NaN, or
 * nothing but minus infinity, makes a row's weights NaN for all rows that it sees.  Pages outside the pool read as zeros and are recorded.  Types, heads and
 * head_dim as for seer_attention_tree (fp32: n_heads * window at most 16384); weights and
 * sums are fp32.
 * ws: seer_attention_mass_workspace_size() bytes, 16-byte aligned; calls that share one
 * must not overlap on the GPU; nothing in it needs to start at zero.  In fp32, and in 16 bits
 * where a key/value head has at most 16 query heads times rows of the window (n_heads * window
 * at most 1024), it holds all scores: 4 * n_heads * window bytes per key of T_kv_cap and per
 * request 64 keys more (fp32, 32 heads, 64 rows, 2^20 keys: 8.6 GB; a smaller window or
 * fewer requests a call take less). */
seer_status seer_attention_mass(const void* q, int ld_q, seer_dtype dt, const int32_t* cu_new, const int32_t* kv_len,
                                const int32_t* accepted, const int32_t* n_accepted, int max_draft, int window, int B,
                                int T_cap, int T_kv_cap, int n_heads, const seer_pages* pages, float keep,
                                const int32_t* gone, const float* mass_in, float* mass_out, int32_t* birth,
                                int ld_mass, void* ws, size_t ws_bytes, void* stream);
seer_status seer_attention_mass_workspace_size(seer_dtype dt, int B, int T_kv_cap, int n_heads, int n_kv_heads,
                                               int head_dim, int window, size_t* bytes);

/* Which rows each request keeps under its budget, and the moves that close the gaps.
 * K = min(budget[b], kv_len[b]) rows stay: first those born at kv_len[b] + gone[b] -
 * min(recent, K) or later, then those born before `sinks`, then the others by mass, the
 * most first (NaN above all); among equals the lower row.  The kept rows t >= K,
 * ascending, go to the places t < K of rows that are not kept, ascending:
 *   len_out[b]  = K, gone_out[b] = gone[b] + kv_len[b] - K, n_moves[b] = m, and
 *   row move_from[b * ld_move + i] becomes row move_to[b * ld_move + i], i < m
 * (entries from m on are untouched; gone NULL: zeros).  m is at most min(K, kv_len[b] -
 * K); where ld_move is less than that, where budget[b] is negative or kv_len[b] outside
 * 0 .. ld_mass the request is recorded and stays as it is (len_out = kv_len, m = 0).
 * gone_out may be gone itself and len_out kv_len itself. */
seer_status seer_evict_select(const float* mass, const int32_t* birth, int ld_mass, const int32_t* kv_len,
                              const int32_t* gone, const int32_t* budget, int B, int sinks, int recent,
                              int32_t* len_out, int32_t* gone_out, int32_t* n_moves, int32_t* move_from,
                              int32_t* move_to, int ld_move, void* stream);

/* Makes the moves in a pool, and in mass and birth (each may be NULL): one call per
 * layer's pool, mass and birth once.  kv_len is the length before the choice (NULL: the
 * rows that the table holds); moves from or to rows outside it, or pages outside the
 * pool, are left out and recorded.  No row is both a source and a place, as
 * seer_evict_select leaves it, and no page that is moved to belongs to two requests.  The
 * table is as before: its entries from ceil(len_out[b] / page_size) up to ceil(kv_len[b] /
 * page_size) are pages to put back, as after seer_kv_accept. */
seer_status seer_kv_evict(seer_dtype dt, const int32_t* kv_len, const int32_t* n_moves, const int32_t* move_from,
                          const int32_t* move_to, int ld_move, int B, const seer_pages* pages, float* mass,
                          int32_t* birth, int ld_mass, void* stream);

/* ---------------------------------------------------------------------------
 * Diagnostics.
 * ------------------------------------------------------------------------- */
/* Thread-local message describing the last failure of this thread. */
const char* seer_last_error(void);

/* Synchronises the current device, then reports (and clears) the first
 * device-side error recorded by any kernel: SEER_OK or SEER_ERR_DEVICE with
 * code_out set (1 bad row count, 2 bad sequence layout, 3 pipeline wait timed
 * out, 4 boundary out of range, 5 capacity exceeded, 6 a stored 16-bit value
 * is infinite or NaN: an f16 intermediate overflowed +-65504, or the input
 * held a non-finite value). */
seer_status seer_check_device(int* code_out);

/* Failure-detection self-test: enqueues a kernel whose pipeline wait can
 * never complete (an mbarrier that no thread arrives on).  Like every wait
 * in the library's kernels it gives up after a time limit, here limit_us
 * (1 .. 1e7), records the timeout code (3) in the device error word and
 * returns, so the context stays usable; seer_check_device then reports
 * SEER_ERR_DEVICE with code 3.  Enqueues only; never waits. */
seer_status seer_selftest_wait_timeout(int limit_us, void* stream);

/* Launch overlap (programmatic dependent launch).  When on (the default),
 * each kernel of the library is launched as a programmatic dependent of the
 * previous kernel in its stream: the GPU may place its blocks while that
 * kernel finishes, which hides most of the launch gap between consecutive
 * kernels.  Every kernel waits, before it touches global memory, until the
 * kernels before it have completed and their writes are visible, so results
 * are the same with the setting on or off.  Process-wide; returns the previous setting (1 or 0). */
int seer_set_launch_overlap(int on);

/* Per-phase timing with CUDA events recorded on the call's stream.
 * Phases: 0 detect GEMM, 1 SNR scan, 2 pack, 3 norm1, 4 QKV, 5 attention,
 * 6 O proj, 7 norm2, 8 gate/up, 9 down, 10 K/V cache copies and prefix
 * projections.  seer_profile_read synchronises on the recorded events and
 * returns accumulated milliseconds and launch counts since the last reset. */
#define SEER_N_PHASES 11
seer_status seer_profile_enable(int on);
/* Restricts recording to the phases whose bit is set in phase_mask (bit i =
 * phase i; default all).  Each recorded phase adds two events to its stream,
 * which also keeps launch overlap from spanning that phase's boundaries. */
seer_status seer_profile_select(uint32_t phase_mask);
seer_status seer_profile_reset(void);
seer_status seer_profile_read(float* ms_out, int32_t* launches_out);

/* Number of SMs of the current device (used to size persistent grids). */
int seer_num_sms(void);

const char* seer_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SEER_H */
