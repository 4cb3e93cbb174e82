/*
 * hyperattn.h - C ABI of the MI355X (gfx950) HyperAttention forward library.
 *
 * HyperAttention (arXiv 2310.05869) approximates softmax attention
 * Att = D^-1 A V, A = exp(Q K^T) (Section 1.1; no 1/sqrt(d) factor: fold any
 * scale into Q or K) in near-linear time:
 *   1. sortLSH (Definition 1, Algorithm 1): every row of Q and K is hashed by r
 *      random hyperplanes; the sign word's position in the reflected Gray code is
 *      the bucket; a stable sort by bucket gives permutations P_Q, P_K and the
 *      mask M^H = 1{floor(P_Q(i)/b) == floor(P_K(j)/b)}: the b x b diagonal
 *      blocks of the sorted attention matrix, which are computed exactly;
 *   2. the rest of each row is estimated from m key indices drawn uniformly
 *      with replacement, one set shared by all rows and reused for the value
 *      product (Algorithm 2 without its caps, as in the Implementation Detail
 *      paragraph of Section 4): weight (#keys/m), samples that fall in the row's
 *      own block contribute nothing;
 *   3. both parts share one normaliser: row sum = block part + estimate;
 *   4. causal masking (Section 3.1, Algorithm 4): recursive halving; the
 *      off-diagonal block (Q_2, K_1, V_1) of every split is an unmasked problem
 *      handled by 1-3, diagonal blocks of n_min rows are exact causal
 *      attention, and a row's partial results are combined by their row sums.
 *
 * Conventions for every entry point
 *   - Tensors are contiguous [B, H, n, d] in DEVICE memory, caller-owned, of the
 *     dtype in ha_shape (HA_BF16: 16-bit bfloat; HA_FP32: IEEE float).  `lse` is
 *     float [B, H, n], natural log of the (estimated) row sum.  Tensors start at a
 *     16-byte boundary, float and index arrays at a 4-byte one (HA_ERR_ALIGN).
 *   - The library allocates no device memory, never synchronises and enqueues
 *     only on `stream` (a hipStream_t passed as void*; NULL = the null stream).
 *     Scratch comes from the caller: `workspace` of at least
 *     ha_workspace_bytes() bytes, 256-byte aligned, device memory.  Two calls may
 *     overlap only if they use different workspaces.
 *   - Inputs are not modified; outputs must not alias inputs.
 *   - Return value: HA_OK (0) or a negative ha_status; nothing aborts.  Argument
 *     errors are detected on the host before anything is enqueued.
 *   - Same inputs, parameters and seed give bit-identical outputs (no floating
 *     point atomics anywhere).
 *   - Pointers named *_host are host memory, everything else is device memory.
 *   - fp32 tensors: attention's products of two fp32 numbers are formed from three bf16 parts of each and summed in fp32.  A product,
 *     rounded, is within 2^-23.2 of its value (2^-25.2 r.m.s., as one rounding to fp32 is).  Infinities, NaN and products past
 *     the largest number have the results that they have in fp32.  Parts below 2^-126 count as zeros: numbers of Q, K, V and d_out are taken
 *     with an absolute error of up to 2^-125, weights and what the backward forms of them with 2^-126, so that numbers keep their
 *     24 bits from 2^-101 upwards and those below 2^-125 count as 0 (an infinity times such a number is NaN).
 */
#ifndef HYPERATTN_H
#define HYPERATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { HA_BF16 = 0, HA_FP32 = 1 } ha_dtype;

typedef enum {
  HA_OK = 0,
  HA_ERR_NULL = -1,      /* a required pointer is NULL */
  HA_ERR_DTYPE = -2,     /* dtype is neither HA_BF16 nor HA_FP32 */
  HA_ERR_SHAPE = -3,     /* shape or parameters outside what is supported (see each call) */
  HA_ERR_WORKSPACE = -4, /* workspace too small or not 256-byte aligned */
  HA_ERR_LAUNCH = -5,    /* the HIP runtime refused a launch (hipGetLastError) */
  HA_ERR_ALIGN = -6,     /* a tensor does not start at a 16-byte boundary, or a float / index array at a 4-byte one */
  HA_ERR_STATIC_LIMIT = -7 /* hyperattn_forward_static: the problem needs more than ha_static_scratch_bytes() of scratch */
} ha_status;

/* [B, H, n, d]; d must be 64 or 128; n <= 2^22; B*H <= 2^20. */
typedef struct {
  int32_t B, H, n, d;
  int32_t dtype; /* ha_dtype */
} ha_shape;

/* b: block size of the sorted diagonal blocks; m: sampled key columns per node
 * (0 = block part only); r: LSH hyperplanes, 1..8; causal: 0/1; n_min: causal
 * recursion stops (exact causal attention) at n <= n_min; seed: selects the
 * hyperplanes and the sample indices. */
typedef struct {
  int32_t b, m, r, causal, n_min;
  uint64_t seed;
} ha_params;

/* Byte offsets of the regions of the workspace, for inspection after a forward
 * call (stage-by-stage parity checks).  `levels` is 1 for the unmasked problem
 * and log2(n / n_min) for the causal one (0 if n <= n_min); n_cov is the number
 * of query (= key) rows all nodes of one level cover per head: n (unmasked) or
 * n/2 (causal).  Node j of level l has s = n_cov >> l rows (causal) and owns
 * entries [j*s, (j+1)*s) of its level's arrays.
 *   codes_q, codes_k  uint8  [B*H][n]                 bucket index of each row
 *   perm_q, perm_k    int32  [levels][B*H][n_cov]     row (index within the head) at each sorted position
 *   pos_k             int32  [levels][B*H][n_cov]     sorted position (within the node) of each key
 *   samples           int32  [total_nodes][m]         l_1..l_m of each node, heap order (level l node j -> 2^l - 1 + j)
 *   samp_blk          int32  [B*H][total_nodes][m]    floor(pos_k[l_j] / b): the sorted block each sampled key falls in
 *   proj              float  [d][r]                   hyperplane matrix R
 *   sort_hist         uint32 [chunks][256]            scratch of the sort: bucket counts per 4096-key chunk
 *   part_o            dtype  [levels][B*H][n_cov][d]   causal only: per-level partial outputs (normalised), in the tensors' dtype
 *   part_l            float  [levels][B*H][n_cov]      causal only: log of the per-level partial row sums
 */
typedef struct {
  int32_t levels, total_nodes;
  int64_t n_cov;
  size_t codes_q, codes_k, perm_q, perm_k, pos_k, samples, samp_blk, proj, sort_hist, part_o, part_l;
  size_t total_bytes;
} ha_ws_layout;

/* Host only.  Validates shape/params as hyperattn_forward does and fills
 * *layout.  Returns HA_OK or the error hyperattn_forward would return. */
int ha_workspace_layout(const ha_shape* shape, const ha_params* params, ha_ws_layout* layout);

/* Host only.  Bytes of workspace hyperattn_forward needs; 0 if shape/params are invalid. */
size_t ha_workspace_bytes(const ha_shape* shape, const ha_params* params);

/* HyperAttention forward (Algorithm 3 in its Section 4 form; Algorithm 4 when
 * params->causal).  out: [B,H,n,d] of shape->dtype; lse: float [B,H,n].
 * HA_ERR_SHAPE unless: d in {64,128}; 1 <= r <= 8; b >= 1; 0 <= m <= 4096;
 * b <= 4096; B*H <= 2^20, n <= 2^22 and B*H*n <= 2^30; unmasked: n % b == 0; causal: n_min >= 1 and either n <= n_min
 * (plain exact causal attention) or n / n_min is a power of two with
 * n_min % b == 0.  The hyperplanes and sample indices are those
 * ha_make_projection / ha_make_samples return for params->seed. */
int hyperattn_forward(const void* Q, const void* K, const void* V, void* out, float* lse,
                      const ha_shape* shape, const ha_params* params,
                      void* workspace, size_t workspace_bytes, void* stream);

/* For callers that cannot allocate device memory or hand over a workspace (code
 * under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): hyperattn_forward with the workspace taken from an array built
 * into the library (device memory of the code object, ha_static_scratch_bytes()
 * = 32 MiB per GPU, held until the process ends).  Same kernels, same results,
 * bit for bit, as hyperattn_forward.  The call allocates and frees nothing; the
 * array's device address is looked up once per device on the first call there.
 * Problems whose ha_workspace_bytes() exceeds the array return
 * HA_ERR_STATIC_LIMIT before anything is enqueued.  All calls on one GPU share
 * the one array: calls that overlap in time on one GPU (different streams or
 * host threads) race and must be serialised by the caller.  Nothing is kept in
 * the array between calls. */
int hyperattn_forward_static(const void* Q, const void* K, const void* V, void* out, float* lse,
                             const ha_shape* shape, const ha_params* params, void* stream);

/* Host only.  Size in bytes of the built-in array hyperattn_forward_static uses. */
size_t ha_static_scratch_bytes(void);

/* Same, with the random draws supplied by the caller: R_dev is float [d][r]
 * (NULL = derive from the seed); samples_dev is int32 [total_nodes][m] in heap
 * order, node-local key indices in [0, s) (NULL = derive from the seed).  Both
 * are device memory and are copied into the workspace on `stream`.  The call
 * never reads device memory on the host, so it cannot reject an index outside
 * [0, s): such an index is clamped into the node by the copying kernel (no
 * access outside the node's keys can result); validate on the host beforehand
 * if the indices come from elsewhere (the Python binding does). */
int hyperattn_forward_ex(const void* Q, const void* K, const void* V, void* out, float* lse,
                         const ha_shape* shape, const ha_params* params,
                         const float* R_dev, const int32_t* samples_dev,
                         void* workspace, size_t workspace_bytes, void* stream);

/* Measurement variant of hyperattn_forward (same computation and results; the sort is always a launch of
 * its own, where hyperattn_forward lets the attention launch of a small problem sort):
 * HIP events are recorded on `stream` between the stages, the call WAITS for the
 * last one, and stage_ms_host[0..5] (host memory) receive the elapsed
 * milliseconds of: [0] always 0 (the random draws, once a launch of their own, are
 * stored by the hashing launch), [1] sortLSH hashing of Q and K with the draws, [2] the
 * sort (Algorithm 1's permutations), [3] block + sampled
 * attention of all nodes, [4] the exact causal base case with the Algorithm 4
 * merge (0 when not causal), [5] the whole call.  Unlike every other entry
 * point this one synchronises with the stream. */
int hyperattn_forward_timed(const void* Q, const void* K, const void* V, void* out, float* lse,
                            const ha_shape* shape, const ha_params* params,
                            void* workspace, size_t workspace_bytes, void* stream,
                            float* stage_ms_host);

/* Measurement variant of hyperattn_forward for bf16 tensors (same computation and
 * results; HA_ERR_DTYPE otherwise): the two attention launches of the forward pass
 * (all nodes of Section 4.1 / Algorithm 4; the causal base case) run an instrumented
 * instantiation of the same kernel, in which every workgroup also writes HA_STAMP_WORDS
 * 64-bit words into device memory, indexed by its tile number:
 *   [0] shader-clock reading at entry, [1] once its key list (block keys + kept
 *   samples) is built, [2] before the loop over key tiles (rows gathered, first
 *   score tile done), [3] after the loop, [4] at the end (results stored);
 *   [5], [6] the constant-rate counter (100 MHz) at entry and at the end;
 *   [7] bits 0-15 the number of 64-key tiles of the workgroup; bits 16-47 the hardware id
 *   register of its first wave (bits 8-11 of that value: CU, 13-15: shader engine);
 *   bits 48-51 the number of its XCD.
 * ha_forward_workgroups gives the number of records of either launch (0 for a launch
 * the problem does not have, and for fp32 tensors); node_stamps_dev / base_stamps_dev
 * are device memory of at least that many records (sizes in bytes, checked:
 * HA_ERR_WORKSPACE), 8-byte aligned, owned by the caller, and may be NULL where the
 * count is 0.  Asynchronous on `stream` like hyperattn_forward. */
#define HA_STAMP_WORDS 8
int ha_forward_workgroups(const ha_shape* shape, const ha_params* params, int64_t* node_wgs, int64_t* base_wgs);
int hyperattn_forward_stamped(const void* Q, const void* K, const void* V, void* out, float* lse,
                              const ha_shape* shape, const ha_params* params,
                              void* workspace, size_t workspace_bytes, void* stream,
                              int64_t* node_stamps_dev, size_t node_stamps_bytes,
                              int64_t* base_stamps_dev, size_t base_stamps_bytes);

/* Host only.  Which launches the calls for this shape and params take where small problems have others (tests,
 * measurements): *sorts_in_attention is 1 if hyperattn_forward lets the attention launch sort, else 0;
 * *shared_workgroups the workgroups of the larger launch that passes of hyperattn_backward share, 0 if they do not. */
int ha_call_routes(const ha_shape* shape, const ha_params* params, int32_t* sorts_in_attention, int64_t* shared_workgroups);

/* Host only.  fp32 tensors: by how many of a workgroup's waves the key tiles of one group of rows are taken in turn (tests): *forward in the
 * node launches of hyperattn_forward and, unmasked, of hyperattn_forward_alg2; *backward in the node passes of hyperattn_backward, 0 where they
 * share launches.  Both 0 without nodes and for bf16 tensors. */
int ha_fp32_ways(const ha_shape* shape, const ha_params* params, int32_t* forward, int32_t* backward);

/* Plain exact attention D^-1 A V (Section 1.1), or D_C^-1 (M^C . A) V with
 * M^C_ij = 1{i >= j} (Section 3.1) when causal != 0; the denominator of the
 * speed-up ratio.  Any n >= 1; d in {64,128}.  Needs no workspace. */
int exact_attn_forward(const void* Q, const void* K, const void* V, void* out, float* lse,
                       const ha_shape* shape, int causal, void* stream);

/* Host only.  The r hyperplane normals used for `seed` (Definition 1 read as
 * sign-of-Gaussian-projection LSH): R_host[c*r + k], c < d, k < r, i.i.d. N(0,1)
 * rounded to bf16-representable floats.  Entry (c,k) depends on (seed,c,k) only. */
int ha_make_projection(uint64_t seed, int32_t d, int32_t r, float* R_host);

/* Host only.  The m key indices, i.i.d. uniform on [0, n_keys) with
 * replacement (Algorithm 2), that node `node` of recursion level `level` uses
 * (level 0, node 0 for the unmasked problem); shared by all batches and heads. */
int ha_make_samples(uint64_t seed, int32_t level, int32_t node, int32_t n_keys, int32_t m,
                    int32_t* idx_host);

/* ---- single stages, for stage-by-stage parity and profiling ---------------- */

/* sortLSH hashing (Definition 1; Algorithm 1 "hash rows of Q, K"): codes[i] =
 * Gray-sequence position of the sign word of X[i,:] R.  X: [rows][d] of dtype,
 * R_dev: float [d][r], codes: uint8 [rows].  The codes equal those of an fp64
 * evaluation of the projections: bf16 rows are projected on the matrix cores in
 * fp32 together with a bound on the accumulation error, and every row with a
 * projection inside that bound is recomputed in fp64 (exact products); fp32 rows
 * are accumulated in fp64 throughout. */
int ha_lsh_hash(const void* X, uint8_t* codes, int64_t rows, int32_t d, int32_t dtype,
                const float* R_dev, int32_t r, void* stream);

/* Algorithm 1's permutation: n_seg independent segments of seg_len consecutive
 * codes each; stable ascending sort.  perm[g*seg_len + p] = index (within the
 * segment) of the row at sorted position p; pos = inverse.  seg_len <= 2^24. */
int ha_seg_sort(const uint8_t* codes, int32_t* perm, int32_t* pos, int32_t n_seg,
                int32_t seg_len, void* stream);

/* Row permutation ("permuting n rows", Section 4): dst[g][p][:] = src[g][idx[g*n + p]][:]
 * for g < groups, p < n; rows of d elements of dtype. */
int ha_gather_rows(const void* src, const int32_t* idx, void* dst, int32_t groups, int32_t n,
                   int32_t d, int32_t dtype, void* stream);

/* Block-diagonal part alone on inputs ALREADY in sorted order (Section 4,
 * Implementation Detail: i-th group of b sorted queries against the i-th group
 * of b sorted keys).  Qs,Ks,Vs: [groups][n][d]; o_b float [groups][n][d] and
 * lse_b float [groups][n], both in sorted order. */
int ha_block_attn(const void* Qs, const void* Ks, const void* Vs, float* o_b, float* lse_b,
                  int32_t groups, int32_t n, int32_t d, int32_t dtype, int32_t b, void* stream);

/* Sampled residual part alone (Algorithm 2's estimator with shared indices):
 * Qs in sorted order [groups][n][d]; K, V in ORIGINAL order [groups][n][d];
 * samples int32 [m] (original key indices), pos_k int32 [groups][n].  Sample j
 * is skipped for the rows of block floor(pos_k[l_j]/b).  o_r float
 * [groups][n][d], lse_r float [groups][n] (includes log(n/m); -inf and zero
 * row where nothing is kept), sorted order. */
int ha_sampled_attn(const void* Qs, const void* K, const void* V, const int32_t* samples,
                    const int32_t* pos_k, float* o_r, float* lse_r, int32_t groups, int32_t n,
                    int32_t d, int32_t dtype, int32_t b, int32_t m, void* stream);

/* Shared normaliser and inverse permutation: L = log(exp lse_b + exp lse_r),
 * out[g][perm_q[g*n+p]] = exp(lse_b-L) o_b[g][p] + exp(lse_r-L) o_r[g][p],
 * lse[g][perm_q[..]] = L.  out is of dtype. */
int ha_merge_unpermute(const float* o_b, const float* lse_b, const float* o_r, const float* lse_r,
                       const int32_t* perm_q, void* out, float* lse, int32_t groups, int32_t n,
                       int32_t d, int32_t dtype, void* stream);

/* ------------------------------------------------------------------------
 * Backward pass (Section 4.2 times forward + backward; the backward is the
 * derivative of the forward above with the random draws, and so the
 * permutations, held fixed).  bf16 tensors run on the matrix cores; fp32 tensors
 * take the same passes, with operands split in three bf16 parts.
 *
 * Because every output row is one softmax over the union of its parts (block
 * keys, kept samples weighted s/m, base-case keys; Algorithms 1, 2, 4), with
 * L = lse and delta_i = <d_out_i, out_i>:
 *   P_ij = w_ij exp(<q_i,k_j> - L_i),  dV_j = sum_i P_ij d_out_i,
 *   dS_ij = P_ij (<d_out_i, v_j> - delta_i),  dQ_i = sum_j dS_ij k_j,  dK_j = sum_i dS_ij q_i.
 *
 * hyperattn_forward_train: hyperattn_forward that also writes out_f32 (device
 * fp32 [B][H][n][d]; NULL: none), the output before its rounding to bf16.  The
 * backward forms delta from it: with the bf16 tensor alone delta carries the
 * output's rounding error (2^-9 relative), which dominates dQ and dK on rows
 * whose weight sits on few keys, where <d_out_i, v_j> - delta_i cancels.
 * exact_attn_forward_train: the same for exact attention.
 *
 * hyperattn_backward: Q, K, V, out, d_out, dQ, dK, dV are device pointers to
 * contiguous [B][H][n][d] of shape->dtype; lse device fp32 [B][H][n]; out_f32 as written
 * by hyperattn_forward_train, or NULL (delta then comes from out; fp32 tensors:
 * must be NULL, HA_ERR_DTYPE otherwise).  out and lse are the
 * results of hyperattn_forward on the same Q, K, V, shape and params, and
 * fwd_workspace is that call's workspace, unmodified since (it holds the sort
 * permutations and sample indices; only read here).  bwd_workspace: device,
 * 256-byte aligned, >= ha_backward_workspace_bytes(); overwritten.  All
 * caller-owned; nothing is allocated; kernels are enqueued on `stream` and the
 * call returns without waiting.  Sums over parts are taken in a fixed order
 * (the node parts level by level into one accumulated fp32 row per tensor row):
 * same inputs give bit-identical gradients.
 * Errors: HA_ERR_NULL, HA_ERR_DTYPE, HA_ERR_SHAPE (as hyperattn_forward; more
 * than 24 recursion levels), HA_ERR_WORKSPACE, HA_ERR_LAUNCH.
 *
 * hyperattn_backward_timed: the same, and WAITS for the stream; stage_ms_host
 * (host, 8 floats) receives the times between events on the stream: delta, dQ
 * of the nodes, dQ of the base case (unmasked problems: 0), dK/dV of the block
 * keys, dK/dV of the sampled keys with their reduction, dK/dV of the base case, 0 (the passes write the final
 * tensors themselves), total.  Unmasked problems and causal ones with n <= n_min (but fp32 tensors at d = 128) form delta in the one
 * dQ pass: the first value is 0 and that pass's holds both.  Small fp32 causal problems, whose passes share launches: the second value is 0, the third
 * the base case with the sampled keys, the fourth all node passes, the fifth the samples' sums, the sixth 0.
 *
 * exact_attn_backward: gradients of exact_attn_forward (Section 1.1; causal:
 * Section 3.1), the denominator of the forward + backward speed-up.  workspace
 * >= exact_attn_backward_workspace_bytes(shape). */
typedef struct {
  size_t delta;                      /* fp32 [B*H][n] */
  size_t acc_a, acc_b;               /* fp32 [B*H][n][d] each: the node parts' rows, added up level by level
                                        (acc_a: dQ, afterwards dK; acc_b: dV); empty for unmasked problems,
                                        not used by small fp32 causal ones, whose gradients hold the sums */
  size_t samp_k, samp_v;             /* fp32 rows of the sampled keys per (level, head, node, query chunk, sample) */
  size_t total_bytes;
} ha_bwd_ws_layout;

int ha_backward_workspace_layout(const ha_shape* shape, const ha_params* params, ha_bwd_ws_layout* layout);
size_t ha_backward_workspace_bytes(const ha_shape* shape, const ha_params* params);
int hyperattn_forward_train(const void* Q, const void* K, const void* V, void* out, float* lse, float* out_f32,
                            const ha_shape* shape, const ha_params* params, void* workspace,
                            size_t workspace_bytes, void* stream);
int exact_attn_forward_train(const void* Q, const void* K, const void* V, void* out, float* lse, float* out_f32,
                             const ha_shape* shape, int causal, void* stream);
int hyperattn_backward(const void* Q, const void* K, const void* V, const void* out, const float* out_f32,
                       const float* lse, const void* d_out, void* dQ, void* dK, void* dV, const ha_shape* shape,
                       const ha_params* params, const void* fwd_workspace, size_t fwd_workspace_bytes,
                       void* bwd_workspace, size_t bwd_workspace_bytes, void* stream);
int hyperattn_backward_timed(const void* Q, const void* K, const void* V, const void* out, const float* out_f32,
                             const float* lse, const void* d_out, void* dQ, void* dK, void* dV, const ha_shape* shape,
                             const ha_params* params, const void* fwd_workspace, size_t fwd_workspace_bytes,
                             void* bwd_workspace, size_t bwd_workspace_bytes, void* stream, float* stage_ms_host);
int exact_attn_backward(const void* Q, const void* K, const void* V, const void* out, const float* out_f32,
                        const float* lse, const void* d_out, void* dQ, void* dK, void* dV, const ha_shape* shape, int causal,
                        void* workspace, size_t workspace_bytes, void* stream);
size_t exact_attn_backward_workspace_bytes(const ha_shape* shape);

/* ------------------------------------------------------------------------
 * Algorithm 2 as printed and Lemma 2 / Algorithm 3, as options (the Section 4
 * form above leaves them out); both dtypes (bf16 tensors on the matrix cores,
 * weights rounded to bf16 as operands like in the forward; fp32 tensors with
 * products and sums to fp32, as above).  Causal problems run them at every off-diagonal node of
 * Algorithm 4 ("the unmasked algorithm on Q_2, K_1"): below, n is then the
 * node's size s, every node has its own subset T, index set and value rows
 * (counters offset by the node's heap index 2^level - 1 + node), the diagonal
 * blocks are exact and the results are added up as in hyperattn_forward.
 *   tau   = max over m rows drawn uniformly (with replacement) of the unmasked row sum
 *   C_i   = cap_scale * m / (n ln n) * (masked row sum_i + tau / kappa)     cap_scale <= 0: no cap
 *   d_i   = (n/m) sum_j (1 - M_{i,l_j}) min(exp<q_i,k_{l_j}>, C_i)
 *   d~_i  = masked row sum_i + max(d_i, tau / kappa)                         kappa <= 0: no lower cap
 *   out_i = (1/d~_i) sum_r exp<q_i,k_{l'_r}> v_{l'_r} / (m p_{l'_r}),  l'_r drawn with p_l ~ |V_l|^2   (vnorm_sampling)
 *        or (1/d~_i) (masked part + (n/m) sum_j (1 - M_{i,l_j}) exp<q_i,k_{l_j}> v_{l_j})             (otherwise)
 * lse receives log d~.  The constants the paper leaves open (the Theta of C_i,
 * kappa) are the caller's.  Lemma 2's rows are drawn with p_l = |V_l|^2 / |V|_F^2
 * by inverting the cumulative distribution in fp64 (draw r of head bh: first l
 * whose inclusive prefix sum of squared norms exceeds u |V|_F^2, u in (0,1) from
 * the top 53 bits of counter (heap * B*H + bh) * m + r of stream 2; T uses counter
 * heap * m + j of stream 0).
 * workspace: device, 256-byte aligned, >= ha_alg2_workspace_bytes(); it starts
 * with the forward's layout (ha_workspace_layout) followed by the regions below
 * ("per level": sized for the largest level and reused from level to level, so
 * after the call they hold the last, deepest level; "per node": every node of
 * every level, nodes in heap order).  Errors as hyperattn_forward. */
typedef struct {
  float cap_scale;
  float kappa;
  int32_t vnorm_sampling;
} ha_alg2_options;

typedef struct {
  size_t forward_bytes;      /* the forward's regions come first */
  size_t pos_q;              /* per level, int32 [B*H][n_cov]: inverse of perm_q within the node */
  size_t tau_rows;           /* per node, int32 [total_nodes][m]: the rows of T (node-local) */
  size_t log_unmasked_t;     /* per level, float [B*H * nodes][m]: log of their unmasked row sums */
  size_t log_tau;            /* per node, float [B*H][total_nodes] */
  size_t vnorm_w;            /* per level, double [B*H][n_cov]: |V_l|^2 of the nodes' value rows */
  size_t vnorm_prefix;       /* per level, double [B*H][n_cov]: inclusive prefix sums within the node */
  size_t vnorm_samples;      /* per node, int32 [B*H][total_nodes][m]: l'_r (node-local) */
  size_t vnorm_logw;         /* per node, float [B*H][total_nodes][m]: log(1 / (m p_{l'_r})) */
  size_t log_unmasked_parts; /* per level, float [8][B*H * nodes][m]: scratch, the unmasked row sums of T over eight ranges of keys */
  size_t part_ref;           /* causal, float [levels][B*H][n_cov]: log of the scale that the rows of part_o are taken against: log d~
                                (part_l), or the largest weight's where that is larger */
  size_t total_bytes;
} ha_alg2_ws_layout;

int ha_alg2_workspace_layout(const ha_shape* shape, const ha_params* params, ha_alg2_ws_layout* layout);
size_t ha_alg2_workspace_bytes(const ha_shape* shape, const ha_params* params);
int hyperattn_forward_alg2(const void* Q, const void* K, const void* V, void* out, float* lse,
                           const ha_shape* shape, const ha_params* params, const ha_alg2_options* options,
                           void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------
 * Packed sequences: exact attention (as exact_attn_forward / exact_attn_backward) over sequences of different lengths that lie
 * one behind the other in one batch of rows, with grouped heads.  Sequence s owns rows [cu_seqlens[s], cu_seqlens[s + 1]) of all
 * tensors; a row sees the keys of its own sequence, causal: those up to itself.  Query head h reads key head h / (Hq / Hk); dK and
 * dV are summed over the query heads of a group.
 *
 * Tensors are [rows][heads][d] with the strides given (elements; the d values of a row are consecutive), so that slices of one
 * projection's output are taken as they lie; strides == NULL: contiguous.  Strides are multiples of 16 bytes; row strides are
 * at least d and at most 2^22.  In what is written the heads of a row lie within the row stride, or the rows of a head within the head stride, and no output
 * overlaps another tensor.  lse: float [Hq][rows], out_f32: float [rows][Hq][d] contiguous (bf16 tensors; may be NULL).
 * cu_seqlens: device int32 [n_seq + 1], not decreasing, within [0, rows]; values outside [0, rows] are clamped where they are read.  Whatever
 * they are no access leaves the tensors and the workspace, but where they decrease the outputs' rows may hold anything, what lay in the workspace
 * among it.  Rows of no sequence are not read and not written: a batch may be padded at its end.
 * A sequence may be empty.  A key row of another sequence counts for nothing, whatever it holds; causal: an Inf or NaN in a row reaches, as 0 times
 * itself, also rows of its own sequence that do not see it where both lie in one tile of 128 rows, as in exact_attn_forward and exact_attn_backward.
 * rows <= 2^24, rows * Hq <= 2^27, n_seq * Hq <= 2^22, Hq % Hk == 0, Hq <= 1024; d in {64, 128}.
 * With out_f32, for a backward pass, bf16 rows are divided by the sum of their weights as rounded for the product with V, without it by the sum of the
 * unrounded ones; out may differ in its last bits.
 * exact_attn_packed_backward: out, lse and out_f32 as exact_attn_packed_forward wrote them; workspace: device, 256-byte aligned, >=
 * exact_attn_packed_backward_workspace_bytes(); nothing in it is kept.  Sums in a fixed order: same inputs, same bits. */
typedef struct {
  int64_t row, head;
} ha_strides;

typedef struct {
  int32_t n_seq, rows, Hq, Hk, d;
  int32_t dtype; /* ha_dtype */
  int32_t causal;
} ha_packed;

typedef struct {
  ha_strides q, k, v, out;       /* the forward takes these four */
  ha_strides d_out, dq, dk, dv;
} ha_packed_strides;

int exact_attn_packed_forward(const void* Q, const void* K, const void* V, const int32_t* cu_seqlens, void* out, float* lse,
                              float* out_f32, const ha_packed* shape, const ha_packed_strides* strides, void* stream);
int exact_attn_packed_backward(const void* Q, const void* K, const void* V, const int32_t* cu_seqlens, const void* out,
                               const float* out_f32, const float* lse, const void* d_out, void* dQ, void* dK, void* dV,
                               const ha_packed* shape, const ha_packed_strides* strides, void* workspace, size_t workspace_bytes,
                               void* stream);
size_t exact_attn_packed_backward_workspace_bytes(const ha_packed* shape);

/* ------------------------------------------------------------------------
 * A paged cache of K and V in 4 bits, for decoding behind a long prompt.
 *
 * Numbers: OCP MX FP4, the 4-bit type that gfx950 converts in one instruction.  32 consecutive channels of a row share a scale 2^(byte - 127)
 * (E8M0; byte 255: NaN), and a value is a code (E2M1: 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) times it, exact in bf16.  A
 * writer takes the smallest scale of 2^-125 ... 2^125 with max |x| <= 6 scale (numbers past 6 * 2^125 count as that) and rounds to the nearest value,
 * ties to the even code: a number is off by at most max |x| / 3, in the r.m.s. 0.115 of that of normal ones.  32 channels with an Inf or NaN are NaN.
 * Readers take any byte; values below 2^-126 may count as zeros in attention.
 *
 * cache: uint8 [n_pages][Hk][page * (d + d / 16)], 16-byte aligned, n_pages * page < 2^31; page: tokens of a page, 16, 32, 64, 128 or 256.
 * A page's block of a head (token t, channel c = 32 g + c'):
 *   K codes  d / 2 bytes a token: 32-bit word (c' / 8) * (d / 32) + g holds the codes of eight channels, channel c in nibble c' % 8
 *   V codes  for four tokens 4 u ... 4 u + 3 together d / 8 pieces of 16 bytes, a 32-bit word per token: d = 128: word c' / 2, byte g, d = 64: word
 *            c' / 4, byte 2 g + c' / 2 % 2; the even channel in the low nibble
 *   K scales d / 32 bytes a token, then V scales d / 32 bytes a token
 * Slot i of the cache is token i % page of page i / page.
 *
 * ha_cache4_write: row i of K and V ([rows][Hk][d] of dtype, strides as above: kv[0] of K, kv[1] of V; NULL: contiguous) to slot slots[i]; rows
 * whose slot lies outside the cache are left out.  Slots given must differ; where two rows name one slot it holds a mixture of both, and no
 * other slot is touched.  ha_cache4_read: the rows of these slots back, as the cache holds them (exact in both types; rows of slots
 * outside the cache: zeros).  rows <= 2^26, rows * Hk <= 2^26. */
typedef struct {
  int32_t n_pages, page, Hk, d;
} ha_cache4;

size_t ha_cache4_bytes(const ha_cache4* cache); /* 0 if it is not a valid one */
int ha_cache4_write(const void* K, const void* V, const int32_t* slots, void* cache, const ha_cache4* shape, int32_t rows,
                    int32_t dtype, const ha_strides* kv, void* stream);
int ha_cache4_read(const void* cache, const int32_t* slots, void* K, void* V, const ha_cache4* shape, int32_t rows, int32_t dtype,
                   const ha_strides* kv, void* stream);

/* Attention over the cache: the queries of the last q_len tokens of every sequence (1: a decoding step; more: drafted tokens that are
 * verified together).  Q, out: [n_seq * q_len][Hq][d] of dtype, row s * q_len + i the query of token lens[s] - q_len + i, which sees tokens 0 ... lens[s] -
 * q_len + i; strides qo[0], qo[1] (NULL: contiguous).  lse: float [Hq][n_seq * q_len].  Token t of sequence s lies in page block_table[s][t / page]
 * (device int32 [n_seq][max_blocks]).  lens (device int32) are taken within [0, max_blocks * page]; tokens of a page number outside [0, n_pages) count
 * as absent.  A query that sees nothing has out 0 and lse -inf.  What lies in a page behind a sequence's last token, or in a token behind the
 * query's own, counts for nothing, NaN included.
 * Products as in exact_attn_forward: bf16 queries on the matrix cores; fp32 queries split in three, to fp32 accuracy of the cached values.  Weighted sums
 * are formed before they are divided, by weights of at most 2^8: results are finite where the largest |V| times the tokens lies below 2^120.
 * 1 <= q_len <= 64, n_seq <= 2^16, n_seq * q_len * Hq <= 2^22, Hq * q_len <= 2^15, Hq % Hk == 0, n_seq * max_blocks <= 2^30, max_blocks * page < 2^31, n_seq *
 * max_blocks * page <= 2^36.
 * workspace: device, 256-byte aligned, >= ha_cache4_attn_workspace_bytes(); nothing in it is kept.  Two calls may overlap only with
 * different workspaces.  Same inputs, same bits. */
typedef struct {
  int32_t n_seq, q_len, Hq;
  int32_t dtype; /* ha_dtype of Q and out */
  int32_t max_blocks;
} ha_cache4_query;

int ha_cache4_attn(const void* Q, const void* cache, const int32_t* block_table, const int32_t* lens, void* out, float* lse,
                   const ha_cache4* shape, const ha_cache4_query* query, const ha_strides* qo, void* workspace,
                   size_t workspace_bytes, void* stream);
size_t ha_cache4_attn_workspace_bytes(const ha_cache4* shape, const ha_cache4_query* query); /* 0 if not valid */

/* Host only.  Which form of its launch ha_cache4_attn takes for these sizes (tests, measurements): *whole_waves is 8 or 4 where a workgroup of so many waves
 * takes a whole sequence, 0 where the tokens are shared out and a second launch joins their parts; *past_caches 1 if the latter reads codes past the caches.  The rules
 * know the table's room, not the lengths: only tables of at most 2048 tokens have the first, so max_blocks is best kept near the step's longest sequence. */
int ha_cache4_attn_form(const ha_cache4* shape, const ha_cache4_query* query, int32_t* whole_waves, int32_t* past_caches);

/* Attention of chunks of new tokens over the cache: any number of them for every sequence (a piece of a prompt, a turn behind a cached prefix, one token of a decoding
 * step, none), in one batch of rows.  Sequence s brings rows [cu_seqlens[s], cu_seqlens[s + 1]) of Q and out ([rows][Hq][d], strides qo[0], qo[1]; NULL: contiguous),
 * the queries of the last n_s = cu_seqlens[s + 1] - cu_seqlens[s] of the lens[s] tokens that the cache holds of it, their own among them: row i of the n_s sees
 * tokens 0 ... lens[s] - n_s + i.  lse: float [Hq][rows].  cu_seqlens: device int32 [n_seq + 1], as exact_attn_packed_forward takes them and
 * ha_page_plan writes them: values outside [0, rows] are clamped, rows of no sequence are not read and not written, and where they decrease the rows may hold
 * anything, but no access leaves the tensors and the workspace.
 * Everything else as in ha_cache4_attn: products, lens and pages, what counts for nothing, the range of results.
 * rows <= 2^22, rows * Hq <= 2^26, n_seq <= 2^16, n_seq * Hq <= 2^22, Hq % Hk == 0, Hq <= 1024, n_seq * max_blocks <= 2^30, max_blocks * page < 2^31 - 256, n_seq *
 * max_blocks * page <= 2^36.
 * workspace: device, 256-byte aligned, >= ha_cache4_attn_chunk_workspace_bytes() (at most 82 MiB; 0: none is needed, and it may be NULL); nothing in it is kept.  Same inputs, same bits. */
typedef struct {
  int32_t n_seq, rows, Hq;
  int32_t dtype; /* ha_dtype of Q and out */
  int32_t max_blocks;
} ha_cache4_chunk;

int ha_cache4_attn_chunk(const void* Q, const void* cache, const int32_t* cu_seqlens, const int32_t* block_table, const int32_t* lens, void* out,
                         float* lse, const ha_cache4* shape, const ha_cache4_chunk* chunk, const ha_strides* qo, void* workspace,
                         size_t workspace_bytes, void* stream);
size_t ha_cache4_attn_chunk_workspace_bytes(const ha_cache4* shape, const ha_cache4_chunk* chunk); /* 0 too if not valid */

/* What attention weight the cache's tokens got from new queries: for token t of sequence s and key head h the sum, over the rows i of the sequence that see it and the query
 * heads x of h, of exp(<Q[i][x], K[t][h]> - lse[x][i]), by what ha_cache4_attn_chunk (or, with one row a sequence, ha_cache4_attn) gave as lse for the same Q, cu_seqlens,
 * block_table and lens.  Rows of part of the new tokens are taken too, as long as they are the last ones;
 * the other new tokens then count as old, and without fresh what a page held before they came (another sequence's weights, perhaps) is added to.  To have part of the new tokens'
 * rows decide and all new tokens start from 0, bring all rows, those that do not count with lse -inf.
 *   weights: float [n_pages][Hk][page], 16-byte aligned: token t's lies at weights[block_table[s][t / page]][h][t % page], as its rows do in the cache, and goes where
 *   these go.  Tokens that the rows bring (the last cu_seqlens[s + 1] - cu_seqlens[s] of lens[s]) start from 0; for the others the sum is added to what is there,
 *   or, with fresh != 0, also starts from 0.  Nothing else is touched: not what lies behind a sequence, nor pages that no sequence holds.
 *   A page belongs to one sequence and lies once in its row of block_table: where two places name one page it holds the sum of some of them.
 * Sums are fp32 in a fixed order (same inputs, same bits); a row whose lse is -inf gives nothing, one that is NaN makes what it sees NaN, and so does a NaN in K its token.
 * fp32 queries as in ha_cache4_attn.  Sizes as in ha_cache4_attn_chunk.  workspace: device, 256-byte aligned, >= ha_cache4_weights_workspace_bytes() (at most 2 MiB;
 * 0: none is needed, and it may be NULL); nothing in it is kept. */
int ha_cache4_weights(const void* Q, const void* cache, const int32_t* cu_seqlens, const int32_t* block_table, const int32_t* lens, const float* lse,
                      float* weights, const ha_cache4* shape, const ha_cache4_chunk* chunk, int32_t fresh, const ha_strides* q, void* workspace,
                      size_t workspace_bytes, void* stream);
size_t ha_cache4_weights_workspace_bytes(const ha_cache4* shape, const ha_cache4_chunk* chunk); /* 0 too if not valid */

/* Eviction: sequence s, of n = lens[s] tokens, is cut to k = keep[s] (device int32 [n_seq]; negative, or at least n: it stays as it is).  Its last r = min(recent, k) tokens stay,
 * and of the n - r others, for every key head by itself, the k - r of largest weights[page][h][token] (as ha_cache4_weights lays them out), of equal ones the first; NaN,
 * and what lies in a page that is not there, counts less than any number.  Afterwards the sequence has places 0 ... k - 1 of its pages:
 *   places 0 ... k - r - 1: kept tokens that lie there stay; the other kept ones, in order, fill the places between, in order
 *   places k - r ... k - 1: the last r tokens, in order
 * (attention does not ask for the order of tokens that all its rows see; a token's place is another one for every key head).  Rows of K and V move as they lie, and
 * their weights go with them, read from weights and written to weights_out, which may be the same array (entries of rows that stay are not written).  What the places hold that
 * come free is not defined.
 *   lens_out[s]   k, or the length where the sequence stays as it is
 *   free_pages    the pages that its tokens no longer need, block_table[s][ceil(k / page) ... ceil(n / page) - 1], are put on top of the stack, sequences in order
 *   free_count_out  as ha_page_plan has them (at most n_pages)
 * block_table is not changed: lens_out tells which entries count.  Layers whose caches lie by one block table and one stack are cut one after the other, each from the same lens,
 * keep, recent and free_count, so that every call frees the same pages into the same places of the stack; lens_out and free_count_out, the same for all, count from the last layer
 * on.  (With the count that a call has written, the next would put these pages there twice; with its lengths, it would keep the first tokens of its layer.)
 * A page belongs to one sequence and lies once in its row; rows from or to pages that are
 * not there are left out.  lens are taken within [0, max_blocks * page].  lens_out and free_count_out overlap neither each other nor lens, keep
 * and free_count (such calls are refused); nothing else that is written may overlap, but weights_out all of weights.
 * n_seq <= 8192, n_seq * Hk <= 2^20, n_seq * max_blocks <= 2^30, max_blocks * page <= 2^30.  weights, weights_out: 16-byte aligned.
 * workspace: device, 256-byte aligned, >= ha_cache4_evict_workspace_bytes(): four bytes for every token and key head that the table has room for; nothing in it is kept. */
typedef struct {
  int32_t n_seq, max_blocks, recent;
} ha_cache4_eviction;

int ha_cache4_evict(void* cache, const float* weights, float* weights_out, const int32_t* block_table, const int32_t* lens, const int32_t* keep,
                    int32_t* free_pages, const int32_t* free_count, int32_t* lens_out, int32_t* free_count_out, const ha_cache4* shape,
                    const ha_cache4_eviction* evict, void* workspace, size_t workspace_bytes, void* stream);
size_t ha_cache4_evict_workspace_bytes(const ha_cache4* shape, const ha_cache4_eviction* evict); /* 0 too if not valid */

/* Block tables and slots, on the GPU from the sequences' lengths: one launch before a step's rows are written.
 *   lens[s]   tokens that sequence s holds, in pages block_table[s][0 ... ceil(lens / page) - 1]
 *   add[s]    >= 0: rows that the step appends to it; < 0: it has ended, its pages are free again
 *   free_pages, free_count   a stack: free_pages[0 ... *free_count - 1]
 * Pages of sequences that end are put on top of the stack, in order; then every sequence, in order, takes the pages that its new
 * rows need from the top, into its row of block_table.  A sequence whose rows do not fit max_blocks, `rows` or, counted up to it, the free pages gets
 * none, unless it needs none: its length stays, and its rows have no slots.
 *   lens_out[s]     the length after the step (0: ended)
 *   cu_seqlens[s]   rows of the step before sequence s, [n_seq + 1]: as exact_attn_packed_forward takes them
 *   slots[i]        slot of row i, i < rows, as ha_cache4_write takes them; -1: none (also behind the last sequence)
 *   free_count_out  free pages left, free_pages[0 ... *free_count_out - 1]
 * block_table and free_pages are changed in place; nothing else may overlap.  All device int32.  lens are taken within [0, max_blocks * page].
 * n_seq <= 8192, rows <= 2^26, n_seq * max_blocks <= 2^30, page as above, n_pages * page < 2^31. */
typedef struct {
  int32_t n_seq, max_blocks, page, n_pages, rows;
} ha_page_plan_shape;

int ha_page_plan(const int32_t* lens, const int32_t* add, int32_t* block_table, int32_t* free_pages, const int32_t* free_count,
                 int32_t* lens_out, int32_t* cu_seqlens, int32_t* slots, int32_t* free_count_out, const ha_page_plan_shape* shape,
                 void* stream);

/* Measurement aids (no passage of the paper: they serve the roofline report).
 * Both run on `stream`, time themselves with events and WAIT for the stream;
 * `buf` is caller-owned device memory that they overwrite.
 *
 * ha_measure_mfma_rate: bf16 matrix-core rate of register-resident chains of the
 * 32x32x16 MFMA the attention kernels use, over operands that change from one
 * instruction to the next, `iters` loop trips per wave (1..2^20; 1000 take about
 * 1.2 ms, and the rate falls with the duration as the chip lowers its clock), in
 * TFLOP/s.  buf >= 512 KiB.
 * ha_measure_hbm_rate: GB/s of a streaming read of the first half of buf, and of
 * a copy of the first half onto the second (read + written bytes counted).
 * buf 16-byte aligned, bytes >= 1 MiB; use a buffer well beyond the caches.
 * Errors: HA_ERR_NULL, HA_ERR_WORKSPACE (buf too small / misaligned),
 * HA_ERR_SHAPE (iters), HA_ERR_LAUNCH. */
int ha_measure_mfma_rate(void* buf, size_t bytes, int32_t iters, float* tflops, void* stream);
int ha_measure_hbm_rate(void* buf, size_t bytes, float* read_gbs, float* copy_gbs, void* stream);

/* Issue-rate probes (measurement aid): what one trip of small instruction loops costs in
 * shader-clock cycles on this GPU, every CU running the same loop in one workgroup of eight
 * waves (two per SIMD).  cycles_host (host memory) receives 2 * ha_issue_probe_count() floats:
 * for probe p, [2p] is the first wave of the workgroup's first half, [2p+1] of its second half.
 * A trip holds, in this order of p: 64 v_exp_f32; 64 v_fma_f32; 64 v_cvt_pk_bf16_f32; 64
 * v_max3_f32; 16 v_mfma_f32_32x32x16_bf16; 16 MFMAs with 4 fma each; with 7 fma each; with 1 exp
 * + 3 fma each; with 1 exp + 4 fma each; waves 0-3 16 MFMAs while waves 4-7 issue 16 exp + 48 fma;
 * 8 ds_read_b128 per wave (64 KiB read per trip and workgroup); 8 ds_read_b64_tr_b16 (32 KiB);
 * 8 ds_write_b128 (64 KiB).  buf: device memory, 16-byte aligned, >= 1 MiB, overwritten.
 * WAITS for the stream.  Errors: HA_ERR_NULL, HA_ERR_WORKSPACE, HA_ERR_LAUNCH. */
int32_t ha_issue_probe_count(void);
int ha_measure_issue_rates(void* buf, size_t bytes, float* cycles_host, void* stream);

/* Text for an ha_status value. */
const char* ha_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* HYPERATTN_H */
