/*
 * optimus.h — C ABI of the per-device hot path of the 2D (SUMMA) transformer
 * scheme of arXiv 2104.05343, for one AMD MI355X (gfx950).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Pointers.  Every tensor pointer is a DEVICE pointer owned by the caller; the
 *   library neither frees nor retains it.  `stream` is a hipStream_t passed as
 *   void* (NULL = the default stream).  Calls validate their arguments on the
 *   host, enqueue kernels on `stream` and return without synchronising.
 *   The structs (`optimus_layer_cfg`, `optimus_layer_tensors`, `optimus_layer_params`, `optimus_layer_grads`,
 *   `optimus_stack_buffers`, ...) and arrays of them are HOST memory holding device pointers.
 * Grid.  The method distributes every matrix over a q x q device mesh
 *   (Section 2.4): a logical row-major matrix T[R x C] is cut evenly into q*q
 *   sub-blocks, block (r, c) belonging to device (r, c).  This library keeps
 *   all q*q blocks resident on one GPU in BLOCK-MAJOR storage: block (r, c)
 *   starts at element (r*q + c) * (R/q) * (C/q) and is itself row-major with
 *   leading dimension C/q — the contiguous panel a broadcast would deliver.
 *   Vectors of length C (biases, LayerNorm affine) are stored whole; device
 *   column j uses elements j*C/q .. (j+1)*C/q-1.
 * Coordinates.  (i, j) names the device whose share is computed.  i = j =
 *   OPTIMUS_ALL (-1) computes the share of every device in one call ("grid
 *   mode"); mixing -1 with a real coordinate is OPTIMUS_ECOORD.  With explicit
 *   (i, j) a call reads only the peer blocks that device would receive and
 *   writes only that device's output block(s).
 * dtype.  OPTIMUS_FP32: fp32 storage, fp32 FMA accumulation.  OPTIMUS_BF16:
 *   bf16 storage (round-to-nearest-even on store), fp32 accumulation on the
 *   matrix cores; statistics, soft-max sums, weight and bias gradients stay
 *   fp32.
 * Errors.  Return value 0 = OK, otherwise one of the OPTIMUS_E* codes below.
 *   Arguments are checked before anything is enqueued: on EINVAL / ESHAPE /
 *   ECOORD / EDTYPE / EWORKSPACE nothing has been enqueued.  OPTIMUS_EHIP (the
 *   runtime refused a launch) can come from a later kernel of a call that
 *   enqueues several.  No exceptions.  Process state: the tuning hooks at the
 *   end of this file (process-wide, atomic), per device one stream with its
 *   events that optimus_layer_bwd creates on first use (see there), and per
 *   device the fixed scratch array of optimus_attention_fused_bwd_static.
 * Determinism.  No floating-point atomics: the same call on the same inputs
 *   gives bitwise identical output.
 */
#ifndef OPTIMUS_H_
#define OPTIMUS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  OPTIMUS_OK = 0,
  OPTIMUS_EINVAL = 1,     /* null pointer or bad enum value                          */
  OPTIMUS_ESHAPE = 2,     /* size <= 0 or not divisible as the partition requires    */
  OPTIMUS_ECOORD = 3,     /* i or j outside [0, q) and not the OPTIMUS_ALL wildcard  */
  OPTIMUS_EDTYPE = 4,     /* dtype not supported by this entry point                 */
  OPTIMUS_EWORKSPACE = 5, /* workspace missing or smaller than the query says        */
  OPTIMUS_EHIP = 6        /* the HIP runtime refused a launch                        */
};

enum { OPTIMUS_FP32 = 0, OPTIMUS_BF16 = 1 };
enum { OPTIMUS_FORM_AB = 0, OPTIMUS_FORM_ABT = 1, OPTIMUS_FORM_ATB = 2 };
#define OPTIMUS_ALL (-1)

/* Human-readable name of an error code (static string, never NULL). */
const char* optimus_error_string(int code);
/* ABI version of this header (bumped when a signature changes). */
int optimus_abi_version(void);

/* ---- block addressing (Section 2.4: "evenly partitioned into q x q sub-blocks") ----
 * Convert between a row-major logical matrix [R x C] and block-major storage.
 * src and dst are distinct device buffers of R*C elements of elem_bytes (2 or 4)
 * bytes each.  Pure data movement: bit-exact.  ESHAPE unless q | R and q | C. */
int optimus_pack_blocks(const void* src_rowmajor, void* dst_blockmajor, int64_t R, int64_t C,
                        int q, int elem_bytes, void* stream);
int optimus_unpack_blocks(const void* src_blockmajor, void* dst_rowmajor, int64_t R, int64_t C,
                          int q, int elem_bytes, void* stream);

/* ---- the same algorithms step by step, from the COMPUTING device (Algorithms 1-3 as printed) ----
 * optimus_summa_step: what device (i, j) multiplies in step l, as one dense fp32 [M/q x N/q] block c_temp:
 *   AB : A_il B_lj           (both received; accumulated on the same device into C_ij)
 *   ABT: A_ij (B_lj)^T       (B_lj received along column j; reduced within row i onto device (i, l) -> C_il)
 *   ATB: (A_il)^T B_ij       (A_il received along row i; reduced within column j onto device (l, j) -> C_lj)
 * optimus_summa_reduce: the reduce onto its root: adds `count` consecutive partial blocks c_temps[0..count) in
 * index order (the order of the reducing grid index) and writes block (root_i, root_j) of the block-major
 * [M x N] matrix C in `dtype`.  Partials in memory are what the owner-view entry points above avoid; these two
 * exist so that the printed algorithms can be replayed and compared with them.  Operand layouts as above. */
int optimus_summa_step(int form, const void* A, const void* B, float* c_temp, int64_t M, int64_t K, int64_t N,
                       int q, int i, int j, int l, int dtype, void* stream);
int optimus_summa_reduce(const float* c_temps, int count, void* C, int64_t M, int64_t N, int q, int root_i,
                         int root_j, int dtype, void* stream);

/* ---- the three SUMMA products (Section 2.4, Algorithms 1-3, Eq. 1-3) ----
 * (M, N) is always the logical OUTPUT shape and K the logical contraction
 * length; all three must be positive multiples of q.  A, B, C are block-major.
 * Device (i, j) ends up holding (owner view of Algorithms 1-3; the per-step
 * broadcasts become reads of resident peer blocks, the row/column reduce of
 * Algorithms 2-3 becomes the sum over l inside one accumulator):
 *   optimus_summa_ab :  C_ij = sum_l A_il   * B_lj      A[M x K], B[K x N]
 *   optimus_summa_abt:  C_ij = sum_l A_il   * (B_jl)^T  A[M x K], B[N x K]
 *   optimus_summa_atb:  C_ij = sum_l (A_li)^T * B_lj    A[K x M], B[K x N]
 * The q panel steps are fused into one k-loop; C is written once.  C must not
 * alias A or B.
 * ws / ws_bytes: optional device scratch (may be NULL / 0).  When it is at
 * least optimus_summa_workspace_bytes(...) the library may split the panel
 * loop of skinny outputs over several workgroups and combine the fp32 partial
 * tiles in a fixed order (still deterministic); without it the same split is
 * walked inside the workgroups, with the same bits. */
int optimus_summa_ab(const void* A, const void* B, void* C, int64_t M, int64_t K, int64_t N,
                     int q, int i, int j, int dtype, void* ws, size_t ws_bytes, void* stream);
int optimus_summa_abt(const void* A, const void* B, void* C, int64_t M, int64_t K, int64_t N,
                      int q, int i, int j, int dtype, void* ws, size_t ws_bytes, void* stream);
int optimus_summa_atb(const void* A, const void* B, void* C, int64_t M, int64_t K, int64_t N,
                      int q, int i, int j, int dtype, void* ws, size_t ws_bytes, void* stream);
size_t optimus_summa_workspace_bytes(int form, int64_t M, int64_t K, int64_t N, int q, int i, int j,
                                     int dtype);

/* Epilogue applied to the accumulator of a SUMMA product before the single
 * store of C_ij (Section 3.2.1: non-linearities are applied locally per
 * block; Section 3.2.2: bias-add uses the column slice of a row-0 parameter).
 * In order:  t = acc;  t += bias[j-slice];  if pre_act: pre_act_ij = t;
 * if act == 1: t = GeLU(t) (exact, x*Phi(x));  if gelu_grad_of: t *= GeLU'(gelu_grad_of_ij);
 * if residual: t += residual_ij;  C_ij = t.
 * bias is fp32 [N]; pre_act, gelu_grad_of, residual are block-major [M x N]
 * in the call's dtype.  out_fp32 != 0 stores C as fp32 even for bf16 inputs
 * (weight gradients).  Any pointer may be NULL to skip its step. */
typedef struct {
  const float* bias;
  void* pre_act;
  int act;
  const void* gelu_grad_of;
  const void* residual;
  int out_fp32;
} optimus_epilogue;

/* form: OPTIMUS_FORM_*.  epi may be NULL (plain product). */
int optimus_summa_ex(int form, const void* A, const void* B, void* C, int64_t M, int64_t K, int64_t N,
                     int q, int i, int j, int dtype, const optimus_epilogue* epi, void* ws,
                     size_t ws_bytes, void* stream);

/* Bias gradient (Section 3.2.2, bias-add backward): device (i, j)'s partial
 * = column sums of its block dY_ij; the reduce up the column to row 0 is the
 * sum over i of these partials.  dY block-major [M x N]; out fp32
 * [q][q][N/q], entry (i, j) written. */
int optimus_bias_grad(const void* dY, float* dbias_part, int64_t M, int64_t N, int q, int i, int j,
                      int dtype, void* stream);

/* ---- 2D LayerNorm (Section 3.2.2) ----
 * X block-major [M x H]; a row's H entries are spread over the q devices of
 * grid row i.  stats is fp32 [q][q][M/q][2]: entry (i, l) holds what device
 * (i, l) contributes to the row all-reduce, (sum x, sum x^2) per local row in
 * forward and (sum xhat*g, sum g) with g = dy*gamma in backward.
 *
 * optimus_layernorm2d_stats(i, l): writes device (i, l)'s forward partial only.
 * optimus_layernorm2d(i, j): computes its own partial (and stores it in
 *   stats[i][j]), adds the q-1 peer partials already in stats[i][*], then
 *   xhat = (x - E[x]) * rstd, rstd = 1/sqrt(max(E[x^2]-E[x]^2, 0) + eps),
 *   y = gamma_j*xhat + beta_j.  Writes Y_ij, xhat_ij (same dtype as X) and
 *   rstd (fp32 [q][q][M/q], entry (i, j)).  In grid mode all partials are
 *   produced first, so no prior _stats call is needed.
 * optimus_layernorm2d_bwd(i, j): dX_ij = rstd*(g - xhat*mean(xhat*g) - mean(g))
 *   [+ dres_ij if dres != NULL: gradient arriving over the residual branch],
 *   with the two means taken over the whole row via `stats` exactly as in
 *   forward; dgamma_part/dbeta_part fp32 [q][q][H/q]: column sums of dy*xhat
 *   and dy over the block's rows (entry (i, j) written).
 * gamma, beta: fp32 [H]. */
int optimus_layernorm2d_stats(const void* X, float* stats, int64_t M, int64_t H, int q, int i, int l,
                              int dtype, void* stream);
int optimus_layernorm2d(const void* X, const float* gamma, const float* beta, void* Y, void* xhat,
                        float* rstd, float* stats, int64_t M, int64_t H, int q, int i, int j,
                        float eps, int dtype, void* stream);
int optimus_layernorm2d_bwd_stats(const void* dY, const void* xhat, const float* gamma, float* stats,
                                  int64_t M, int64_t H, int q, int i, int l, int dtype, void* stream);
int optimus_layernorm2d_bwd(const void* dY, const void* xhat, const float* rstd, const float* gamma,
                            const void* dres, void* dX, float* dgamma_part, float* dbeta_part,
                            float* stats, int64_t M, int64_t H, int q, int i, int j, int dtype,
                            void* stream);

/* ---- head-partitioned attention on the device's blocks (Sections 2.1, 3.2.1) ----
 * Device (i, j) holds n/q heads of b/q whole sequences.  qkv is block-major
 * [b*s x 3h] (rows sequence-major: row = seq*s + t; columns head-major:
 * head*3d + {0:Q,1:K,2:V}*d + e with d = h/n), so block (i, j) contains Q, K,
 * V of heads j*n/q.. of sequences i*b/q...  For every local (sequence, head):
 * S = Q K^T / sqrt(d), causal mask if causal != 0, P = softmax rows (fp32),
 * O = P V.  probs: [q][q][(b/q)*(n/q)][s][s] in the call's dtype (entries above
 * the diagonal are exact zeros when causal); attn: block-major [b*s x h].
 * Backward: dV = P^T dO, dP = dO V^T, dS = P*(dP - rowsum(dP*P)),
 * dQ = dS K / sqrt(d), dK = dS^T Q / sqrt(d); d_qkv has qkv's layout.
 * ws must hold optimus_attention_workspace_bytes(...) bytes (scratch for one
 * device's scores); a whole-grid call (i = j = -1) takes g devices per launch
 * when ws holds g times that (same bits, fewer and larger launches). bf16 only.
 * Requires q | b, q | n, n | h, d % 8 == 0, s % 8 == 0, s <= 4096 (what the
 * soft-max over scores in memory holds in one wavefront, which some sizes still
 * take; longer sequences: optimus_attention_fused_*);
 * OPTIMUS_ESHAPE otherwise. */
int optimus_attention_fwd(const void* qkv, void* probs, void* attn, int b, int s, int h, int n, int q,
                          int i, int j, int causal, int dtype, void* ws, size_t ws_bytes, void* stream);
int optimus_attention_bwd(const void* qkv, const void* probs, const void* d_attn, void* d_qkv, int b,
                          int s, int h, int n, int q, int i, int j, int causal, int dtype, void* ws,
                          size_t ws_bytes, void* stream);
size_t optimus_attention_workspace_bytes(int b, int s, int h, int n, int q);

/* ---- the row soft-max of attention by itself ("Nonlinear" of Section 2.1; local per device, Section 3.2.1) ----
 * The two bandwidth-bound kernels between the attention products, exported so that they can be measured and
 * tested alone.  scores / d_probs: nmat matrices [s x s] fp32, contiguous; probs / d_scores: the same shape in
 * bf16.  Forward: P = softmax over each row of S (with causal != 0 only columns <= row take part and the entries
 * above the diagonal are written as exact zeros).  Backward: dS = P * (dP - rowsum(dP * P)) row by row (entries
 * of dP above the diagonal are not read when causal).  Device memory; requires s % 4 == 0, 4 <= s <= 4096,
 * nmat >= 1, nmat * s < 2^31 (OPTIMUS_ESHAPE otherwise); null pointers: OPTIMUS_EINVAL. */
int optimus_softmax_rows(const float* scores, void* probs, int64_t nmat, int s, int causal, void* stream);
int optimus_softmax_rows_bwd(const float* d_probs, const void* probs, void* d_scores, int64_t nmat, int s,
                             int causal, void* stream);

/* ---- the same attention without the [s x s] tensors (the operator fusion proposed in Section 6) ----
 * Same qkv / attn / d_qkv layouts and the same mathematics as above, but neither scores nor probabilities are
 * ever written to memory, so sequence length is no longer bounded by the [b/q, n/q, s, s] tensor.  The forward
 * keeps, per query row, lse = log sum_u exp(S_tu) (natural logarithm of the scaled, masked scores):
 * lse is [q][q][(b/q)*(n/q)][s] fp32 in device order; the backward rebuilds P = exp(S - lse) tile by tile and
 * uses rowsum(dO * O) for rowsum(dP * P), so it also reads the forward's attn output.
 * Device memory, all of them; ws (backward only) must hold optimus_attention_fused_workspace_bytes(...) bytes.
 * bf16 only; head width d = h/n must be 64 or 128 (OPTIMUS_ESHAPE otherwise); any s >= 1 up to 2^20;
 * requires q | b, q | n, n | h. */
int optimus_attention_fused_fwd(const void* qkv, void* attn, float* lse, int b, int s, int h, int n, int q,
                                int i, int j, int causal, int dtype, void* stream);
int optimus_attention_fused_bwd(const void* qkv, const void* attn, const float* lse, const void* d_attn,
                                void* d_qkv, int b, int s, int h, int n, int q, int i, int j, int causal,
                                int dtype, void* ws, size_t ws_bytes, void* stream);
size_t optimus_attention_fused_workspace_bytes(int b, int s, int h, int n, int q);

/* ---- optimus_attention_fused_bwd for callers that cannot allocate ----
 * For code under HIP graph capture, tight serving loops and harnesses that forbid hipMalloc: the same operation,
 * arguments, layouts and results (bit for bit) as optimus_attention_fused_bwd, without the ws argument.  The one
 * scratch buffer of that call (one fp32 per query row of every (sequence, head) matrix of the launch) lives in a
 * static device array of OPTIMUS_STATIC_SCRATCH_BYTES that every GPU the library runs on holds until the process
 * ends; the call allocates and frees nothing.  A launch that needs more -- (i = j = -1 ? q*q : 1) * (b/q) * (n/q)
 * * s * 4 bytes -- is rejected with OPTIMUS_EWORKSPACE before anything is enqueued.  All calls on one GPU share
 * the array (it keeps the last call's contents; every call overwrites what it reads, nothing needs clearing):
 * two calls that overlap on one GPU (different streams, several host threads) race on it.  The array's address
 * is looked up on the first call made with a device current; make that first call outside stream capture. */
#define OPTIMUS_STATIC_SCRATCH_BYTES (4u << 20)
int optimus_attention_fused_bwd_static(const void* qkv, const void* attn, const float* lse, const void* d_attn,
                                       void* d_qkv, int b, int s, int h, int n, int q, int i, int j,
                                       int causal, int dtype, void* stream);

/* ---- the same attention with changed scores: capped, biased by distance, masked by documents or opened by a prefix ----
 * Layouts, lse, d_qkv, coordinates and limits as in optimus_attention_fused_*; per pair (t, u) of a (sequence, head):
 *   S = Q K^T / sqrt(d);  with cap from 1e-3 to 1e30: S = cap tanh(S / cap), 0: none, others EINVAL;
 *   with slopes: S -= slopes[head] |t - u|;  or, with table: S += table[head][bucket(t - u)] (not both: EINVAL).
 * A pair is left out
 *   with causal != 0 where u > t, unless u < prefix[sequence] (prefix needs causal != 0: EINVAL; values are clamped to 0 .. s);
 *   with documents where documents[t] != documents[u], or either is negative: a token of a negative document is padding;
 *   where the table's number is -1e30 or less (-infinity included).
 * A row without a pair has attn 0, lse -infinity and gradients 0.  What qkv, attn and d_attn hold in rows of padding is not looked at,
 * NaN included; their rows of attn and d_qkv are written as zeros.  (Other pairs that are left out have weight zero, and zero times
 * an infinity or NaN is NaN: as without changes, the values of tokens that are not padding are taken to be finite.)
 * Accuracy: P, and dS in the backward, are rounded to bf16 before their products with V, dO, Q and K, as the operands are; sums, soft-max
 * statistics and scores are fp32.  The tanh is off by at most 3e-7 (a cap of 50: 1.4e-5 of a score), with a cap beyond 64 only from a
 * quarter of the cap on, below it by a few roundings of itself.  The forward takes finite scores of any size.  In the backward
 * P = exp(S - lse), at most 1, is off by some 2e-7 |S| of itself, the rounding of an fp32 lse: little up to scores of 1e4; from 1e7 on the
 * gradients of such a row mean nothing, those of others are not touched.
 * bucket(n) of the distance n = t - u: a side has `side` buckets: buckets, or buckets / 2 with two_sided; near = side / 2.  Distances
 * 0 .. near - 1 have a bucket each; bucket near + k begins at the first whole number not below near * (max_distance / near)^(k / (side -
 * near)); the last has no end.  n < 0 (a later key): bucket 0, or with two_sided side + bucket(-n).  2 <= side, even `buckets` with
 * two_sided, buckets <= 128, near < max_distance <= 1024 (ESHAPE).
 * Backward: S is rebuilt and P = exp(S - lse); dS = P (dO V^T - rowsum(dO attn)); d_table sums dS over the pairs of a bucket; then
 * dS (1 - tanh^2) is the gradient of Q K^T / sqrt(d).  d_table: fp32 [q][q][n/q * buckets], entry (i, j) written: device (i, j)'s partial,
 * the gradient of table rows j*n/q .. is the sum over i; NULL: not computed.  No gradient of slopes.
 * slopes: fp32 [n]; table: fp32 [n][buckets]; documents: int32 [b*s], in any order; prefix: int32 [b]: device memory or NULL.
 * ws: optimus_attention_biased_workspace_bytes(...) bytes (0 for arguments that are refused), 16-byte aligned; the forward needs it with
 * documents only.  Calls that may overlap need a workspace each.  (n/q + 1) * b/q <= 65535, b/q * n/q * ceil(s/64) < 2^23 (ESHAPE). */
typedef struct {
  float cap;
  const float* slopes;
  const float* table;
  int buckets, max_distance, two_sided;
  const int32_t* documents;
  const int32_t* prefix;
} optimus_attention_bias;
int optimus_attention_biased_fwd(const void* qkv, void* attn, float* lse, int b, int s, int h, int n, int q, int i, int j, int causal,
                                 int dtype, const optimus_attention_bias* bias, void* ws, size_t ws_bytes, void* stream);
int optimus_attention_biased_bwd(const void* qkv, const void* attn, const float* lse, const void* d_attn, void* d_qkv, float* d_table,
                                 int b, int s, int h, int n, int q, int i, int j, int causal, int dtype,
                                 const optimus_attention_bias* bias, void* ws, size_t ws_bytes, void* stream);
size_t optimus_attention_biased_workspace_bytes(int b, int s, int h, int n, int q, const optimus_attention_bias* bias);

/* ---- attention over chosen blocks of keys ----
 * For sequences too long for all pairs: keys come in blocks of `block` (a multiple of 64, up to 4096; at most 1024 blocks in a sequence), and
 * a query attends to `count` blocks (1 .. 64) at most.  Two steps, of which the second takes any choice:
 * optimus_attention_select(qkv): mean[v] = mean of block v's keys (sum in 64 bits, rounded to fp32 and then to bf16); a query t chooses its
 *   own block, t / block, and the count - 1 others with the largest products q_t . mean[v]: with causal != 0 among the blocks in front of
 *   its own, else among all.  The order is that of the exact products (fp32 ones decide where they leave no doubt, 64-bit ones else); of
 *   equal ones the lower block is chosen, a product that is NaN is below all others.  selected int32 [q][q][(b/q)*(n/q)][s][count] in device
 *   order: ascending, -1 behind them.  No gradient goes through the choice.
 * optimus_attention_selected_fwd: S = Q K^T / sqrt(d) over the keys of the blocks in `selected` (causal != 0: and u <= t), P = softmax, O = P V,
 *   lse as in optimus_attention_fused_*.  Entries in any order; those below 0, beyond the sequence, repeated, or of blocks that a causal query
 *   does not see count as not there.  A query without a key has attn 0, lse -infinity and gradients 0.
 * optimus_attention_selected_bwd: from the same `selected` and the forward's attn and lse: P = exp(S - lse), dS = P (dO V^T - rowsum(dO attn)).
 * lengths: int32 [b] device memory or NULL (all s): tokens of a sequence that count (clamped to 0 .. s).  What qkv and d_attn hold behind them
 * is not looked at, NaN included; there selected is -1, attn 0, lse -infinity and d_qkv 0.
 * P and dS are rounded to bf16 before their products, as the operands are, and what a query gets from one block may be rounded to 11 bits (fp16,
 * scaled) before the blocks' parts are added; scores and sums are fp32; lse enters as in optimus_attention_biased_bwd: the
 * forward takes finite scores of any size, the gradients of a row mean something up to scores of 1e7.  The values of tokens inside the lengths
 * are taken to be finite: a pair that is left out has weight zero, and zero times an infinity or NaN is NaN.
 * qkv, attn, d_attn, d_qkv (16-byte aligned: EINVAL), lse, coordinates and limits as in optimus_attention_fused_*; bf16 only;
 * b*n (whole grid) or b/q * n/q (one device) up to 65535, q up to 46340, 3h < 2^31 (ESHAPE).
 * ws: optimus_attention_selected_workspace_bytes(...) bytes for all three (0 for arguments that are refused), 256-byte aligned, nothing kept in it
 * from call to call: calls that may overlap need one each.  It holds some 9 bytes an entry of the choice, 40 a query and 1024 a (sequence, head),
 * and up to 1 GiB of partial results, or where that is more one (sequence, head)'s: at most d * (3 s * count + 8 (s + block)) bytes.
 * How it is computed (all blocks with a mask, or lists of each block's queries), and with it the last bits, follows the sizes, those of one
 * device whatever the call covers: b/q and n/q too, so that a sequence alone and the same one in a batch may differ in their last bits. */
typedef struct {
  int block, count;
  const int32_t* lengths;
} optimus_selection;
int optimus_attention_select(const void* qkv, int32_t* selected, int b, int s, int h, int n, int q, int i, int j, int causal, int dtype,
                             const optimus_selection* selection, void* ws, size_t ws_bytes, void* stream);
int optimus_attention_selected_fwd(const void* qkv, const int32_t* selected, void* attn, float* lse, int b, int s, int h, int n, int q, int i, int j,
                                   int causal, int dtype, const optimus_selection* selection, void* ws, size_t ws_bytes, void* stream);
int optimus_attention_selected_bwd(const void* qkv, const int32_t* selected, const void* attn, const float* lse, const void* d_attn, void* d_qkv,
                                   int b, int s, int h, int n, int q, int i, int j, int causal, int dtype, const optimus_selection* selection,
                                   void* ws, size_t ws_bytes, void* stream);
size_t optimus_attention_selected_workspace_bytes(int b, int s, int h, int n, int q, int i, int j, const optimus_selection* selection);

/* ---- rotary positions of one to four axes, between the 3h projection and the attention ----
 * The attention above knows the order of its tokens by masks and biases only; rotary positions turn queries and keys by angles, so that
 * their products depend on differences of positions.  Layouts, coordinates as in optimus_attention_*; dtype FP32 or BF16, any head width up
 * to 4096.  With P the sum of pairs[0 .. axes), pair p < P of every head's query and key are its elements p and P + p, or with interleaved
 * 2p and 2p + 1; further elements, and values, are not changed.  A pair belongs to an axis: the first pairs[0] to axis 0, the next to axis 1
 * and so on, or with in_turn the axes take turns, one pair each, those that have all of theirs passed over.  Its frequency is
 * base^(-k / pairs[axis]) for the k-th pair of its axis, or with shared_ladder base^(-p / P).
 *   angle = positions[axis][token] * scale[axis] * frequency;  (x, y) -> (x cos - y sin, x sin + y cos)
 * The angle is a product of 64 bits, its whole turns are taken off before it is rounded to fp32.  positions: int32 device memory [axes][b*s]
 * (rows sequence-major, every device of a grid row reads the same ones), of any sign; host: scale and base > 0, finite, scale * frequency below
 * 2 pi 2^20, 2^20 turns a position (EINVAL).
 * optimus_rotary writes the blocks of `out` whole, values too; out == qkv turns them in place; blocks that overlap otherwise: EINVAL.
 * optimus_rotary_bwd is the gradient, the turn by -angle: of d_out with respect to qkv, in place with d_qkv == d_out.
 * axes 1 .. 4, pairs[] >= 1, P <= 128, 2P <= h/n, even h/n with interleaved, 3h/q <= 2^18, 3h < 2^31, q <= 46340, b/q * s below 2^24
 * (up to eight times as many where rows are narrow) (ESHAPE).  Pointers need the alignment of their elements
 * only.  The struct is read before the call returns; one row (s = 1) is a call like any other. */
typedef struct {
  const int32_t* positions;
  int axes;
  int pairs[4];
  double scale[4];
  double base;
  int interleaved, in_turn, shared_ladder;
} optimus_rotary_axes;
int optimus_rotary(const void* qkv, void* out, int b, int s, int h, int n, int q, int i, int j, int dtype, const optimus_rotary_axes* axes,
                   void* stream);
int optimus_rotary_bwd(const void* d_out, void* d_qkv, int b, int s, int h, int n, int q, int i, int j, int dtype,
                       const optimus_rotary_axes* axes, void* stream);

/* ---- one transformer layer on device (i, j) (Section 3.2; Eq. 1) ----
 * Wiring: a1 = LN1(x); qkv = a1 Wqkv + b; attn = local attention;
 * h_mid = x + attn Wo + b; a2 = LN2(h_mid); pre = a2 W1 + b; g = GeLU(pre);
 * out = h_mid + g W2 + b.  Backward follows Eq. 1 for every linear layer
 * (dX = dY W^T by the AB^T product, dW = X^T dY by the A^T B product), uses the
 * saved activations (no recomputation) and no dropout.
 * Every matrix is block-major over the q x q grid; vectors are fp32 and whole.
 * In grid mode (i = j = -1) each stage runs for all q*q devices before the
 * next starts, filling every block of every tensor.  With explicit (i, j) only
 * that device's blocks are recomputed; peers' blocks of the previous stage must
 * be resident (left by a grid-mode call on the same tensors).
 * Shared memory in the backward pass.  A matrix that it writes may lie where another one lies that is not needed
 * any more, in this order: d_pre_gelu; d_w2, d_b2; d_ln2_out; d_w1, d_b1; d_ln2_g, d_ln2_b, d_h_mid (from d_ln2_out, xhat2, d_out); d_attn;
 * d_w_o, d_b_o; d_qkv; d_ln1_out; d_w_qkv, d_b_qkv; d_ln1_g, d_ln1_b, d_x (from d_ln1_out, xhat1, d_h_mid).  In place, element for
 * element: d_pre_gelu of pre_gelu, d_h_mid of d_out or d_ln2_out, d_x of d_h_mid or d_ln1_out.  Where the faster schedules would
 * still read what is overwritten, the pass keeps to that order on `stream`, with the same bits.  Statistics and vector gradients share
 * memory with nothing.  (What has been overwritten is of course no peer's block for a later call on one device.) */
typedef struct {
  int b, s, h, n, q;
  float eps;
  int causal;
  int dtype; /* OPTIMUS_BF16 only */
  int fused_attention; /* 0: scores and probabilities in memory (probs saved for the backward pass);
                          1: optimus_attention_fused_* (lse saved instead; needs h/n = 64 or 128) */
} optimus_layer_cfg;

typedef struct {
  /* inputs / parameters */
  const void* x;      /* [M x h]  */
  const float* ln1_g; const float* ln1_b;  /* [h] */
  const void* w_qkv;  /* [h x 3h] */
  const float* b_qkv; /* [3h]     */
  const void* w_o;    /* [h x h]  */
  const float* b_o;   /* [h]      */
  const float* ln2_g; const float* ln2_b;  /* [h] */
  const void* w1;     /* [h x 4h] */
  const float* b1;    /* [4h]     */
  const void* w2;     /* [4h x h] */
  const float* b2;    /* [h]      */
  /* forward tensors, written by optimus_layer_fwd, read by optimus_layer_bwd */
  void* ln1_out; void* xhat1; float* rstd1; float* stats1; /* [M x h], [M x h], [q][q][M/q], [q][q][M/q][2] */
  void* qkv;      /* [M x 3h] */
  void* probs;    /* [q][q][(b/q)(n/q)][s][s]; unused (may be NULL) with fused_attention */
  void* attn;     /* [M x h]  */
  void* h_mid;    /* [M x h]  */
  void* ln2_out; void* xhat2; float* rstd2; float* stats2;
  void* pre_gelu; /* [M x 4h] */
  void* gelu;     /* [M x 4h] */
  void* out;      /* [M x h]  */
  /* backward: input gradient, activation gradients (resident for peers), outputs */
  const void* d_out;  /* [M x h] */
  void* d_pre_gelu;   /* [M x 4h] */
  void* d_ln2_out;    /* [M x h]  */
  void* d_h_mid;      /* [M x h]  */
  void* d_attn;       /* [M x h]  */
  void* d_qkv;        /* [M x 3h] */
  void* d_ln1_out;    /* [M x h]  */
  void* d_x;          /* [M x h]  */
  float* bstats1; float* bstats2; /* [q][q][M/q][2] backward LayerNorm partials */
  float* d_w_qkv; float* d_w_o; float* d_w1; float* d_w2;         /* fp32, block-major, weight shapes */
  float* d_b_qkv; float* d_b_o; float* d_b1; float* d_b2;         /* fp32 partials [q][q][N/q]        */
  float* d_ln1_g; float* d_ln1_b; float* d_ln2_g; float* d_ln2_b; /* fp32 partials [q][q][h/q]        */
  float* lse;     /* [q][q][(b/q)(n/q)][s] fp32, forward tensor; only with fused_attention (else may be NULL) */
} optimus_layer_tensors;

/* Scratch bytes optimus_layer_fwd / _bwd want in `ws`: attention scores and
 * their gradients for one device -- with fused_attention only one fp32 per
 * query row --, plus split-k partial tiles: one region for
 * the activation chain and one for the parameter gradients, with room for all
 * four weight gradients' tiles where a pass runs on `stream` alone and combines
 * them at its end.  Less is accepted down to regions of the largest product's
 * tiles: each weight gradient is then combined at once, with the same bits.
 * In longer passes optimus_layer_bwd runs the parameter gradients concurrently
 * on a stream of the library's own that
 * it forks from and joins back into `stream` with events; when the call
 * returns, every kernel of both is ordered before later work on `stream`.
 * The library creates that stream (default priority) and its events on the
 * first call per device that is not made under stream capture; until then the
 * branch runs on `stream` itself, as it does in every call too short for a
 * second stream to pay unless that call is captured, and where matrices share
 * memory that both streams would use.  They are shared by all
 * calls on a device:
 * optimus_layer_bwd must not be called from several host threads at once
 * for the same device. */
size_t optimus_layer_workspace_bytes(const optimus_layer_cfg* cfg);
/* The size to give whole-grid calls (i = j = -1) that should run fast: the minimum above plus attention scratch
 * for more devices, so that the unfused attention of several devices is one batch per launch instead of one device
 * after the other (as many as stay inside the 256 MB Infinity Cache, at least one).  optimus_layer_fwd / _bwd use
 * whatever `ws_bytes` holds beyond the products' regions for this; the results do not depend on it, bit for bit. */
size_t optimus_layer_workspace_bytes_grid(const optimus_layer_cfg* cfg);
int optimus_layer_fwd(const optimus_layer_cfg* cfg, const optimus_layer_tensors* t, int i, int j,
                      void* ws, size_t ws_bytes, void* stream);
int optimus_layer_bwd(const optimus_layer_cfg* cfg, const optimus_layer_tensors* t, int i, int j,
                      void* ws, size_t ws_bytes, void* stream);

/* ---- a stack of identical layers with distributed activation checkpointing and pre-allocated buffers
 *      (Section 3.2.3 "memory pre-allocation and checkpointing" and its figure; Table 1's backward rows) ----
 * Forward keeps only the input of every layer (checkpoint[l], [M x h] block-major each: b*s*h/p elements per device
 * and layer); all layers share ONE set of forward tensors (forward buffer), ONE set of activation gradients
 * (backward buffer), two [M x h] slots for the gradient passed between consecutive layers (conjunction buffer) and
 * the workspace.  Backward recomputes layer l's forward pass from checkpoint[l] (without its last product, which
 * no gradient needs), then runs optimus_layer_bwd on it, for l = L-1 .. 0.
 * grads[l] says where layer l's parameter gradients go (layouts as in optimus_layer_tensors); entries may all
 * point into one parameter-gradient buffer if the caller consumes them in `done`, which is called on the host
 * after layer l's backward kernels have been enqueued (stream-ordered work enqueued from it sees the gradients and
 * precedes the next layer's; may be NULL).
 * These calls compute every device's share (grid mode): buffers that all layers share cannot keep the peers' blocks
 * of every layer resident.  x, out, d_out, d_x: [M x h] block-major device memory; buffers: device memory of at least
 * the sizes optimus_stack_sizes_of reports (256-byte aligned); params / grads: host arrays of n_layers entries of
 * device pointers.  The caller's out and d_x must not alias the buffers. */
typedef struct {
  const float* ln1_g; const float* ln1_b; const void* w_qkv; const float* b_qkv; const void* w_o; const float* b_o;
  const float* ln2_g; const float* ln2_b; const void* w1; const float* b1; const void* w2; const float* b2;
} optimus_layer_params;
typedef struct {
  float* d_w_qkv; float* d_w_o; float* d_w1; float* d_w2; float* d_b_qkv; float* d_b_o; float* d_b1; float* d_b2;
  float* d_ln1_g; float* d_ln1_b; float* d_ln2_g; float* d_ln2_b;
} optimus_layer_grads;
typedef struct { size_t workspace, forward, backward, param_grad, conjunction, checkpoint; } optimus_stack_sizes;
typedef struct { void* workspace; void* forward; void* backward; void* conjunction; void* checkpoint; } optimus_stack_buffers;
typedef void (*optimus_layer_done_fn)(int layer, void* user);
int optimus_stack_sizes_of(const optimus_layer_cfg* cfg, int n_layers, optimus_stack_sizes* out);
/* Lays one layer's parameter gradients out in a buffer of optimus_stack_sizes.param_grad bytes. */
int optimus_layer_grads_in(const optimus_layer_cfg* cfg, void* param_grad, optimus_layer_grads* out);
int optimus_stack_fwd(const optimus_layer_cfg* cfg, int n_layers, const optimus_layer_params* params, const void* x,
                      const optimus_stack_buffers* buf, void* out, void* stream);
int optimus_stack_bwd(const optimus_layer_cfg* cfg, int n_layers, const optimus_layer_params* params,
                      const optimus_layer_grads* grads, const void* d_out, const optimus_stack_buffers* buf, void* d_x,
                      optimus_layer_done_fn done, void* user, void* stream);

/* ---- the ends of the model in the 2D partition (Section 3.2.1, last paragraph; Section 3.2.2, cross entropy) ----
 * tokens / labels: int32 [b*s] (rows sequence-major, as everywhere): grid row i owns entries i*M/q ..; every device of
 * a grid row reads the same ones.  Indices outside [0, v) are clamped into range (no error is raised from a kernel).
 * table: block-major [v x h] (block (l, j) = rows l*v/q.., columns j*h/q..).
 * optimus_embedding_fwd(i, j): x_ij[t] = table[tokens[t]] restricted to columns j, i.e. the paper's one-hot product
 *   sum_l onehot_il table_lj (Algorithm 1) as a row gather; x block-major [M x h]; bit-exact copy.
 * optimus_embedding_bwd(l, j): the owner's block of the table gradient, d_table_lj = sum_i onehot_il^T dX_ij (the
 *   A^T B form, Algorithm 3, reduced within column j onto (l, j)); reads ALL token indices and the blocks (i, j) of
 *   d_x of every i (resident peers); d_table fp32 block-major [v x h], block (l, j) written completely (zeros where
 *   no token refers to a row); sums in fp32 in the order of the tokens (deterministic).
 * lm-head logits = hidden table^T: optimus_summa_abt(hidden, table, logits, M, h, v, ...).
 * Cross entropy over logits block-major [M x v] (a row spans the q devices of a grid row):
 *   stats fp32 [q][q][M/q][2]: entry (i, l) = (max, sum exp(x - max)) over device (i, l)'s columns;
 *   optimus_cross_entropy2d_stats(i, l) writes that partial only; optimus_cross_entropy2d(i, j) computes its own
 *   partial, combines the q partials of row i in the order l = 0..q-1 (peers' partials resident, as with LayerNorm),
 *   and writes loss[i][j][t] = log sum_k exp(x_tk) - x_t,label and lse[i][j][t] (both fp32 [q][q][M/q]; the q
 *   devices of a row write identical values).  optimus_cross_entropy2d_bwd(i, j):
 *   d_logits_ij = scale * (exp(x - lse) - [column == label]) in the logits' dtype (the soft-max is rebuilt from lse
 *   instead of being saved).  i = j = -1 runs every device.  dtype fp32 or bf16. */
int optimus_embedding_fwd(const int32_t* tokens, const void* table, void* x, int64_t M, int64_t v, int64_t h,
                          int q, int i, int j, int dtype, void* stream);
int optimus_embedding_bwd(const int32_t* tokens, const void* d_x, float* d_table, int64_t M, int64_t v, int64_t h,
                          int q, int l, int j, int dtype, void* stream);
int optimus_cross_entropy2d_stats(const void* logits, float* stats, int64_t M, int64_t v, int q, int i, int l,
                                  int dtype, void* stream);
int optimus_cross_entropy2d(const void* logits, const int32_t* labels, float* loss, float* lse, float* stats,
                            int64_t M, int64_t v, int q, int i, int j, int dtype, void* stream);
int optimus_cross_entropy2d_bwd(const void* logits, const int32_t* labels, const float* lse, void* d_logits,
                                float scale, int64_t M, int64_t v, int q, int i, int j, int dtype, void* stream);

/* ---- the norm of all gradients, and clipping by it, between the backward pass and the update ----
 * norm = sqrt(sum over tensors and elements of g^2), g the sum of an element's parts in fp32, in their order (partial gradients [q][q][N/q] of
 * optimus_layer_bwd are q parts of N elements); squares and their sums in 64 bits.  scale = max_norm / norm where norm is above max_norm, else 1:
 * what optimus_adamw_cfg.grad_scale takes, so that an optimus_adamw_step behind optimus_stack_bwd clips without a pass of its own
 * (optimus_stack_bwd_adamw updates a layer before the gradients of all are there).  A gradient that holds an infinity or NaN: scale
 * is NaN.  norm: 1 float; scale: 1 float or NULL; norms: [count], each tensor's own, or NULL: device memory, written.  max_norm > 0, infinity
 * included (EINVAL).  ws: optimus_gradient_norm_workspace_bytes(...) bytes (0 for a list that is refused), 8-byte aligned.
 * optimus_gradient_clip: clipped = *scale * g, in the gradient's dtype, the parts added (in fp32, in order): clipped[n] may be grad
 * itself (in place, with parts its first n elements; a scale of 1 then leaves a gradient without parts as it is), else it meets no
 * other clipped and no gradient (EINVAL).  The norm does not look at clipped.
 * gradients: host array, read before the call returns.  Pointers need the alignment of their elements only.  n from 1 to 2^34, parts to 65536,
 * count to 65536 (ESHAPE).  A captured call reads the addresses it was captured with. */
typedef struct {
  const void* grad;    /* [parts][n] */
  void* clipped;       /* [n]; optimus_gradient_clip only */
  int64_t n;
  int dtype;           /* OPTIMUS_FP32 / OPTIMUS_BF16 */
  int parts;
} optimus_gradient;
int optimus_gradient_norm(const optimus_gradient* gradients, int count, float max_norm, float* norm, float* scale, float* norms, void* ws,
                          size_t ws_bytes, void* stream);
size_t optimus_gradient_norm_workspace_bytes(const optimus_gradient* gradients, int count);
int optimus_gradient_clip(const optimus_gradient* gradients, int count, const float* scale, void* stream);

/* ---- one AdamW step over many tensors (the update of Section 3.2.3, which lets the layers share one parameter-gradient buffer) ----
 * Per element, in fp32 whatever the types (root and reciprocal to a unit in the last place each, 4e-7 of the update; rounded exactly where
 * eps is below 2^-42 / sqrt(1 - beta2)):  g = grad_scale * sum over the parts of grad;  m = beta1 m + (1 - beta1) g;
 *   v = beta2 v + (1 - beta2) g^2;  w = w - (lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps) + lr * weight_decay * w).
 * A vector's partial gradients [q][q][N/q] of optimus_layer_bwd are q parts of N elements: they are added in order here.
 * Weights: fp32; or bf16 with an fp32 `master` (which is updated; param receives it rounded to nearest even); or bf16 alone, rounded
 *   up or down at random in proportion to the place between the two neighbours (to nearest, updates below half a step would be lost).
 * Moments: fp32 m, v [n]; or, with m_scale and v_scale, 8 bits: e4m3 numbers (OCP: 1 sign, 4 exponent, 3 mantissa bits), element k
 *   standing for number * 2^(scale[k / 128] - 127) (scale 255: NaN), rounded at random like the weights; a v above zero stays above zero.
 *   Zeroed memory is a valid state of either kind.  A group with a gradient whose square is not finite in fp32 turns NaN as a whole.
 * The random bits are a hash of (seed, step, index in `tensors`, element): the same call gives the same bits.
 * grad_scale, lr_on_device, step_on_device: NULL, or device memory that is read when the step runs, in place of 1, lr and step: what
 *   a captured step changes between its replays.
 * tensors: host array, read before the call returns.  Pointers need the alignment of their elements only.  The parameters may not
 *   overlap (OPTIMUS_EINVAL); nor may any other memory that is written (not checked).  n from 1 to 2^34. */
typedef struct {
  void* param;
  float* master;
  const void* grad;         /* [grad_parts][n] */
  void* m; void* v;
  uint8_t* m_scale; uint8_t* v_scale;   /* [(n + 127) / 128] each, or both NULL */
  int64_t n;
  int param_dtype, grad_dtype;          /* OPTIMUS_FP32 / OPTIMUS_BF16 */
  int grad_parts;
  float weight_decay;
} optimus_adamw_tensor;
typedef struct {
  double lr, beta1, beta2, eps;         /* 0 <= beta < 1, eps > 0 (in fp32) */
  int64_t step;                         /* 1 in the first step */
  uint64_t seed;
  const float* grad_scale; const float* lr_on_device; const int64_t* step_on_device;
} optimus_adamw_cfg;
int optimus_adamw_step(const optimus_adamw_cfg* cfg, const optimus_adamw_tensor* tensors, int count, void* stream);

/* optimus_stack_bwd that updates each layer as soon as its gradients are complete, so that all layers share ONE parameter-gradient
 * buffer (Section 3.2.3): the parameters in `params` are written.  param_grad: optimus_stack_sizes.param_grad bytes.  states: host array
 * of n_layers entries.  m, v, m_scale, v_scale: as in optimus_adamw_tensor, for optimus_stack_adamw_elements(cfg) elements: w_qkv, w_o,
 * w1, w2, b_qkv, b_o, b1, b2, ln1_g, ln1_b, ln2_g, ln2_b one after the other, each from a multiple of 128 elements on.  master: fp32
 * [12 h h], the four matrices, or NULL.  weight_decay: of the matrices; vectors have none.  Random bits: those of a list of these
 * twelve tensors and the seed adamw->seed + layer.  No two parameters, of whatever layers, may overlap (OPTIMUS_EINVAL). */
typedef struct { void* m; void* v; uint8_t* m_scale; uint8_t* v_scale; float* master; } optimus_adamw_state;
int64_t optimus_stack_adamw_elements(const optimus_layer_cfg* cfg);   /* 0 for a cfg that is refused */
int optimus_stack_bwd_adamw(const optimus_layer_cfg* cfg, int n_layers, const optimus_layer_params* params,
                            const optimus_adamw_state* states, const optimus_adamw_cfg* adamw, float weight_decay, void* param_grad,
                            const void* d_out, const optimus_stack_buffers* buf, void* d_x, void* stream);

/* ---- flop accounting (Table 1) ----
 * optimus_gemm_flops: 2*(M/q)*K*(N/q), one device's share of one product.
 * optimus_layer_flops: one device's share of a layer; what = 0 forward,
 * 1 backward without recomputation.  Attention is counted densely (non-causal)
 * so that forward equals 2*(12 b s h^2 + 2 b s^2 h)/q^2. */
int64_t optimus_gemm_flops(int64_t M, int64_t K, int64_t N, int q);
int64_t optimus_layer_flops(const optimus_layer_cfg* cfg, int what);

/* Measurement aid: a loop of matrix-core instructions only (v_mfma_f32_32x32x16_bf16 on register operands, no LDS,
 * no memory) on `workgroups` workgroups of eight wavefronts, `iters` times eight instructions per wavefront, with
 * all-zero (random_data = 0) or pseudo-random bf16 operands.  Timed by the caller; flops = workgroups * 8 * iters *
 * 8 * 32768.  out: device memory for workgroups * 512 floats (written, never read back by the library). */
int optimus_debug_mfma_rate(float* out, int workgroups, int iters, int random_data, void* stream);

/* ---- tuning hooks for benchmark sweeps (no effect on results beyond summation order) ----
 * Force the matrix-core tile variant used by bf16 products: 0 = 256x256, 1 = 256x128, 2 = 128x256,
 * 3 = 128x128, 4 = alias of 0, 5 = the any-shape kernel, 6 = 128x64, 7 = 64x64, 8 = 256x128 and 9 = 128x256 with
 * four wavefronts; -1 = automatic.  1000 + v selects, for the tiles compiled with two k-loops (0, 1, 2, 8, 9), the
 * four-slab ring instead of the 64-wide stages (identical bits); 1255 = automatic tile with that loop.
 * A tile with a ragged form (3, 6, 7) runs it where it does not divide the block.  Another tile that does not divide the block
 * gives way: to the any-shape kernel if 64x64 tiles divide the block, else to the automatic choice.  Same bits where the panel
 * split is the same; optimus_debug_last_gemm_plan tells what ran. */
void optimus_debug_set_gemm_variant(int v);
/* The same for the products optimus_layer_bwd runs side by side on two streams only: chain_v for the
 * activation-gradient chain (the four A B^T products), branch_v for the parameter-gradient branch (the four A^T B
 * products); -1 = automatic. */
void optimus_debug_set_corun_variants(int chain_v, int branch_v);
/* The tile plan a bf16 product of this shape would be launched with: out3 = {tile variant, panel split, 1 if the
 * split is walked inside the workgroups (no partial tiles in memory)}.  Host arithmetic only, nothing is enqueued and
 * no GPU is needed.  corun: 0 = the product runs alone, 1 / 2 = it is the chain / branch product of a pair that
 * optimus_layer_bwd runs side by side; have_ws: whether the caller would pass the workspace the plan asks for.
 * The panel split (the only part of a plan that changes bits) depends on the block shape alone: not on (i, j) versus
 * grid mode, not on corun.  OPTIMUS_EDTYPE when the matrix-core tiles do not take the shape (rows of A or B not
 * multiples of 8 elements, panels beyond the 2 GiB a buffer load reaches, shapes the any-shape kernel runs faster). */
int optimus_debug_plan_summa(int form, int64_t M, int64_t K, int64_t N, int q, int i, int j, int corun, int have_ws, int* out3);
/* Whether the input's and the weight's gradient of a linear layer y = x W, x [M x K], W [K x N], would share a launch in an
 * optimus_layer_bwd on one stream (host arithmetic only; -1 for invalid arguments). */
int optimus_debug_plan_pair(int64_t M, int64_t K, int64_t N, int q, int i, int j);
/* The plan of the most recent matrix-core product launched by this process: variant | (panel splits << 8) |
 * (1 << 16 if the split is emulated inside each workgroup) | (1 << 17 if 64x64 tiles ran with four stages in LDS) |
 * (1 << 18 if it was the weight gradient of a pair in one launch) | (1 << 19 if 128x64 or 128x128 tiles ran with four stages);
 * -1 before the first one.  Host state only, not synchronised between threads. */
int optimus_debug_last_gemm_plan(void);
/* The streams an optimus_layer_bwd of this size runs on when it is not captured (a captured one: two, once the library
 * has its stream): 1 or 2, or -1 for arguments that optimus_layer_bwd refuses.  Host arithmetic only. */
int optimus_debug_layer_bwd_streams(const optimus_layer_cfg* cfg, int i, int j);
/* Force how optimus_attention_selected_fwd / _bwd run: 1 = all blocks with a mask (up to 256 blocks in a sequence), 0 = lists of the queries of
 * each block, -1 = automatic.  The workspace that is asked for follows. */
void optimus_debug_set_attention_selected_form(int form);
/* Whether an optimus_attention_selected_fwd, or with backward != 0 _bwd, of this size computes all blocks with a mask (1), or lists (0);
 * -1 for arguments that these refuse.  Host arithmetic only. */
int optimus_debug_attention_selected_masked(int backward, int b, int s, int h, int n, int q, int i, int j, int causal, const optimus_selection* selection);
/* Rows of a workgroup, 64 or 128, in which an optimus_attention_biased_fwd, or with backward != 0 _bwd (table_gradient: with d_table), of
 * this size would run; -1 for arguments that these refuse.  Host arithmetic only. */
int optimus_debug_attention_biased_rows(int backward, int b, int s, int h, int n, int q, int i, int j, const optimus_attention_bias* bias,
                                        int table_gradient);

#ifdef __cplusplus
}
#endif
#endif /* OPTIMUS_H_ */
