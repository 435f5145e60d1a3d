/*
 * moevie.h -- C ABI of the GB300 (sm_103a) MoE-ViE fine-grained MoE FFN layer.
 *
 * The layer (paper "MoE-ViE", Sec. 2.1-2.2 and App. B, Algorithm 1) maps tokens
 * x[T, d] to y[T, d]:
 *
 *   s      = x . W_r                                  (Eq. 1; W_r stored [d, E])
 *   T(x)   = the k experts with the largest sigmoid(s_e) + b_e      (Eq. 7)
 *   g'_e   = sigmoid(s_e) / sum_{i in T(x)} sigmoid(s_i)            (Eqs. 4-5)
 *   y      = sum_{e in T(x)} g'_e E_e(x) + lambda * S(x)             (Eq. 6)
 *   E_e(x) = GELU(x W1[e]) W2[e],   S(x) = GELU(x Ws1) Ws2 (optional shared expert)
 *
 * GELU is the erf form u/2 (1 + erf(u / sqrt 2)).  The bias b only selects; it
 * never enters a gate.  Ties in the selection key go to the lower expert id.  A
 * token's k ids are stored in ascending order.  The expert-major row order is the
 * stable sort of the flat slots t*k + j by expert id (Algorithm 1, phase 1).
 *
 * Conventions for every entry point
 *  - Every array argument is DEVICE memory owned by the caller, unless a comment
 *    says otherwise.  The library never allocates, frees or synchronises on these
 *    calls (moevie_get_device_status excepted); all work is enqueued on `stream`
 *    (a cudaStream_t passed as void*; NULL is the legacy default stream) and runs
 *    asynchronously.
 *  - bf16 tensors are passed as void* pointing at __nv_bfloat16 data.  Matrices are
 *    row-major: x[T, d], W1[E, d, h], W2[E, h, d], Ws1[d, h_s], Ws2[h_s, d],
 *    y[T, d]; W_r[d, E] and b[E] are fp32.  Rows start 16 bytes apart: a matrix
 *    whose rows hold h values has row stride hp = h rounded up to a multiple of 8
 *    elements.  This matters only for W1 and W3 (stored [E][d][hp], expert stride
 *    d*hp) and Ws1 and Ws3 ([d][h_s rounded up to 8]) when h or h_s is not a
 *    multiple of 8 (the paper's L and H models: h = 684, 854); the pad columns are
 *    never read.  Every other matrix is dense.
 *  - Device pointers must be 16-byte aligned.  Sizes must satisfy d % 8 == 0,
 *    1 <= k <= E <= 1024 and T * k < 2^31; otherwise MOEVIE_ERR_UNSUPPORTED.
 *    T == 0 is valid and launches nothing.
 *  - Argument errors are reported synchronously, before anything is enqueued.
 *    A failed kernel launch returns MOEVIE_ERR_CUDA.  Errors found on the device
 *    (an out-of-range expert id, a pipeline wait that ran past its time limit) are
 *    written to a status block at the start of the workspace and read back with
 *    moevie_get_device_status; kernels never trap.
 *  - `ws` is caller-owned device scratch of `ws_bytes` bytes.  A workspace of
 *    moevie_workspace_size(T_max, d, E, k, h, h_s) bytes serves every entry point
 *    for any T <= T_max with the same sizes.  It must be set up once with
 *    moevie_workspace_init before first use.  Calls that share one workspace must
 *    be ordered on one stream.
 */
#ifndef MOEVIE_H
#define MOEVIE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int moevie_status;
#define MOEVIE_OK 0
#define MOEVIE_ERR_INVALID_ARG 1   /* null / misaligned pointer, negative size      */
#define MOEVIE_ERR_UNSUPPORTED 2   /* sizes outside the supported set above         */
#define MOEVIE_ERR_WORKSPACE 3     /* ws_bytes smaller than the entry point needs   */
#define MOEVIE_ERR_CUDA 4          /* a CUDA runtime call or kernel launch failed   */
#define MOEVIE_ERR_TIMEOUT 5       /* device: a bounded wait gave up (see status)   */
#define MOEVIE_ERR_DEVICE 6        /* device: a bounds check failed (see status)    */

/* Human-readable name of a status code (static string). */
const char* moevie_status_string(moevie_status s);

/* Library ABI version (major * 10000 + minor * 100 + patch). */
int moevie_version(void);

/* Bytes of workspace needed by moevie_moe_forward for up to T_max tokens (h_s = 0:
 * no shared expert).  Host-only; no device query.  Monotone in T_max. */
moevie_status moevie_workspace_size(int64_t T_max, int64_t d, int64_t E, int64_t k, int64_t h,
                                    int64_t h_s, size_t* bytes);

/* Zero the workspace's device status block (enqueued on stream).  Call once per
 * workspace before its first use; the status is sticky until cleared again. */
moevie_status moevie_workspace_init(void* ws, size_t ws_bytes, void* stream);

/* Router (Eqs. 1, 7, 4-5).  x bf16 [T, d], W_r fp32 [d, E], b fp32 [E].
 * Out: idx int32 [T, k] (ascending ids per token), gate fp32 [T, k] (same order).
 * Logits are fp32 (tensor cores); a token whose selection the fp32 logits cannot
 * certify (its k-th and (k+1)-th keys closer than their error bounds) is re-decided
 * from exact logits of the experts near its boundary -- an integer long accumulator
 * of the bf16 x fp32 products, within d 2^-64 sum|x_i w_i| of the exact dot product --
 * with the keys sigmoid(s) + b then formed in fp64, so idx equals the
 * exact-arithmetic selection. */
moevie_status moevie_route(const void* x, const float* W_r, const float* b, int64_t T, int64_t d,
                           int64_t E, int64_t k, int32_t* idx, float* gate, void* ws,
                           size_t ws_bytes, void* stream);

/* Expert-major order (App. B, Algorithm 1, phase 1: Sort, index = pos // K,
 * BinCount, CumSum).  idx int32 [T, k].  Out: counts int32 [E], offsets int32
 * [E + 1] (exclusive prefix; offsets[E] = the number of valid slots, T*k when every
 * id is valid), perm int32 [T*k] (row -> flat slot t*k + j, stable), inv int32 [T*k]
 * (flat slot -> row).  An id outside [0, E) is a device error (MOEVIE_ERR_DEVICE in
 * the status block): that slot is dropped, its inv entry is -1, it is not counted in
 * counts / offsets, and perm rows from offsets[E] to T*k are left unwritten. */
moevie_status moevie_permute(const int32_t* idx, int64_t T, int64_t k, int64_t E, int32_t* counts,
                             int32_t* offsets, int32_t* perm, int32_t* inv, void* ws,
                             size_t ws_bytes, void* stream);

/* Un-gated expert outputs in expert-major row order (App. B, Algorithm 1, Kernels
 * 1 and 2 without the routing weight): out_rows[r, :] = GELU(x[perm[r] / k] W1[e])
 * W2[e] for r in [offsets[e], offsets[e+1]).  out_rows bf16 [T*k, d]; fp32
 * accumulation, the hidden activation is rounded to bf16. */
moevie_status moevie_expert_ffn(const void* x, const int32_t* perm, const int32_t* offsets,
                                const void* W1, const void* W2, int64_t T, int64_t d, int64_t h,
                                int64_t E, int64_t k, void* out_rows, void* ws, size_t ws_bytes,
                                void* stream);

/* Shared expert (Sec. 2.2.1, Eq. 6, second term, without lambda):
 * out[t, :] = GELU(x[t] Ws1) Ws2, out bf16 [T, d]. */
moevie_status moevie_shared_expert(const void* x, const void* Ws1, const void* Ws2, int64_t T,
                                   int64_t d, int64_t h_s, void* out, void* ws, size_t ws_bytes,
                                   void* stream);

/* Gate-weighted combine (Eq. 6): y[t] = sum_j gate[t, j] out_rows[inv[t*k + j]]
 * + lambda * shared_out[t]   (shared_out bf16 [T, d] or NULL).  fp32 sums, y bf16. */
moevie_status moevie_combine(const void* out_rows, const int32_t* inv, const float* gate,
                             const void* shared_out, float lambda, int64_t T, int64_t k, int64_t d,
                             void* y, void* stream);

/* Layer description for moevie_moe_forward.  Weights are device pointers. */
typedef struct moevie_layer {
    int64_t d, E, k, h;
    int64_t h_s;            /* 0: no shared expert (Ws1, Ws2 ignored) */
    const float* W_r;       /* fp32 [d, E] */
    const float* b;         /* fp32 [E]    */
    const void* W1;         /* bf16 [E, d, h], rows h rounded up to 8 apart */
    const void* W2;         /* bf16 [E, h, d] */
    const void* Ws1;        /* bf16 [d, h_s], rows h_s rounded up to 8 apart */
    const void* Ws2;        /* bf16 [h_s, d]  */
    float lambda;           /* weight of the shared expert */
    const void* W3;         /* bf16 [E, d, h] (rows as W1) or NULL.  NULL: GELU experts GELU(x W1[e]) W2[e].
                             * Else SwiGLU experts (App. B): (SiLU(x W1[e]) * (x W3[e])) W2[e],
                             * W1 the gate and W3 the up projection. */
    const void* Ws3;        /* bf16 [d, h_s] (rows as Ws1): with W3, the shared expert's up projection
                             * (SwiGLU shared expert (SiLU(x Ws1) * (x Ws3)) Ws2); ignored
                             * without W3 or without a shared expert. */
} moevie_layer;

/* Optional routing by-products of moevie_moe_forward; any member may be NULL. */
typedef struct moevie_routing {
    int32_t* idx;       /* [T, k]   */
    float* gate;        /* [T, k]   */
    int32_t* counts;    /* [E]      */
    int32_t* offsets;   /* [E + 1]  */
    int32_t* perm;      /* [T * k]  */
    int32_t* inv;       /* [T * k]  */
} moevie_routing;

/* The whole layer forward (Eqs. 1, 4-7; Algorithm 1): router, expert-major
 * order, grouped up-projection with GELU fused into its epilogue and the token
 * gather fused into its operand load, grouped down-projection whose epilogue
 * scales each row by its gate and adds it into an fp32 accumulator of y (the
 * scatter-add of Algorithm 1), and the shared expert.  x bf16 [T, d] -> y bf16
 * [T, d].  `routing` may be NULL. */
moevie_status moevie_moe_forward(const moevie_layer* layer, const void* x, int64_t T, void* y,
                                 const moevie_routing* routing, void* ws, size_t ws_bytes,
                                 void* stream);

/* The layer from host memory to host memory, the copies overlapped with the compute.
 * Every token's output depends on that token alone (Eqs. 4-7: routing, gates and the
 * experts act per token), so the layer runs piece by piece over contiguous token ranges
 * of at most Tc = ceil(T / chunks) tokens: one piece with chunks = 1; otherwise a first
 * piece of ceil(Tc / 2) tokens, then pieces of Tc, the last one what is left (so the first
 * copy in and the last copy out, which no layer hides, are short).  A piece's rows of x
 * go from x_host to x_dev on the library's copy-in stream, moevie_moe_forward runs it on
 * `stream`, and its rows of y go from y_dev to y_host on the copy-out stream, so each
 * piece's layer overlaps the copies of its neighbours.  `stream` completes after the last
 * copy out: synchronise it (or wait on it) before reading y_host.
 * x_host, y_host: host memory [T, d] bf16 (pinned, for the copies to be asynchronous);
 * x_dev, y_dev: caller-owned device buffers [T, d] bf16, 16-byte aligned; ws:
 * moevie_workspace_size(Tc, ...) bytes at least, set up with moevie_workspace_init;
 * 1 <= chunks <= MOEVIE_HOST_MAX_CHUNKS, else MOEVIE_ERR_UNSUPPORTED.  The first call in a
 * context creates the two copy streams and their events (make it before any stream
 * capture); calls on one device share them, so calls from several host threads must
 * not overlap.  Errors as for moevie_moe_forward; device errors land in ws's status. */
#define MOEVIE_HOST_MAX_CHUNKS 16
moevie_status moevie_moe_forward_host(const moevie_layer* layer, const void* x_host, int64_t T, void* y_host,
                                      void* x_dev, void* y_dev, int64_t chunks, void* ws, size_t ws_bytes,
                                      void* stream);

/* moevie_permute without a workspace (the paper has no counterpart: this is a
 * calling convention, not part of the method).  Same inputs, outputs, ordering and
 * validation as moevie_permute, and bit-identical results.
 *
 * Who it is for: callers that cannot give the library scratch memory and cannot let
 * it allocate any -- e.g. code running inside another framework's operator that
 * only hands over its input and output buffers, or a process whose device memory
 * is all reserved up front by its own pool, where a cudaMalloc would fail or would
 * synchronise the device at a bad moment.  This entry point makes no cudaMalloc or
 * cudaFree and calls no allocating library: its scratch is one fixed array of
 * 2,179,584 bytes in the library's device image, one copy per device.
 *
 * Limits: T * k <= 1048576 (2^20) flat slots, plus the limits of moevie_permute
 * (1 <= k <= E <= 1024); larger inputs return MOEVIE_ERR_UNSUPPORTED before
 * anything is enqueued.
 *
 * Set-up: the first call on a device (with that device current) looks up the
 * array's device address, which may load the library's device code; make that
 * first call before any stream capture.  Later calls reuse the address as long as
 * the device's context is the same; after cudaDeviceReset the next call looks it up
 * again in the new context (again, before any capture).
 *
 * Concurrency: all calls on one device share the one array.  Two calls whose GPU
 * work overlaps (different streams, or several host threads without ordering) race
 * on it and give undefined results; order them on one stream or with events.
 *
 * Device-side errors: each call clears the array's status block; an expert id
 * outside [0, E) drops its slot (inv = -1, not counted in counts / offsets) and is
 * recorded there, but no entry point reads that status back -- check inv for -1
 * where ids are untrusted. */
moevie_status moevie_permute_static(const int32_t* idx, int64_t T, int64_t k, int64_t E,
                                    int32_t* counts, int32_t* offsets, int32_t* perm,
                                    int32_t* inv, void* stream);

/* Number of kernels this library has launched since it was loaded (all
 * threads, all devices).  Host-only. */
uint64_t moevie_launch_count(void);

/* Loss-free balancing (Sec. 2.2.2): update the selection bias b[E] (fp32, device,
 * in place) from one step's expert loads counts[E] (int32, device; e.g. the counts
 * moevie_permute / moevie_moe_forward return), E <= 1024.  With mu the mean load and
 * sigma the population standard deviation of the loads over the E experts:
 *   rule 0, z-score (Eq. 9):  b_e <- b_e - alpha (t_e - mu) / sigma
 *                              (all loads equal, sigma = 0: b unchanged)
 *   rule 1, sign (Eq. 8):     b_e <- b_e - alpha sign(t_e - mu), sign(0) = 0.
 * Arithmetic in fp64, each new b_e rounded to fp32.  One tiny kernel on `stream`;
 * `ws` (>= 256 bytes, the workspace of the other entry points will do) receives the
 * device status: a negative load leaves b unchanged and records MOEVIE_ERR_DEVICE.
 * Argument errors (E outside [1, 1024], rule not 0 or 1, null or misaligned
 * pointers) return before anything is enqueued. */
moevie_status moevie_update_bias(const int32_t* counts, int64_t E, float alpha, int rule, float* b,
                                 void* ws, size_t ws_bytes, void* stream);

/* Launch plan of moevie_moe_forward for these sizes, GELU or SwiGLU experts alike
 * (host-only, no GPU work; the paper has no counterpart -- it describes how this
 * library schedules Eq. 6's shared term).  Returns the number S of always-on groups of
 * width h that carry the shared expert inside the routed up- and down-projection
 * launches (its hidden units in S = h_s / h chunks, every token with gate lambda), or 0
 * when it runs as its own GEMMs (no shared expert, h not dividing h_s, several chunks
 * of a width h that is not a multiple of 8, or a band-ordered down-projection).
 * Invalid sizes return 0. */
int64_t moevie_shared_groups(int64_t T, int64_t d, int64_t E, int64_t k, int64_t h, int64_t h_s);

/* ---------------------------------------------------------------- training path
 *
 * Backward pass of the layer, GELU or SwiGLU experts, with or without a shared expert (App. B:
 * the paper trains with grouped GEMMs and applies the activation as its own step).  Given
 * the forward's selection idx (held fixed: top-k is piecewise constant in the logits, so
 * it has no gradient) and the output gradient dy, it returns the gradients of
 * L = sum_t dy_t . y_t:
 *   through each selected expert e of token t, with gate g (Eqs. 4-5) and the hidden
 *   activation a (GELU(u), u = x_t W1[e]; SwiGLU: SiLU(u) v, v = x_t W3[e]):
 *     dW2[e] += a^T (g dy_t),   da = g dy_t W2[e]^T,
 *     GELU:   du = da GELU'(u);   SwiGLU: du = da v SiLU'(u), dv = da SiLU(u),
 *     dW1[e] += x_t^T du,  dW3[e] += x_t^T dv,  dx_t += du W1[e]^T + dv W3[e]^T;
 *   through the gates (Eqs. 4-5), with sigma_j = sigmoid(s_{e_j}), S = sum_j sigma_j and
 *   dg_j = dy_t . E_{e_j}(x_t):
 *     ds_{e_j} = sigma_j (1 - sigma_j) (dg_j - sum_l g_l dg_l) / S,
 *     dW_r[:, e_j] += x_t ds_{e_j},   dx_t += ds_{e_j} W_r[:, e_j];
 *   through the shared expert (Eq. 6, second term; h_s > 0), every token with the
 *   constant weight lambda, the expert's rules with g = lambda and Ws1, Ws2, Ws3 in place
 *   of W1[e], W2[e], W3[e] (lambda gets no gradient).
 * The bias b gets no gradient (it only selects; moevie_update_bias moves it).
 *
 * Inputs: the layer (W_r, W1, W2, for SwiGLU experts W3, and the shared expert's Ws1, Ws2,
 * Ws3 and lambda when h_s > 0, as for moevie_moe_forward), x bf16 [T, d], dy bf16 [T, d],
 * idx int32 [T, k] (the forward's selection, e.g. moevie_routing.idx; ids in [0, E)).
 * Outputs, fp32, all overwritten: dx [T, d], dW_r [d, E], dW1 [E, d, h] with rows h
 * rounded up to 8 apart (as W1; the pad columns hold zeros), dW2 [E, h, d], for SwiGLU
 * experts dW3 laid out as dW1 (NULL otherwise); with a shared expert dWs1 [d, h_s] with
 * rows h_s rounded up to 8 apart (as Ws1), dWs2 [h_s, d] and, for SwiGLU, dWs3 laid out as
 * dWs1 (all three NULL without one).  The gates are recomputed from x and W_r in fp32.
 * Arithmetic: bf16 GEMM operands with fp32 accumulation (the recomputed pre-activations,
 * activations, their gradients, g dy and ds are rounded to bf16 as GEMM operands); dx,
 * and every weight gradient summed over more than 4096 rows (an expert's rows padded to
 * 64; all T tokens for dW_r and the shared expert's), take fp32 reductions over chunks of
 * rows, so their last bits depend on the order in which the GEMM's work items finish;
 * the other weight gradients are written once.  Sizes: k <= 32, d and h <=
 * 65535 (h_s too), plus the limits of moevie_moe_forward.  `ws`:
 * moevie_backward_workspace_size(T_max, d, E, k, h, h_s, swiglu) bytes (swiglu nonzero for
 * SwiGLU experts), set up with moevie_workspace_init; device errors land in its status
 * block.  T == 0 launches nothing: the weights' gradients, zeros then, are not written (the Python
 * binding clears them). */
moevie_status moevie_backward_workspace_size(int64_t T_max, int64_t d, int64_t E, int64_t k, int64_t h,
                                             int64_t h_s, int swiglu, size_t* bytes);
moevie_status moevie_moe_backward(const moevie_layer* layer, const void* x, const void* dy, int64_t T,
                                  const int32_t* idx, float* dx, float* dW_r, float* dW1, float* dW2,
                                  float* dW3, float* dWs1, float* dWs2, float* dWs3, void* ws,
                                  size_t ws_bytes, void* stream);

/* The whole layer for a few tokens (1 <= T <= MOEVIE_FEW_MAX_TOKENS): the function of
 * moevie_moe_forward, for callers that run the layer token by token or on small batches, where
 * its time is that of reading the router and the selected experts once.  GELU or SwiGLU
 * experts, with or without a shared expert, the layer's weights as for moevie_moe_forward.
 * idx [T, k] (ascending ids per token) and gate [T, k] are optional outputs (NULL: not
 * returned).  The selection is that of exact arithmetic up to the rounding of a 64-bit sum
 * (products of bf16 and fp32 are exact in 64 bits; keys in 64 bits; ties to the lowest id; a
 * key that is NaN comes after every number).  Hidden activations keep more than bf16's bits, so
 * y is as precise as 32-bit arithmetic rounded once to bf16.  A token's ids and y do not depend
 * on the others' values but for the order of sums: how those are split goes by the number of
 * tokens and by what they select.  The same call gives the same bits.
 * Sizes: those of moevie_moe_forward, k <= 32 and d, h, h_s <= 65535; T == 0 launches nothing.
 * ws: moevie_few_workspace_size(T_max, ...) bytes, set up with moevie_workspace_init.  After
 * MOEVIE_ERR_TIMEOUT in its status set it up again: calls may leave their outputs as they were
 * until then. */
#define MOEVIE_FEW_MAX_TOKENS 64
moevie_status moevie_few_workspace_size(int64_t T_max, int64_t d, int64_t E, int64_t k, int64_t h,
                                        int64_t h_s, size_t* bytes);
moevie_status moevie_moe_few(const moevie_layer* layer, const void* x, int64_t T, void* y, int32_t* idx,
                             float* gate, void* ws, size_t ws_bytes, void* stream);

/* Newton-Schulz orthogonalisation of a stack of N matrices U [rows, cols] (the update of the
 * Muon optimiser).  With X0 = U / |U|_F (X0 = 0 for U = 0) and, per step, coefficients
 * (a, b, c) = coef[3 i .. 3 i + 2]:
 *     A = X X^T,   X <- a X + (b A + c A^2) X,
 * which moves every singular value s of X0 to the odd quintic a s + b s^3 + c s^5 of itself
 * and keeps the singular vectors.  (For rows > cols it is formed from X^T X; the result is
 * the same.)  Each matrix of the stack is treated by itself; one that holds an infinity or a
 * NaN gives NaN and leaves the others alone.
 *   U: fp32 (u_bf16 = 0) or bf16 (u_bf16 = 1), row stride ld_u >= cols and matrix stride
 *   stride_u elements; any alignment of rows (16-byte aligned rows are read faster).
 *   O: bf16, row stride ld_o >= cols, matrix stride stride_o.  O does not overlap U.
 * Arithmetic: fp16 tensor-core operands (11 bits), fp32 accumulation, X carried from step to
 * step in 22 bits (where |a| <= 3.5 in the last two steps, the last one takes 11).  Matrices of
 * which one side is at most 128: 22-bit operands but for X X^T.  Of which one side is at most 32,
 * and few matrices (some tens) of which one is at most 64: fp32 throughout.  Each step rounds anew
 * and multiplies what was there by the slope of its polynomial, so the error depends on
 * coefficients and matrix.  In 2-norm, before the rounding to bf16, against the formula's result:
 *   - coefficients (3.4445, -4.7750, 2.0315), five steps, matrices whose singular vectors are
 *     spread over their entries (as gradients' are), of full or low rank: 1e-3 to 2e-3, and
 *     below 1e-3 where one side is at most 128;
 *   - the same, but matrices of a few large entries, whose roundings do not average: up to
 *     2e-2 for a singular value that the steps' slopes (up to 4) magnify;
 *   - directions that are null in U hold X's rounding (2^-22; 2^-24 in fp32), which every step
 *     multiplies by a: matrices of low rank take about eight such steps, and after twelve
 *     (fourteen) what was rounding counts as much as what was U;
 *   - coefficients whose polynomials are steep where singular values arrive lose as much as
 *     their slopes say: first steps such as (8.29, -23.6, 17.3), slope 24 at 1, leave several
 *     percent on matrices of rank 1.
 * coef: HOST memory, steps x 3 floats, finite; 1 <= steps <= 32.  For matrices whose smaller
 * side is above 32, all steps from singular values in [0, 1] on must keep those of X (but the
 * last), of A and of b A + c A^2 at 60 or below, as fp16 holds them (the usual quintics stay
 * below 10), else MOEVIE_ERR_UNSUPPORTED.  Sizes: rows and cols in [1, 8192],
 * 0 <= N <= 65535, matrix strides below 2^38, else MOEVIE_ERR_UNSUPPORTED; N == 0 launches
 * nothing.  ws:
 * moevie_orthogonalize_workspace_size bytes, set up with moevie_workspace_init. */
moevie_status moevie_orthogonalize_workspace_size(int64_t N, int64_t rows, int64_t cols, size_t* bytes);
moevie_status moevie_orthogonalize(const void* U, int u_bf16, int64_t ld_u, int64_t stride_u, int64_t N,
                                   int64_t rows, int64_t cols, const float* coef, int steps, void* O,
                                   int64_t ld_o, int64_t stride_o, void* ws, size_t ws_bytes, void* stream);

/* One Muon step on a stack of N weight matrices W [rows, cols] (e.g. W1 of all experts with
 * dW1 of moevie_moe_backward), all in place:
 *     M <- momentum M + G,     U = G + momentum M (nesterov) or M,
 *     O = the Newton-Schulz orthogonalisation of U (as moevie_orthogonalize),
 *     W <- (1 - lr weight_decay) W - lr scale O,      W_bf16 = bf16(W).
 * W, M, G: fp32, W_bf16: bf16 or NULL; all four have row stride ld (a multiple of 8,
 * >= cols) and matrix stride `stride` (a multiple of 8, >= rows ld), 16-byte aligned: the
 * layout of W1 and of dW1.  Pad columns are neither read nor written.  A zero U (an expert
 * that got no token, without momentum) only decays its weights.  Workspace, coef, steps and
 * sizes as for moevie_orthogonalize.  Where a status other than MOEVIE_OK is returned for these
 * reasons, M and W are as they were; after a timeout on the device (moevie_get_device_status)
 * they are undefined. */
moevie_status moevie_muon_update(float* W, void* W_bf16, float* M, const float* G, int64_t N, int64_t rows,
                                 int64_t cols, int64_t ld, int64_t stride, float lr, float momentum,
                                 int nesterov, float weight_decay, float scale, const float* coef, int steps,
                                 void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------ a residual block's steps around the layer
 *
 * Between the layer f = y(u) and the next one a block norms, gates and adds (Sec. 2.1: the layer
 * takes the place of the MLP in a pre-norm block):
 *     r1 = residual_scale r + gate * N_post(f),      u = N_pre(r1).
 * N is an RMS norm, N(x) = x / sqrt(mean(x^2) + eps) w + b, or a layer norm, which first subtracts
 * the row's mean.  The gate has d values for every run of tokens: one run (LayerScale), or one for
 * each image or clip (a gate that a condition modulates). */
#define MOEVIE_NORM_NONE 0
#define MOEVIE_NORM_RMS 1
#define MOEVIE_NORM_LAYER 2

typedef struct moevie_norms {
    int64_t d;              /* d % 8 == 0, d <= 8192 */
    int32_t pre, post;      /* MOEVIE_NORM_*: N_pre, N_post */
    const float* w_pre;     /* fp32 [d] each; NULL: 1 for w, 0 for b */
    const float* b_pre;
    const float* w_post;
    const float* b_post;
    const float* gate;      /* fp32 [G, d] or NULL: 1 */
    const int32_t* seg;     /* int32 [G + 1], device: run g is rows [seg[g], seg[g + 1]); NULL: one run
                             * of all rows (G = 1).  Ascending within [0, T] (else MOEVIE_ERR_DEVICE in the
                             * status); runs may be empty.  Every warp reads them for itself: they must not
                             * change while a call runs.  Rows in front of seg[0] and from seg[G] on are
                             * padding: never read, and left as they were in every output (moevie_moe_forward
                             * and moevie_moe_backward read all rows: clear them in what these get, with
                             * moevie_clear_padding, once where the buffer is kept). */
    int64_t G;
    float residual_scale;   /* finite */
    float eps;              /* > 0, finite */
} moevie_norms;

/* Rows [T, d] of one of three types; an MOEVIE_Q8 is an 8-bit checkpoint (moevie_checkpoint_store). */
#define MOEVIE_BF16 0
#define MOEVIE_F32 1
#define MOEVIE_Q8 2
typedef struct moevie_rows {
    const void* data;       /* bf16, fp32, or int8 codes */
    const float* scale;     /* MOEVIE_Q8: fp32 [T, ceil(d / 128)]; ignored otherwise */
    int32_t type;
} moevie_rows;

/* 8-bit checkpoint of activations x [T, d] (bf16, or fp32 where x_f32): of each row every block of 128
 * columns (the last one what is left) keeps amax = max |x| as scale = amax / 127 in fp32 and its values as
 * int8 codes, the whole number nearest to 127 x / amax (an even one between two, decided exactly).  A
 * value is code * scale, off by at most amax / 254 and a rounding (where amax is the largest finite float, whose
 * scale times 127 would not be finite, scale is the next float below).  A block whose values all lie below
 * 2^-110 is kept as zeros; one that holds an infinity or a NaN comes back as NaN.  d % 8 == 0;
 * codes: int8 [T, d], 16-byte aligned; scale: fp32 [T, ceil(d / 128)].  moevie_checkpoint_load writes the
 * values as bf16 or fp32.  T == 0 launches nothing. */
moevie_status moevie_checkpoint_store(const void* x, int x_f32, int64_t T, int64_t d, int8_t* codes, float* scale,
                                      void* stream);
moevie_status moevie_checkpoint_load(const int8_t* codes, const float* scale, int64_t T, int64_t d, void* x,
                                     int x_f32, void* stream);

/* The step forward.  r: the residual stream (bf16 or fp32); f: the layer's output, bf16.  Outputs: r_out,
 * of r's type (may be r itself), u bf16 [T, d], and where not NULL the statistics that the backward
 * takes, stats_pre and stats_post fp32 [T, 2]: mean (0 for an RMS norm) and 1 / sqrt(... + eps) of each
 * row.  All arithmetic is fp32, u is normed from r1 before its rounding to bf16, and each output is
 * rounded once.
 *   f == NULL: the stream's first norm, u = N_pre(r); r may then be an MOEVIE_Q8 (the layer's input formed
 *   again for its backward); r_out is not written.
 *   pre == MOEVIE_NORM_NONE: no u (NULL): the stream's last step.  post == MOEVIE_NORM_NONE: N_post(f) = f.
 *   save_r, save_f (with their scales; NULL: not wanted): 8-bit checkpoints of r and f, what
 *   moevie_checkpoint_store gives for them, written while they are read for the last time.
 * ws: moevie_residual_norm_workspace_size(T_max, d, G) bytes, set up with moevie_workspace_init.
 * T < 2^31, G <= 2^20; T == 0 launches nothing. */
moevie_status moevie_residual_norm_workspace_size(int64_t T_max, int64_t d, int64_t G, size_t* bytes);
moevie_status moevie_residual_norm(const moevie_norms* n, const moevie_rows* r, const void* f, int64_t T, void* r_out,
                                   void* u, float* stats_pre, float* stats_post, int8_t* save_r, float* save_r_scale,
                                   int8_t* save_f, float* save_f_scale, void* ws, size_t ws_bytes, void* stream);

/* Its backward: from dr1 (the gradient of r1 but for what comes through u; of the residual stream's type,
 * fp32 where res_f32, else bf16; NULL: zero) and du (the gradient of u, fp32 where du_f32, e.g. dx of
 * moevie_moe_backward, else bf16; NULL with pre == MOEVIE_NORM_NONE):
 *     dR = dr1 + the gradient that N_pre passes on,   dr = residual_scale dR,
 *     df = the gradient that N_post passes on from gate * dR,
 * and the gradients of w_pre, b_pre, w_post, b_post [d] and gate [G, d], fp32 (each NULL: not wanted).
 * r1 and f are the forward's rows, or their checkpoints (MOEVIE_Q8); r1 whole is of the residual stream's
 * type, f whole is bf16.  stats_pre, stats_post: as the forward wrote them.  dr is of dr1's type and may be
 * dr1 itself; df is bf16, dy of moevie_moe_backward.
 *   df == NULL: the forward ran without f; f, stats_post and the gradients of w_post, b_post and gate
 *   are then NULL, and dr = dR.  f may be NULL where post == MOEVIE_NORM_NONE and dgate is not wanted.
 * Sums over rows are fp32, in an order that goes by T, d and the runs alone: the same call gives
 * the same bits.  Rows outside every run do not enter them; a run without rows gets a zero dgate.
 * T == 0 launches nothing: the gradients, zeros then, are not written (the Python binding clears them).  ws
 * as for moevie_residual_norm. */
moevie_status moevie_residual_norm_backward(const moevie_norms* n, const void* dr1, int res_f32, const void* du,
                                            int du_f32, const moevie_rows* r1, const moevie_rows* f,
                                            const float* stats_pre, const float* stats_post, int64_t T, void* dr,
                                            void* df, float* dw_pre, float* db_pre, float* dw_post, float* db_post,
                                            float* dgate, void* ws, size_t ws_bytes, void* stream);

/* Zeros in rows of padding, which the calls above and moevie_balance_loss leave as they were: of up to 16 buffers of
 * T rows, row_bytes each (a multiple of 4; rows 4-byte aligned, one behind the other), the rows in front of seg[0]
 * and from seg[G] on (seg as in moevie_norms; an end outside [0, T] counts as its nearest end).  T < 2^31, G <= 2^20;
 * T == 0 launches nothing. */
typedef struct moevie_buffer {
    void* rows;
    int64_t row_bytes;
} moevie_buffer;
moevie_status moevie_clear_padding(const moevie_buffer* buffers, int n_buffers, int64_t T, const int32_t* seg, int64_t G,
                                   void* stream);

/* ------------------------------------------------ balance loss
 *
 * The auxiliary loss that the loss-free bias (moevie_update_bias) stands in for, for training with
 * both or with it alone.  s fp32 [T, E] (rows ld_s apart): the router's logits; idx int32 [T, k]: the
 * selection (e.g. moevie_routing.idx).  Over every run b of T_b tokens (seg, G as in moevie_norms; NULL: one
 * run of all tokens; one run for each sequence balances each by itself), with n_be the ids of its tokens
 * that are e and p_te = softmax(s_t)_e (MOEVIE_SCORE_SOFTMAX) or sigmoid(s_te) / sum_j sigmoid(s_tj)
 * (MOEVIE_SCORE_SIGMOID, the scores behind Eqs. 4-5):
 *     loss = coef sum_b (T_b / T) sum_e (E n_be / (k T_b)) (mean over the run of p_te),
 * T the tokens of all runs: coef for loads that are even.  The counts carry no gradient.  Outputs: loss fp32
 * [1], counts int32 [G, E], and ds fp32 [T, E] (rows ld_ds apart; NULL: not wanted; may be s itself with
 * ld_ds = ld_s), the gradient of loss, which moevie_moe_backward_balanced takes.  Rows outside every run are
 * neither read nor written.  A logit of minus infinity has no probability; a row of nothing else adds
 * nothing, its ds is zero; a NaN, or plus infinity under a softmax, gives NaN in its row and in loss.  An id
 * outside [0, E) is not counted, and is MOEVIE_ERR_DEVICE in the status, as are runs that do not ascend
 * within [0, T].  fp32 arithmetic; the same call gives the same bits.  1 <= k <= E <= 1024, T k < 2^31 and
 * G <= 2^20, else MOEVIE_ERR_UNSUPPORTED.  T == 0: loss and counts are zeros.  ws:
 * moevie_balance_workspace_size(T_max, E, k, G_max) bytes, set up with moevie_workspace_init. */
#define MOEVIE_SCORE_SOFTMAX 0
#define MOEVIE_SCORE_SIGMOID 1
moevie_status moevie_balance_workspace_size(int64_t T_max, int64_t E, int64_t k, int64_t G, size_t* bytes);
moevie_status moevie_balance_loss(const float* s, int64_t ld_s, const int32_t* idx, int64_t T, int64_t E, int64_t k,
                                  const int32_t* seg, int64_t G, int score, float coef, float* loss, int32_t* counts,
                                  float* ds, int64_t ld_ds, void* ws, size_t ws_bytes, void* stream);

/* The router's logits s = x W_r (Eq. 1) for moevie_balance_loss: x bf16 [T, d], W_r fp32 [d, E], s fp32 [T, E]
 * with rows E rounded up to a multiple of 32 apart (16-byte aligned; the columns between hold zeros).  On the
 * tensor cores with fp32 accumulation, W_r as the sum of two bf16 pieces (off by at most 2^-16 of it): the
 * logits that moevie_route starts from.  ws: moevie_workspace_size(T_max, d, E, 1, 0, 0) bytes or those of the
 * whole layer. */
moevie_status moevie_router_logits(const void* x, const float* W_r, int64_t T, int64_t d, int64_t E, float* s, void* ws,
                                   size_t ws_bytes, void* stream);

/* moevie_moe_backward with a gradient of the logits besides the one through the gates: ds fp32 [T, E], rows
 * ld_ds >= E apart, every row of it read (e.g. that of moevie_balance_loss):
 *     dx += ds W_r^T,   dW_r += x^T ds,
 * ds and W_r rounded to bf16 as GEMM operands, fp32 accumulation.  Everything else, the workspace included,
 * as for moevie_moe_backward. */
moevie_status moevie_moe_backward_balanced(const moevie_layer* layer, const void* x, const void* dy, int64_t T,
                                           const int32_t* idx, const float* ds, int64_t ld_ds, float* dx, float* dW_r,
                                           float* dW1, float* dW2, float* dW3, float* dWs1, float* dWs2, float* dWs3,
                                           void* ws, size_t ws_bytes, void* stream);

/* Synchronise `stream`, then read the workspace's device status into *out
 * (MOEVIE_OK when no device-side error was recorded).  `detail` (host, may be
 * NULL) receives 4 ints: code, site, and two values describing the failure. */
moevie_status moevie_get_device_status(const void* ws, void* stream, moevie_status* out,
                                       int32_t* detail);

#ifdef __cplusplus
}
#endif

#endif /* MOEVIE_H */
