/*
 * moe_hotpath.h - C ABI of the MI355X (gfx950) SparseMoE expert hot path.
 *
 * The calls follow the five stages of the paper's FastSparseMoE block
 * (Section 3.1, Algorithm 1) for ONE GPU holding the local experts
 * [e_begin, e_begin + e_count) of an E-expert layer (e_count == E when there is
 * no expert parallelism):
 *
 *   moe_route                 Stage 1   Softmax + TopK of the router logits
 *   moe_permute               Stages 2-3 and the gather that opens Stage 4
 *   moe_grouped_gemm_fwd      Stage 4   three grouped products around Silu(gate)*up
 *   moe_unpermute_combine     Stage 5   ExpertOutputReductionForward
 *   moe_unpermute_combine_bwd Stage 5   ExpertOutputReductionBackward
 *   moe_grouped_gemm_bwd      derivative of Stage 4 (dgrad + wgrad; left to autograd in the paper)
 *   moe_permute_bwd           derivative of the Stage-4 gather
 *
 * Fused variants of the same stages: moe_grouped_gemm_fwd_gather / _bwd_gather (the products read the routed
 * rows of x themselves, no permuted copy), and moe_permute_gate, moe_grouped_gemm_fwd_folded,
 * moe_unpermute_sum, moe_grouped_gemm_bwd_folded (gate weights folded into the expert MLP: Stage 5 becomes a
 * plain sum and needs no backward pass of its own).  Stage 1's Router layer and the derivatives of Stage 1:
 * moe_router_fwd, moe_route_bwd, moe_router_bwd.
 *
 * In front of the layer and behind it: moe_add_rms_norm (_8bit, _bwd), the residual's addition and the norm; moe_head_ce_fwd / _bwd and
 * moe_head_distill_fwd / _bwd, the vocabulary head's losses without its logits.
 * moe_head_score_fwd / _bwd, log probabilities of given tokens with entropies and the likeliest alternatives.
 * In front of attention: moe_qk_norm_rope (_bwd), norms of queries and keys with the rotation.  Behind a backward pass: moe_grad_norm, moe_grad_clip.
 *
 * Conventions, valid for every function below
 * -------------------------------------------
 * - Every pointer except `stream` is a DEVICE pointer to memory the caller owns,
 *   16-byte aligned, dense and row-major.  The library allocates nothing, frees
 *   nothing and never synchronises: all work is enqueued on `stream`
 *   (a hipStream_t passed as void*; NULL is the default stream).  Results are
 *   ready when the stream reaches them.  The only state the library keeps between
 *   calls is, per device, what it has looked up or configured once there (number of
 *   compute units, the kernels' LDS limit) and the benchmark facility at the end
 *   of this file.
 * - Outputs are overwritten, never accumulated into (weight gradients of
 *   experts without rows are written as zeros).
 * - Group sizes stay on the device (`expert_offsets`); no call reads them back.
 *   R_cap is the row capacity of the grouped buffers (T*k is always enough);
 *   rows at or beyond expert_offsets[e_count] are neither read nor written.
 * - moe_bf16 is a raw bfloat16 bit pattern.  Products accumulate in fp32; bf16
 *   results are rounded to nearest-even once, from the fp32 value.
 * - Return value: MOE_OK, or a negative MOE_ERR_* code.  Argument checks run on
 *   the host before anything is enqueued; a failed call enqueues nothing.
 *   Not checked (preconditions): logits finite; topk_idx values in [0, E) and
 *   distinct within a token; expert_offsets non-decreasing, starting at 0 and
 *   ending at most at R_cap.
 * - A row of g, u, h and yp is a function of its token, its expert's weights and its gate weight alone, bit for bit:
 *   not of the expert's number, of e_begin and e_count, nor of the other rows of the call.
 * - Calls on different streams may overlap as long as their buffers (including
 *   workspaces) do not.
 */
#ifndef MOE_HOTPATH_H
#define MOE_HOTPATH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef uint16_t moe_bf16;

enum {
  MOE_OK = 0,
  MOE_ERR_INVALID = -1,   /* null/misaligned pointer, non-positive or unsupported size */
  MOE_ERR_WORKSPACE = -2, /* workspace smaller than the matching *_workspace_bytes() */
  MOE_ERR_LAUNCH = -3     /* the HIP runtime refused a launch (hipGetLastError) */
};

/* Size limits (checked; MOE_ERR_INVALID beyond them):
 *   1 <= k <= E <= 512, e_count <= 512, d % 8 == 0, f % 8 == 0 for the row
 *   movers; the grouped products additionally need d % 64 == 0 and f % 64 == 0. */
#define MOE_MAX_EXPERTS 512

/* Library identification string (static storage). */
const char* moe_version(void);

/* Workspace sizes in bytes (host computation only). */
size_t moe_permute_workspace_bytes(int T, int k, int e_count);
size_t moe_grouped_gemm_bwd_workspace_bytes(int R_cap, int f);
/* Upper bound that is enough for any call on a layer of this shape with R_cap <= T*k and at most E local
 * experts: the largest of moe_permute_workspace_bytes(T, k, E), moe_grouped_gemm_bwd_workspace_bytes(T*k, f),
 * moe_grouped_gemm_bwd_folded_workspace_bytes(T*k, f) and moe_router_bwd_workspace_bytes(T, d, E).
 * 0 for a non-positive size or when T*k does not fit an int. */
size_t moe_workspace_bytes(int T, int E, int k, int d, int f);

/*
 * Stage 1 (Algorithm 1: probs = Softmax(logits); weights, indices = TopK(probs)).
 *   logits   [T, E] fp32
 *   topk_idx [T, k] int32  slot i holds the expert with the i-th largest logit;
 *                          equal logits go to the lower expert id (-0.0 == +0.0)
 *   topk_w   [T, k] fp32   softmax probability of each chosen expert; divided by
 *                          the sum over the k chosen ones when renormalize != 0
 *                          (renormalize == 0 is Algorithm 1 as printed)
 */
int moe_route(const float* logits, int T, int E, int k, int renormalize,
              int32_t* topk_idx, float* topk_w, void* stream);

/*
 * Stages 2-3 (token counting, index generation) and mlp_in = input[input_indices].
 * The (token, slot) pairs whose expert is local are grouped by expert; inside an
 * expert they keep token order (a stable counting sort, done without atomics, so
 * the result is unique and reproducible).
 *   x              [T, d] bf16
 *   topk_idx       [T, k] int32, values in [0, E_total)
 *   expert_offsets [e_count+1] int32  out: exclusive prefix sum of the per-expert
 *                                     row counts (Algorithm 1: cum_token_counts)
 *   row_token      [T*k] int32        out: token of each grouped row (input_indices);
 *                                     entries at or beyond R are left untouched
 *   slot_row       [T, k] int32       out: grouped row of pair (t, i), -1 when its
 *                                     expert is not local (dense form of
 *                                     output_indices / selected_expert_indices)
 *   xp             [T*k, d] bf16      out: xp[r] = x[row_token[r]] for r < R.
 *                                     May be NULL: then only the index arrays are
 *                                     produced and x is not read (for the *_gather
 *                                     products below, which read x through row_token)
 *   ws             at least moe_permute_workspace_bytes(T, k, e_count)
 */
int moe_permute(const moe_bf16* x, const int32_t* topk_idx,
                int T, int d, int E_total, int k, int e_begin, int e_count,
                int32_t* expert_offsets, int32_t* row_token, int32_t* slot_row,
                moe_bf16* xp, void* ws, size_t ws_bytes, void* stream);

/*
 * moe_permute without a workspace argument, for callers that cannot allocate device memory at all
 * (code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the histogram
 * table lives in a device array inside the library image, moe_permute_static_ws_capacity() bytes
 * (1 MiB) on every GPU the library is used on, held until the process ends.  Arguments and results are
 * exactly those of moe_permute.  A shape whose table does not fit
 * (moe_permute_workspace_bytes(T, k, e_count) > capacity) is refused with MOE_ERR_WORKSPACE and nothing
 * is enqueued.  The call allocates nothing and frees nothing.  Its first call on a device looks the
 * array's address up (no allocation, but do it before a graph capture begins).  All calls on one GPU
 * share that GPU's array: two such calls that overlap in time on one GPU (different streams) race;
 * calls on one stream, or ordered by events, are fine.
 */
size_t moe_permute_static_ws_capacity(void);
int moe_permute_static_ws(const moe_bf16* x, const int32_t* topk_idx,
                          int T, int d, int E_total, int k, int e_begin, int e_count,
                          int32_t* expert_offsets, int32_t* row_token, int32_t* slot_row,
                          moe_bf16* xp, void* stream);

/* dx[t] = sum over the local slots i of token t of dxp[slot_row[t, i]] (fp32 sum
 * in slot order, rounded once); a token without local slot gets zeros.
 *   dxp [R_cap, d] bf16, slot_row [T, k] int32, dx [T, d] bf16 */
int moe_permute_bwd(const moe_bf16* dxp, const int32_t* slot_row, int T, int k, int d,
                    moe_bf16* dx, void* stream);

/*
 * Stage 4 (Algorithm 1: gate_out, up_out = Grouped_mm(mlp_in, gate/up_weight);
 * mul_out = Silu(gate_out) * up_out; mlp_out = Grouped_mm(mul_out, down_weight)).
 * For each local expert e with rows r in [expert_offsets[e], expert_offsets[e+1]):
 *   g[r] = xp[r] . Wg[e]^T,  u[r] = xp[r] . Wu[e]^T,  h[r] = silu(g[r]) * u[r],
 *   yp[r] = h[r] . Wd[e]^T.
 *   xp [R_cap, d]; Wg, Wu [E, f, d]; Wd [E, d, f]  (each expert's [out, in]
 *   weight, stacked over the E local experts); g, u, h [R_cap, f] are saved for
 *   the backward call; yp [R_cap, d].  All bf16; h is formed from the fp32
 *   accumulators, before g and u are rounded.
 */
int moe_grouped_gemm_fwd(const moe_bf16* xp, const int32_t* expert_offsets,
                         const moe_bf16* Wg, const moe_bf16* Wu, const moe_bf16* Wd,
                         int E, int R_cap, int d, int f,
                         moe_bf16* g, moe_bf16* u, moe_bf16* h, moe_bf16* yp, void* stream);

/*
 * Stage 4 with mlp_in = input[input_indices] folded into the first product: the
 * same results as moe_grouped_gemm_fwd on xp[r] = x[row_token[r]], but the gate/up
 * product loads the rows of x itself, so xp need not exist.
 *   x [T, d] bf16, T*d*2 bytes at most 4 GiB (row offsets are 32-bit);
 *   row_token [R_cap] int32 as written by moe_permute; everything else as above.
 */
int moe_grouped_gemm_fwd_gather(const moe_bf16* x, int T, const int32_t* row_token,
                                const int32_t* expert_offsets,
                                const moe_bf16* Wg, const moe_bf16* Wu, const moe_bf16* Wd,
                                int E, int R_cap, int d, int f,
                                moe_bf16* g, moe_bf16* u, moe_bf16* h, moe_bf16* yp, void* stream);

/*
 * Derivative of Stage 4.  With s = sigmoid(g):
 *   dh = dyp . Wd[e];  dg = dh * u * s * (1 + g * (1 - s));  du = dh * g * s;
 *   dxp = dg . Wg[e] + du . Wu[e];
 *   dWd[e] = dyp^T . h;  dWg[e] = dg^T . xp;  dWu[e] = du^T . xp   (zeros if e has no rows).
 *   dyp, xp, dxp [R_cap, d]; g, u, h [R_cap, f]; dWg, dWu [E, f, d]; dWd [E, d, f]; all bf16.
 *   ws at least moe_grouped_gemm_bwd_workspace_bytes(R_cap, f), 256-byte aligned.  On return it holds
 *   dg [R_cap, f] bf16 at ws and du [R_cap, f] bf16 at ws + (that size / 2) (rows below
 *   expert_offsets[E] written): a caller may read them, e.g. to check them.
 */
int moe_grouped_gemm_bwd(const moe_bf16* dyp, const moe_bf16* xp,
                         const moe_bf16* g, const moe_bf16* u, const moe_bf16* h,
                         const int32_t* expert_offsets,
                         const moe_bf16* Wg, const moe_bf16* Wu, const moe_bf16* Wd,
                         int E, int R_cap, int d, int f,
                         moe_bf16* dxp, moe_bf16* dWg, moe_bf16* dWu, moe_bf16* dWd,
                         void* ws, size_t ws_bytes, void* stream);

/* The same with xp[r] = x[row_token[r]] read through row_token by the two weight-gradient
 * products that need it (dWg, dWu); x, T, row_token as for moe_grouped_gemm_fwd_gather. */
int moe_grouped_gemm_bwd_gather(const moe_bf16* dyp, const moe_bf16* x, int T, const int32_t* row_token,
                                const moe_bf16* g, const moe_bf16* u, const moe_bf16* h,
                                const int32_t* expert_offsets,
                                const moe_bf16* Wg, const moe_bf16* Wu, const moe_bf16* Wd,
                                int E, int R_cap, int d, int f,
                                moe_bf16* dxp, moe_bf16* dWg, moe_bf16* dWu, moe_bf16* dWd,
                                void* ws, size_t ws_bytes, void* stream);

/*
 * Stages 1-3 in one call (Algorithm 1: Softmax, TopK, token counting, index generation), and the Stage-4
 * gather if xp is given: the results of moe_route followed by moe_permute (or moe_permute_gate), bit for
 * bit, with one launch fewer: the routing kernel counts its own winners per local expert, so the pairs are
 * not read back to be counted.
 *   logits, topk_idx, topk_w, renormalize   as moe_route (both outputs are written in full)
 *   x, xp                                   as moe_permute; both may be NULL (index generation only)
 *   row_weight                              as moe_permute_gate, or NULL
 *   expert_offsets, row_token, slot_row, ws as moe_permute (a workspace beyond the minimum is put to use: the
 *                                           count table may then have more, shorter rows of tokens, which
 *                                           spares the routing kernel a second pass; the results do not change)
 */
int moe_route_permute(const float* logits, const moe_bf16* x, int T, int d, int E_total, int k, int renormalize,
                      int e_begin, int e_count, int32_t* topk_idx, float* topk_w,
                      int32_t* expert_offsets, int32_t* row_token, int32_t* slot_row, float* row_weight,
                      moe_bf16* xp, void* ws, size_t ws_bytes, void* stream);

/*
 * The layer with the gate weights folded into the expert MLP (Stages 2-5 and their derivatives give the
 * same out, dx, dW and dgate; the gate-weighted sum of Stage 5 is linear, so the weight of a routed row
 * may multiply h instead of the expert's output).  Forward: moe_permute_gate, moe_grouped_gemm_fwd_folded,
 * moe_unpermute_sum.  Backward: moe_grouped_gemm_bwd_folded, moe_permute_bwd.  The backward then needs
 * neither yp nor the scaled output gradient dyp[r] = w_r dout[token_r]: no separate pass over [R, d] rows
 * computes dgate and dyp.
 *
 * moe_permute_gate: moe_permute without moving rows, plus the gate weight of every routed row:
 *   row_weight[slot_row[t, i]] = topk_w[t, i] for every local slot.  topk_w [T, k] fp32 (device),
 *   row_weight [R_cap] fp32 (device, written for rows below expert_offsets[e_count]); the rest as moe_permute.
 */
int moe_permute_gate(const int32_t* topk_idx, const float* topk_w, int T, int E_total, int k, int e_begin, int e_count,
                     int32_t* expert_offsets, int32_t* row_token, int32_t* slot_row, float* row_weight,
                     void* ws, size_t ws_bytes, void* stream);

/*
 * moe_grouped_gemm_fwd_gather with hw = w_r * silu(g) * u in place of h (w_r = row_weight[r], applied to
 * the fp32 value before the one rounding to bf16) and therefore ypw = hw . Wd[e]^T = w_r * yp in place of yp.
 * g and u are as before.  row_weight [R_cap] fp32 (device); the rest as moe_grouped_gemm_fwd_gather.
 */
int moe_grouped_gemm_fwd_folded(const moe_bf16* x, int T, const int32_t* row_token, const float* row_weight,
                                const int32_t* expert_offsets,
                                const moe_bf16* Wg, const moe_bf16* Wu, const moe_bf16* Wd,
                                int E, int R_cap, int d, int f,
                                moe_bf16* g, moe_bf16* u, moe_bf16* hw, moe_bf16* ypw, void* stream);

/* out[t] = sum over local slots i, in slot order, of ypw[slot_row[t, i]] (fp32 sum, rounded once): Stage 5
 * for rows that already carry their gate weight.  Shapes as moe_unpermute_combine. */
int moe_unpermute_sum(const moe_bf16* ypw, const int32_t* slot_row, int T, int k, int d, moe_bf16* out, void* stream);

/*
 * Derivative of Stages 4 and 5 after moe_grouped_gemm_fwd_folded, from dout [T, d] itself.  With
 * t_r = row_token[r], w_r = row_weight[r], s = sigmoid(g):
 *   dh0 = dout[t_r] . Wd[e];  dgate[t, i] = sum_c dh0[r, c] * silu(g[r, c]) * u[r, c] for r = slot_row[t, i]
 *   (0 for a slot without local row; fp32: per 64-column strip in column order, strips added in order);
 *   dh = w_r * dh0;  dg, du, dxp, dWg, dWu as in moe_grouped_gemm_bwd (rows of x read through row_token);
 *   dWd[e] = dout[t_r]^T . hw   (rows of dout read through row_token).
 *   dout, x [T, d] bf16 (T*d*2 bytes at most 4 GiB); slot_row [T, k] int32; g, u, hw [R_cap, f] bf16;
 *   dgate [T, k] fp32; dxp [R_cap, d]; dWg, dWu [E, f, d]; dWd [E, d, f]; all device memory.
 *   ws at least moe_grouped_gemm_bwd_folded_workspace_bytes(R_cap, f): dg, du and the strips' partial sums.
 */
size_t moe_grouped_gemm_bwd_folded_workspace_bytes(int R_cap, int f);
int moe_grouped_gemm_bwd_folded(const moe_bf16* dout, const moe_bf16* x, int T, int k,
                                const int32_t* row_token, const float* row_weight, const int32_t* slot_row,
                                const moe_bf16* g, const moe_bf16* u, const moe_bf16* hw,
                                const int32_t* expert_offsets,
                                const moe_bf16* Wg, const moe_bf16* Wu, const moe_bf16* Wd,
                                int E, int R_cap, int d, int f,
                                moe_bf16* dxp, moe_bf16* dWg, moe_bf16* dWu, moe_bf16* dWd, float* dgate,
                                void* ws, size_t ws_bytes, void* stream);

/*
 * Stage 5, ExpertOutputReductionForward:
 *   out[t] = sum over local slots i, in slot order, of topk_w[t, i] * yp[slot_row[t, i]]
 * (fp32 sum, rounded once); zeros for a token without local slot.
 *   yp [R_cap, d] bf16, slot_row [T, k] int32, topk_w [T, k] fp32, out [T, d] bf16
 */
int moe_unpermute_combine(const moe_bf16* yp, const int32_t* slot_row, const float* topk_w,
                          int T, int k, int d, moe_bf16* out, void* stream);

/*
 * Stage 5, ExpertOutputReductionBackward:
 *   dyp[slot_row[t, i]] = topk_w[t, i] * dout[t]
 *   dgate[t, i] = <yp[slot_row[t, i]], dout[t]>   (0 where slot_row[t, i] < 0)
 * dgate is the gradient with respect to the weights as used by the combine.
 *   dout [T, d] bf16, yp, dyp [R_cap, d] bf16, dgate [T, k] fp32
 */
int moe_unpermute_combine_bwd(const moe_bf16* dout, const moe_bf16* yp,
                              const int32_t* slot_row, const float* topk_w,
                              int T, int k, int d, moe_bf16* dyp, float* dgate, void* stream);

/*
 * The router itself and the derivative of Stage 1 (Algorithm 1: logits = Router(input), a Linear
 * layer; the paper leaves the backward pass to autograd).  These calls complete the layer as a
 * drop-in block: moe_router_fwd feeds moe_route, and dgate from moe_unpermute_combine_bwd goes
 * back through moe_route_bwd and moe_router_bwd.
 *
 * moe_router_fwd:  logits[t, e] = sum_j x[t, j] * Wr[e, j]   (no bias)
 *   x [T, d] bf16, Wr [E, d] fp32, logits [T, E] fp32 out.  d % 16 == 0, E <= MOE_MAX_EXPERTS.
 *   The products are formed exactly and summed in fp32 (the summation order differs from a host
 *   matrix product, so logits agree to fp32 rounding, not bit for bit).
 */
int moe_router_fwd(const moe_bf16* x, const float* Wr, int T, int d, int E, float* logits, void* stream);

/*
 * moe_route_bwd:  gradient with respect to the logits for given dgate[t, i] = dL/d topk_w[t, i],
 * the chosen experts held fixed.  With p = Softmax(logits), s_i = p[topk_idx[t, i]], S = sum_i s_i:
 *   renormalize != 0:  dL/ds_i = (dgate_i - sum_j dgate_j * s_j / S) / S ;  otherwise dL/ds_i = dgate_i
 *   dlogits[t, e] = p_e * (dL/dp_e - sum_i dL/ds_i * s_i),  dL/dp_e = dL/ds_i if e = topk_idx[t, i], else 0.
 *   logits [T, E] fp32, topk_idx [T, k] int32 (distinct per token), dgate [T, k] fp32,
 *   dlogits [T, E] fp32 out.
 */
int moe_route_bwd(const float* logits, const int32_t* topk_idx, const float* dgate, int T, int E, int k,
                  int renormalize, float* dlogits, void* stream);

/*
 * moe_router_bwd:  derivative of the Linear layer.
 *   dWr[e, j] = sum_t dlogits[t, e] * x[t, j]                  fp32 [E, d] out (overwritten)
 *   dx[t, j] += sum_e dlogits[t, e] * Wr[e, j]                 bf16 [T, d] IN-OUT: the router's share
 *     is ADDED to what dx holds (the expert path's gradient from moe_permute_bwd), in fp32, and the
 *     sum is rounded once.  This is the one argument of the library that is accumulated into.
 *   ws at least moe_router_bwd_workspace_bytes(T, d, E): partial sums of dWr over chunks of 256
 *   tokens, reduced in a fixed order (no atomics: results are reproducible).
 */
size_t moe_router_bwd_workspace_bytes(int T, int d, int E);
int moe_router_bwd(const moe_bf16* x, const float* Wr, const float* dlogits, int T, int d, int E,
                   moe_bf16* dx, float* dWr, void* ws, size_t ws_bytes, void* stream);

/*
 * In front of a layer: the residual's addition and the root-mean-square norm, with s = bf16(x + r) and
 * q[t] = 1 / sqrt(mean over c of s[t, c]^2 + eps):
 *   sum[t, c] = s[t, c];  y[t, c] = s[t, c] * q[t] * w[c]  (fp32, rounded once);  rstd[t] = q[t] if rstd is not NULL
 *   x, r, sum, y [T, d] bf16; w [d] fp32; rstd [T] fp32 or NULL.  r may be NULL (the first norm: s = x); sum may then be NULL.
 *   sum may be x or r, and y too.  d % 8 == 0, d <= 32768; eps >= 0 (0: a row of zeros has no norm, its y is NaN).
 *   A row whose squares sum up to more than fp32 holds (values of 1e19) counts as infinite: q = 0.
 */
int moe_add_rms_norm(const moe_bf16* x, const moe_bf16* r, const float* w, int T, int d, float eps,
                     moe_bf16* sum, moe_bf16* y, float* rstd, void* stream);

/*
 * The same with y in 8 bits, the input of products in e4m3: each `group` columns of a row share a scale,
 *   scale[t, i] = max |y| / 448 over the group;  codes[t, c] = e4m3(y[t, c] / scale)  (codes of an all-zero group are zero)
 *   codes [T, d] bytes (OCP e4m3, nearest even); scale [T, d / group] fp32.  group: 0 (one per row), or a power of two from 8 to 512
 *   that divides d.  The rest as moe_add_rms_norm.
 */
int moe_add_rms_norm_8bit(const moe_bf16* x, const moe_bf16* r, const float* w, int T, int d, float eps, int group,
                          moe_bf16* sum, uint8_t* codes, float* scale, float* rstd, void* stream);

/*
 * Derivative of moe_add_rms_norm, from dy and the gradient dsum of the sum itself (NULL: none):
 *   dx[t, c] = dsum[t, c] + q (dy w - s q^2 mean over c of (dy w s)): the gradient of x and of r alike
 *   dw[c] = sum over t of dy s q   (fp32, a fixed order)
 *   dy, dsum, sum, dx [T, d] bf16 (dx may be dy or dsum); w, dw [d] fp32; rstd [T] as the forward call left it.
 *   ws at least moe_add_rms_norm_bwd_workspace_bytes(T, d).
 */
size_t moe_add_rms_norm_bwd_workspace_bytes(int T, int d);
int moe_add_rms_norm_bwd(const moe_bf16* dy, const moe_bf16* dsum, const moe_bf16* sum, const float* w, const float* rstd,
                         int T, int d, moe_bf16* dx, float* dw, void* ws, size_t ws_bytes, void* stream);

/*
 * Behind the layers: softmax cross entropy of the vocabulary head without the logits in memory.  With z[t] = x[t] . W^T:
 *   lse[t] = log sum over v of exp(z[t, v]);  loss[t] = lse[t] - z[t, target[t]]
 * and zeros for a token whose target lies outside [0, V): it counts for nothing, and takes no time in the products (but in a forward pass of up to 256
 * tokens, one pass over W in any case, or with a teacher in any pass of up to 128).  z[t, target[t]] is summed in 64 bits.
 *   x [T, d] bf16; W [V, d] bf16; target [T] int32; loss, lse [T] fp32.  d % 64 == 0; V <= 2^20.
 *   ws at least moe_head_fwd_workspace_bytes(T, d, V, 0): about T d * 2 + T V * 3 / 16 bytes.
 * A token with a logit that is NaN or infinite has NaN for its losses and its dx, and makes all of dW NaN.  So has one whose logits (for kd: over the
 * temperature) are 2^30 or larger; up to 2^29 the losses are right.
 */
size_t moe_head_fwd_workspace_bytes(int T, int d, int V, int K);
int moe_head_ce_fwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, int T, int d, int V,
                    float* loss, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * Its derivative for given dloss [T] fp32 (weights, and the division by a number of tokens, are in it):
 *   dz[t, v] = dloss[t] (exp(z[t, v] - lse[t]) - [v == target[t]]);  dx = dz . W;  dW = dz^T . x
 *   dx [T, d], dW [V, d] bf16, overwritten (zeros for a token without a target); loss, lse as the forward call left them.
 * The logits are formed again, dz is rounded to bf16 in the workspace, a piece of v_piece columns of the vocabulary at a time (a multiple
 * of 256; 0: as many as keep a piece under 2 GiB).  The workspace is about T d * 2 + T v_piece * 2 bytes and
 * T d * 4 for each part that dx is summed in.
 */
size_t moe_head_bwd_workspace_bytes(int T, int d, int V, int K, int v_piece);
int moe_head_ce_bwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const float* loss, const float* lse, const float* dloss,
                    int T, int d, int V, int v_piece, moe_bf16* dx, moe_bf16* dW, void* ws, size_t ws_bytes, void* stream);

/*
 * Cross entropy together with distillation from a teacher's top logits.  A token's entries are ids[t, j] with teacher[t, j], j < K <= 1024,
 * those with an id outside [0, V) or a logit of -infinity left out.  With q = softmax over the entries of teacher / temperature:
 *   kd[t] = sum over the entries of q (log q - log p),  p = softmax over the vocabulary of z / temperature
 *   lse_t[t] = log sum over v of exp(z[t, v] / temperature)
 * (zeros for a token without entries), and loss, lse as above, either of the two with or without the other.
 *   ids [T, K] int32; teacher [T, K] fp32; kd, lse_t [T] fp32; 0 < temperature < infinity.
 * Backward, for dloss and dkd [T] fp32:  dz += dkd / temperature (p - q) for a token with entries.
 * Entries may lie as far below each other as fp32 goes: one with q = 0 still has its p in kd and the gradient.
 * Preconditions: a token's valid ids are distinct, their logits not +infinity.  (One that is NaN is left out.)
 */
int moe_head_distill_fwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const int32_t* ids, const float* teacher,
                         float temperature, int T, int d, int V, int K, float* loss, float* lse, float* kd, float* lse_t,
                         void* ws, size_t ws_bytes, void* stream);
int moe_head_distill_bwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const int32_t* ids, const float* teacher,
                         float temperature, const float* loss, const float* lse, const float* lse_t, const float* dloss, const float* dkd,
                         int T, int d, int V, int K, int v_piece, moe_bf16* dx, moe_bf16* dW, void* ws, size_t ws_bytes, void* stream);

/*
 * What the head says of given tokens, at a temperature: with s = x[t] . W^T / temperature and p = softmax(s) over the vocabulary,
 *   lse[t] = log sum over v of exp(s[v]);  logp[t] = s[target[t]] - lse[t];  entropy[t] = -sum over v of p log p
 *   ids[t, 0 .. K), top[t, 0 .. K): the K columns of largest s, largest first, of equal ones the lower column first, and their log p.
 * A token whose target lies outside [0, V) counts for nothing: zeros, and ids of -1; beyond 256 tokens it takes no time in the products.
 *   x [T, d], W [V, d] bf16; target, ids int32; the rest fp32.  d % 64 == 0; V <= 2^20; 0 <= K <= 64 and K <= V (0: ids, top may be NULL); 0 < temperature < infinity.
 * Logits are compared in 64 bits among the K + 4 that are largest by the matrix product in 32 (its error is about 1e-6 of |x| |W row|).
 * Log probabilities and entropies are sums of positive terms: they keep their digits next to zero (down to 1e-35; what is smaller may be 0).  Logits that are NaN or +infinite, or 2^30 and more over the
 * temperature, give NaN; one of -infinity is a column that is not there (its log p is -infinity; with fewer columns than K ids are -1 and top NaN), for the forward call.  ws at least moe_head_score_fwd_workspace_bytes(T, d, V, K): about T d * 2 + T V * 5 / 8 bytes, T d * 2 + T V / 4 without alternatives; with
 * alternatives from a small vocabulary (up to 4000 columns, and up to 16384 if many are wanted) the logits themselves, T d * 2 + T V * 4; and up to eight times
 * T V * 4 where few tokens and columns (up to 16384) have long rows, whose products go in parts.
 */
size_t moe_head_score_fwd_workspace_bytes(int T, int d, int V, int K);
int moe_head_score_fwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, float temperature, int T, int d, int V, int K,
                       float* logp, float* entropy, float* lse, int32_t* ids, float* top, void* ws, size_t ws_bytes, void* stream);

/*
 * Its derivative for given dlogp and dentropy [T] fp32 (NULL: zeros), with logp, entropy and lse as the forward call left them:
 *   dz[t, v] = (dlogp ([v == target] - p) - dentropy p (log p + entropy)) / temperature;  dx = dz . W;  dW = dz^T . x
 * Sizes, pieces of the vocabulary and rounding as moe_head_ce_bwd; dW takes what rounding dz loses for up to 256 tokens that count.  ws at least
 * moe_head_score_bwd_workspace_bytes(T, d, V, v_piece).  (A workspace of that size for T tokens serves fewer tokens as well, here and in the forward call, as it does in
 * moe_head_ce_* and moe_head_distill_*; where the reductions have room for fewer parts than the rules take, sums are added up in another order.)
 * p is off by about 1e-6 of the logits' size over the temperature times itself, and log p + entropy by as much, but for the likeliest column of a token with an entropy below
 * 1/4: that is formed apart, so that the gradient of an entropy next to zero has the digits of any other.  Logits of 10^6 and more over the temperature leave p no digits, and
 * their tokens' gradients may be NaN.
 */
size_t moe_head_score_bwd_workspace_bytes(int T, int d, int V, int v_piece);
int moe_head_score_bwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, float temperature, const float* logp, const float* entropy,
                       const float* lse, const float* dlogp, const float* dentropy, int T, int d, int V, int v_piece, moe_bf16* dx, moe_bf16* dW,
                       void* ws, size_t ws_bytes, void* stream);

/*
 * Between a block's projections and its attention: the norm of every head's queries and keys, and the rotation by position, in one pass.  For a head's
 * row x of D columns:  v = x w / sqrt(mean(x^2) + eps);  then R of its columns are turned, pair i by the angle pos[t] freq[i] (formed in 64 bits):
 *   (a, b) -> (a cos - b sin, a sin + b cos),  the pairs being (2 i, 2 i + 1) if `pairs` is not 0, else (i, i + R / 2);  columns from R on stay.
 *   q, qo [T, Hq, D], k, ko [T, Hk, D] bf16, each with its own distance `ld` from a token to the next in elements (a multiple of 8, at least H D: queries and
 *   keys may be columns of a wider matrix); wq, wk [D] fp32; pos [T] int32 of any value; freq [R / 2] fp32 (may be NULL for R = 0).
 *   D % 8 == 0, D <= 512; R % 16 == 0, 0 <= R <= D; Hq, Hk <= 4096; T <= 2^30.  qo may be q and ko may be k (with the same ld); no other overlap.
 *   eps >= 0 (0: a head of zeros has no norm, its columns are NaN, and one whose mean square is below 2^-126, values of 1e-19, loses digits).  A head whose squares sum up to more than fp32 holds (values of 1e19) counts as infinite: zeros.
 */
int moe_qk_norm_rope(const moe_bf16* q, long long q_ld, const moe_bf16* k, long long k_ld, const float* wq, const float* wk, const int32_t* pos,
                     const float* freq, int pairs, float eps, int T, int Hq, int Hk, int D, int R, moe_bf16* qo, long long qo_ld,
                     moe_bf16* ko, long long ko_ld, void* stream);

/*
 * Its derivative, from the gradients dqo, dko of what it gave and the q, k that it was given (root and rotation are formed again):
 *   dv = dqo turned back;  dq = r (dv w - q r^2 mean(dv w q)), r = 1 / sqrt(mean(q^2) + eps);  dwq = sum over tokens and heads of dv q r  (fp32, a fixed order)
 * and likewise for k.  dq may be dqo or q, dk may be dko or k (with the same ld).  ws at least moe_qk_norm_rope_bwd_workspace_bytes(T, Hq, Hk, D).
 */
size_t moe_qk_norm_rope_bwd_workspace_bytes(int T, int Hq, int Hk, int D);
int moe_qk_norm_rope_bwd(const moe_bf16* dqo, long long dqo_ld, const moe_bf16* dko, long long dko_ld, const moe_bf16* q, long long q_ld,
                         const moe_bf16* k, long long k_ld, const float* wq, const float* wk, const int32_t* pos, const float* freq, int pairs,
                         float eps, int T, int Hq, int Hk, int D, int R, moe_bf16* dq, long long dq_ld, moe_bf16* dk, long long dk_ld,
                         float* dwq, float* dwk, void* ws, size_t ws_bytes, void* stream);

/*
 * Behind a backward pass: the norm of all gradients of a model together, and their scaling to a largest norm.
 *   norm[0] = sqrt(sum over all tensors of g^2)  (summed in 64 bits in a fixed order, then rounded to fp32)
 *   moe_grad_clip: out = g min(1, largest / (norm + 1e-6)), the scale and the product rounded to fp32, then to the type; the norm is that of the 64-bit sum.  A norm of infinity makes finite gradients 0, one
 *   of NaN makes all of them NaN.
 * `grads` is a HOST array of n <= 2^20 tensors; it is read before the call returns, so a captured call keeps the addresses that it was given.  A tensor is dense, at any
 * multiple of its elements' size, and may have no elements (its pointers are then not looked at).  out may be in: nothing is written where the scale is
 * 1, as where norm + 1e-6 is no larger than `largest`.  An output that overlaps another tensor's input or output, the norm or the workspace is refused, and so is a norm or a workspace over an
 * input or over each other.  moe_grad_norm does not look at `out`.
 *   norm [1] fp32; 0 < largest < infinity.  ws at least moe_grad_norm_workspace_bytes(n).
 */
enum { MOE_TYPE_BF16 = 0, MOE_TYPE_F32 = 1 };
typedef struct moe_grad {
  const void* in;
  void* out;
  int64_t count, type;
} moe_grad;
size_t moe_grad_norm_workspace_bytes(int n);
int moe_grad_norm(const moe_grad* grads, int n, float* norm, void* ws, size_t ws_bytes, void* stream);
int moe_grad_clip(const moe_grad* grads, int n, double largest, float* norm, void* ws, size_t ws_bytes, void* stream);

/*
 * Several stages of one layer with one call: the calls above in the layer's order, on buffers that the caller
 * laid out once, so that a small step does not spend its time crossing a language boundary a dozen times.
 * `what` is a sum of MOE_LAYER_ROUTER (moe_router_fwd into logits), MOE_LAYER_FWD (Stages 1-5), MOE_LAYER_BWD
 * (their derivatives; the forward call's buffers must be as it left them) and MOE_LAYER_ROUTER_BWD (moe_route_bwd,
 * moe_router_bwd).  `path` chooses the calls: MOE_LAYER_PLAIN (xp is materialised, dyp is used), MOE_LAYER_GATHER
 * (rows gathered by the products, no xp), MOE_LAYER_FOLD (gate weights folded: h and yp hold hw and ypw; no xp, no
 * dyp, row_weight is used).  Sizes, buffers and errors are those of the calls; pointers that the chosen stages and
 * path do not use may be NULL.  A stage that fails leaves the stages before it enqueued.  With FWD and BWD in one call
 * `dout` may be `out` (the gradient of half the squared output): the backward reads what the forward has written.
 * A forward pass of few tokens runs several stages in one kernel, with the results of the calls one by one.
 */
enum { MOE_LAYER_PLAIN = 0, MOE_LAYER_GATHER = 1, MOE_LAYER_FOLD = 2 };
enum { MOE_LAYER_ROUTER = 1, MOE_LAYER_FWD = 2, MOE_LAYER_BWD = 4, MOE_LAYER_ROUTER_BWD = 8 };
typedef struct moe_layer {
  int32_t T, d, E, k, f, e_begin, e_count, renormalize, path, reserved;
  const moe_bf16 *x, *dout, *Wg, *Wu, *Wd;
  const float* Wr;
  float* logits;                  /* read by MOE_LAYER_FWD, written by MOE_LAYER_ROUTER */
  float *dlogits, *dWr;
  int32_t* topk_idx;
  float* topk_w;
  int32_t *expert_offsets, *row_token, *slot_row;
  float* row_weight;
  moe_bf16 *xp, *g, *u, *h, *yp, *out, *dyp, *dxp, *dx;
  float* dgate;
  moe_bf16 *dWg, *dWu, *dWd;
  void* ws;
  size_t ws_bytes;
} moe_layer;
int moe_layer_run(const moe_layer* layer, int what, void* stream);

/*
 * Per-kernel timing for benchmarks (not part of the paper's method).  While
 * enabled, every kernel the library launches is bracketed by two HIP events
 * recorded on the launch stream.  moe_prof_read synchronises on the recorded
 * events and returns, for entry `index` (0 .. moe_prof_count()-1), the kernel's
 * name, its summed duration in milliseconds and its launch count.  These calls
 * create HIP events (host objects) and are not thread-safe; leave profiling off
 * in production.
 */
int moe_prof_enable(int on);        /* also clears what was recorded */
int moe_prof_count(void);
int moe_prof_read(int index, char* name, int name_cap, float* total_ms, int* launches);

/*
 * Matrix-pipe probe for benchmarks (not part of the paper's method): what rate of
 * v_mfma_f32_16x16x32_bf16 (the form the grouped products use) the chip sustains for given operand VALUES.  The clock
 * of the chip follows its power draw, which depends on how many operand bits
 * toggle, so the ceiling for real data lies below the published peak.
 *   a    [workgroups*512, 32] bf16, device: 4 activation fragments per lane
 *   b    [workgroups*512, 16] bf16, device: 2 weight fragments per lane
 *   sink [workgroups*512] f32, device, overwritten (keeps the loop alive)
 * Launches `workgroups` workgroups of 8 waves, each lane issuing 8*iters MFMAs on
 * its register-resident fragments with no memory traffic, waits for the kernel
 * (this call synchronises on its own events) and returns its duration in
 * milliseconds, its FLOP count and the core clock in GHz observed by wave 0.
 */
int moe_prof_mfma_ceiling(const moe_bf16* a, const moe_bf16* b, int workgroups, int iters, float* sink,
                          float* ms, double* flop, double* clock_ghz, void* stream);

/*
 * Memory probe for benchmarks (not part of the paper's method): a kernel that only reads.  `workgroups`
 * workgroups of 256 threads read the first bytes / 16384 whole 16 KB blocks of src (device, 16-byte aligned)
 * with 16-byte loads and write one word per thread to sink [workgroups * 256] (device).  Enqueued on
 * `stream` like any other call (timed through moe_prof_enable / moe_prof_read under the name
 * "stream_read"); the rate it reaches on buffers that no cache holds is what the row movers' rates
 * should be read against.
 */
int moe_prof_stream_read(const void* src, size_t bytes, uint32_t* sink, int workgroups, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_HOTPATH_H */
