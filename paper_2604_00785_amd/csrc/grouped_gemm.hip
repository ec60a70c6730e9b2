// Stage 4 of Algorithm 1 (the three Grouped_mm calls around Silu(gate)*up) and
// its derivative, as grouped bf16 MFMA GEMMs: one launch covers every expert.
// The kernels stand in gemm_tile.h; here the calls fill in their arguments.
#include "gemm_tile.h"
#include "small_gemm.h"

namespace {

bool bad_gemm_dims(int E, int R_cap, int d, int f) {
  return E <= 0 || E > MOE_MAX_EXPERTS || R_cap <= 0 || d <= 0 || f <= 0 || d % 64 != 0 || f % 64 != 0;
}

inline const uint16_t* U16(const moe_bf16* p) { return p; }

}  // namespace

extern "C" size_t moe_grouped_gemm_bwd_workspace_bytes(int R_cap, int f) {
  if (R_cap <= 0 || f <= 0) return 0;
  const size_t one = (static_cast<size_t>(R_cap) * f * sizeof(moe_bf16) + 255) & ~static_cast<size_t>(255);
  return 2 * one;
}

extern "C" size_t moe_workspace_bytes(int T, int E, int k, int d, int f) {
  if (T <= 0 || k <= 0 || E <= 0 || d <= 0 || f <= 0) return 0;
  const unsigned long long rows = static_cast<unsigned long long>(T) * static_cast<unsigned long long>(k);
  if (rows > 0x7FFFFFFFull) return 0;   // no call takes that many routed rows
  const int R_cap = static_cast<int>(rows);
  // the largest of every workspace any call may ask for on a layer of this shape
  const size_t sizes[] = {moe_permute_workspace_bytes(T, k, E), moe_grouped_gemm_bwd_workspace_bytes(R_cap, f),
                          moe_grouped_gemm_bwd_folded_workspace_bytes(R_cap, f), moe_router_bwd_workspace_bytes(T, d, E)};
  size_t m = 0;
  for (size_t v : sizes) m = v > m ? v : m;
  return m;
}

// xp grouped rows, or (row_token not null) the token rows themselves, gathered by the GEMM's loads
extern "C" int moe_gemm_fwd(const moe_bf16* xp, const int32_t* row_token, const float* row_weight, const int32_t* expert_offsets, const moe_bf16* Wg,
                 const moe_bf16* Wu, const moe_bf16* Wd, int E, int R_cap, long long rows, int most, int d, int f,
                 moe_bf16* g, moe_bf16* u, moe_bf16* h, moe_bf16* yp, void* stream, int* edges) {
  if (!xp || !expert_offsets || !Wg || !Wu || !Wd || !g || !u || !h || !yp) return MOE_ERR_INVALID;
  if (bad_gemm_dims(E, R_cap, d, f) || bad_edges(edges)) return MOE_ERR_INVALID;
  const void* ptrs[] = {xp, expert_offsets, Wg, Wu, Wd, g, u, h, yp};
  for (const void* p : ptrs) if (!moe_aligned16(p)) return MOE_ERR_INVALID;
  hipStream_t s = static_cast<hipStream_t>(stream);
  // Few rows for certain: the streaming kernels.  Few rows expected, but not for certain (a rank's share of the experts): both,
  // and on the device one of the two finds that the rows are not for it (see small_gemm.h).
  const int few = STREAM_ROWS * E;
  const bool tiled = edges != nullptr && (edges[0] != 0 || edges[1] != 0);
  const bool streamed = !tiled && (R_cap <= few || most <= STREAM_TOKENS), either = !tiled && !streamed && rows <= few;
  int rc = MOE_OK;
  StreamFwdArgs p{}, q{};
  if (streamed || either) {
    p.A = U16(xp); p.row_token = row_token; p.row_weight = row_weight; p.offsets = expert_offsets;
    p.B0 = U16(Wg); p.B1 = U16(Wu); p.O0 = g; p.O1 = u; p.O2 = h; p.E = E; p.K = d; p.N = f;
    q.A = U16(h); q.offsets = expert_offsets; q.B0 = U16(Wd); q.O0 = yp; q.E = E; q.K = f; q.N = d;
    p.max_rows = q.max_rows = either ? few : R_cap;
    if ((rc = moe_stream_gate_up(p, rows, s)) != MOE_OK) return rc;
    if (streamed) return moe_stream_down(q, rows, s);
  }
  GemmArgs a{};
  a.offsets = expert_offsets; a.E = E; a.row_token = row_token; a.row_weight = row_weight;
  // gate | up with the SwiGLU epilogue
  a.A0 = U16(xp); a.B0 = U16(Wg); a.B1 = U16(Wu); a.O0 = g; a.O1 = u; a.O2 = h;
  a.K = d; a.N = f;
  a.stream_rows = either ? few : 0;
  rc = run_gemm<GATE_UP>(a, R_cap, rows, s, "gemm_gate_up", edges);
  if (rc != MOE_OK) return rc;
  // down
  if (either && (rc = moe_stream_down(q, rows, s)) != MOE_OK) return rc;
  GemmArgs b{};
  b.offsets = expert_offsets; b.E = E;
  b.A0 = U16(h); b.B0 = U16(Wd); b.O0 = yp;
  b.K = f; b.N = d;
  b.stream_rows = a.stream_rows;
  return run_gemm<DOWN>(b, R_cap, rows, s, "gemm_down", edges != nullptr ? edges + 1 : nullptr);
}

namespace {
// byte offsets of gathered rows are 32-bit lane offsets from the start of x (T*width*2 bytes just under 4 GiB at most)
bool bad_gather(const moe_bf16* x, int T, const int32_t* row_token, int width) {
  return !x || !row_token || T <= 0 || !moe_aligned16(row_token) ||
         static_cast<unsigned long long>(T) * width * sizeof(moe_bf16) > 0xFFFFFFFFull - 65536;   // lane offsets carry a small bias on top
}
}  // namespace

// x, row_token: rows gathered; row_weight (or null): gate weights folded into h.  No expert has more rows than
// there are tokens, since a token's experts are distinct.
int moe_gemm_fwd_gather(const moe_bf16* x, int T, const int32_t* row_token, const float* row_weight, const int32_t* expert_offsets,
                        const moe_bf16* Wg, const moe_bf16* Wu, const moe_bf16* Wd, int E, int R_cap, long long rows, int d,
                        int f, moe_bf16* g, moe_bf16* u, moe_bf16* h, moe_bf16* yp, void* stream) {
  if (bad_gather(x, T, row_token, d)) return MOE_ERR_INVALID;
  return moe_gemm_fwd(x, row_token, row_weight, expert_offsets, Wg, Wu, Wd, E, R_cap, rows, T, d, f, g, u, h, yp, stream);
}

extern "C" int moe_grouped_gemm_fwd(const moe_bf16* xp, const int32_t* expert_offsets, const moe_bf16* Wg,
                                    const moe_bf16* Wu, const moe_bf16* Wd, int E, int R_cap, int d, int f,
                                    moe_bf16* g, moe_bf16* u, moe_bf16* h, moe_bf16* yp, void* stream) {
  return moe_gemm_fwd(xp, nullptr, nullptr, expert_offsets, Wg, Wu, Wd, E, R_cap, R_cap, R_cap, d, f, g, u, h, yp, stream);
}

extern "C" int moe_grouped_gemm_fwd_gather(const moe_bf16* x, int T, const int32_t* row_token,
                                           const int32_t* expert_offsets, const moe_bf16* Wg, const moe_bf16* Wu,
                                           const moe_bf16* Wd, int E, int R_cap, int d, int f, moe_bf16* g,
                                           moe_bf16* u, moe_bf16* h, moe_bf16* yp, void* stream) {
  return moe_gemm_fwd_gather(x, T, row_token, nullptr, expert_offsets, Wg, Wu, Wd, E, R_cap, R_cap, d, f, g, u, h, yp, stream);
}

extern "C" int moe_grouped_gemm_fwd_folded(const moe_bf16* x, int T, const int32_t* row_token, const float* row_weight,
                                           const int32_t* expert_offsets, const moe_bf16* Wg, const moe_bf16* Wu,
                                           const moe_bf16* Wd, int E, int R_cap, int d, int f, moe_bf16* g,
                                           moe_bf16* u, moe_bf16* hw, moe_bf16* ypw, void* stream) {
  if (!row_weight || !moe_aligned16(row_weight)) return MOE_ERR_INVALID;
  return moe_gemm_fwd_gather(x, T, row_token, row_weight, expert_offsets, Wg, Wu, Wd, E, R_cap, R_cap, d, f, g, u, hw, ypw,
                             stream);
}

// xp grouped rows, or (row_token not null) the token rows themselves, gathered by the loads of the
// two weight-gradient products that read them
extern "C" int moe_gemm_bwd(const moe_bf16* dyp, const moe_bf16* xp, int T, const int32_t* row_token, const moe_bf16* g, const moe_bf16* u,
                 const moe_bf16* h, const int32_t* expert_offsets, const moe_bf16* Wg, const moe_bf16* Wu,
                 const moe_bf16* Wd, int E, int R_cap, long long rows, int d, int f, moe_bf16* dxp, moe_bf16* dWg,
                 moe_bf16* dWu, moe_bf16* dWd, void* ws, size_t ws_bytes, void* stream, int* edges) {
  if ((row_token != nullptr && bad_gather(xp, T, row_token, d)) || bad_edges(edges)) return MOE_ERR_INVALID;
  if (!dyp || !xp || !g || !u || !h || !expert_offsets || !Wg || !Wu || !Wd || !dxp || !dWg || !dWu || !dWd || !ws)
    return MOE_ERR_INVALID;
  if (bad_gemm_dims(E, R_cap, d, f)) return MOE_ERR_INVALID;
  const void* ptrs[] = {dyp, xp, g, u, h, expert_offsets, Wg, Wu, Wd, dxp, dWg, dWu, dWd, ws};
  for (const void* p : ptrs) if (!moe_aligned16(p)) return MOE_ERR_INVALID;
  if (ws_bytes < moe_grouped_gemm_bwd_workspace_bytes(R_cap, f)) return MOE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  uint16_t* dg = static_cast<uint16_t*>(ws);
  uint16_t* du = reinterpret_cast<uint16_t*>(static_cast<char*>(ws) + moe_grouped_gemm_bwd_workspace_bytes(R_cap, f) / 2);

  // Two launches of two independent products each (the second list of a launch takes over the workgroups
  // that the first leaves idle at its end).
  // dh = dyp . Wd, then the SwiGLU derivative -> dg, du (first: its tiles are the long ones) ; dWd = dyp^T h
  GemmArgs wd{};
  wd.offsets = expert_offsets; wd.E = E;
  wd.A0 = U16(dyp); wd.B0 = U16(h); wd.O0 = dWd; wd.M = d; wd.N = f;
  GemmArgs a{};
  a.offsets = expert_offsets; a.E = E;
  a.A0 = U16(dyp); a.B0 = U16(Wd); a.G = U16(g); a.U = U16(u); a.O0 = dg; a.O1 = du;
  a.K = d; a.N = f;
  int rc = run_gemm_pair<DGRAD_H, WGRAD>(a, wd, R_cap, rows, s, "gemm_dgrad_h+wgrad_down", edges);
  if (rc != MOE_OK) return rc;
  // dxp = dg . Wg + du . Wu ; dWg = dg^T xp and dWu = du^T xp (one list: both read the same rows of xp)
  GemmArgs w{};
  w.offsets = expert_offsets; w.E = E; w.row_token = row_token;
  w.A0 = dg; w.A1 = du; w.B0 = U16(xp); w.O0 = dWg; w.O1 = dWu; w.M = f; w.N = d;
  GemmArgs b{};
  b.offsets = expert_offsets; b.E = E;
  b.A0 = dg; b.A1 = du; b.B0 = U16(Wg); b.B1 = U16(Wu); b.O0 = dxp;
  b.K = f; b.N = d;
  // dgrad_x first: its tiles are the long ones, the weight gradients' many short tiles fill its tail
  int* edge = edges != nullptr ? edges + 1 : nullptr;
  if (row_token != nullptr) return run_gemm_pair<DGRAD_X, WGRAD_GATHER>(b, w, R_cap, rows, s, "gemm_wgrad_gate_up+dgrad_x", edge);
  return run_gemm_pair<DGRAD_X, WGRAD>(b, w, R_cap, rows, s, "gemm_wgrad_gate_up+dgrad_x", edge);
}

extern "C" int moe_grouped_gemm_bwd(const moe_bf16* dyp, const moe_bf16* xp, const moe_bf16* g, const moe_bf16* u,
                                    const moe_bf16* h, const int32_t* expert_offsets, const moe_bf16* Wg,
                                    const moe_bf16* Wu, const moe_bf16* Wd, int E, int R_cap, int d, int f,
                                    moe_bf16* dxp, moe_bf16* dWg, moe_bf16* dWu, moe_bf16* dWd, void* ws,
                                    size_t ws_bytes, void* stream) {
  return moe_gemm_bwd(dyp, xp, 0, nullptr, g, u, h, expert_offsets, Wg, Wu, Wd, E, R_cap, R_cap, d, f, dxp, dWg, dWu, dWd,
                      ws, ws_bytes, stream);
}

extern "C" int moe_grouped_gemm_bwd_gather(const moe_bf16* dyp, const moe_bf16* x, int T, const int32_t* row_token,
                                           const moe_bf16* g, const moe_bf16* u, const moe_bf16* h,
                                           const int32_t* expert_offsets, const moe_bf16* Wg, const moe_bf16* Wu,
                                           const moe_bf16* Wd, int E, int R_cap, int d, int f, moe_bf16* dxp,
                                           moe_bf16* dWg, moe_bf16* dWu, moe_bf16* dWd, void* ws, size_t ws_bytes,
                                           void* stream) {
  if (row_token == nullptr) return MOE_ERR_INVALID;
  return moe_gemm_bwd(dyp, x, T, row_token, g, u, h, expert_offsets, Wg, Wu, Wd, E, R_cap, R_cap, d, f, dxp, dWg, dWu, dWd,
                      ws, ws_bytes, stream);
}

// ---------------------------------------------------------------------------------------------
// Backward of a forward pass that folded the gate weights into h (moe_grouped_gemm_fwd_folded).
namespace {
// dgate[t, i] = sum over the column strips of the row's partial dot products (0 for a slot without a local row)
__global__ __launch_bounds__(256) void dgate_finish_kernel(const float* __restrict__ part, int strips,
                                                           const int32_t* __restrict__ slot_row, int n,
                                                           float* __restrict__ dgate) {
  const int idx = blockIdx.x * 256 + threadIdx.x;
  if (idx >= n) return;
  const int row = slot_row[idx];
  float sum = 0.f;
  if (row >= 0) {
    const float* p = part + static_cast<size_t>(row) * strips;
    for (int c = 0; c < strips; ++c) sum += p[c];
  }
  dgate[idx] = sum;
}

size_t folded_part_bytes(int R_cap, int f) {
  return (static_cast<size_t>(f / 64) * R_cap * sizeof(float) + 255) & ~static_cast<size_t>(255);
}
}  // namespace

extern "C" size_t moe_grouped_gemm_bwd_folded_workspace_bytes(int R_cap, int f) {
  if (R_cap <= 0 || f <= 0) return 0;
  return moe_grouped_gemm_bwd_workspace_bytes(R_cap, f) + folded_part_bytes(R_cap, f);
}

const float* moe_folded_part(const void* ws, int R_cap, int f) {
  return reinterpret_cast<const float*>(static_cast<const char*>(ws) + moe_grouped_gemm_bwd_workspace_bytes(R_cap, f));
}

extern "C" int moe_gemm_bwd_folded(const moe_bf16* dout, const moe_bf16* x, int T, int k,
                                           const int32_t* row_token, const float* row_weight, const int32_t* slot_row,
                                           const moe_bf16* g, const moe_bf16* u, const moe_bf16* hw,
                                           const int32_t* expert_offsets, const moe_bf16* Wg, const moe_bf16* Wu,
                                           const moe_bf16* Wd, int E, int R_cap, long long rows, int d, int f, moe_bf16* dxp,
                                           moe_bf16* dWg, moe_bf16* dWu, moe_bf16* dWd, float* dgate, void* ws,
                                           size_t ws_bytes, void* stream, int* edges) {
  if (!dout || !g || !u || !hw || !expert_offsets || !Wg || !Wu || !Wd || !dxp || !dWg || !dWu || !dWd || !ws || !row_weight || !slot_row || k <= 0)
    return MOE_ERR_INVALID;
  if (bad_gemm_dims(E, R_cap, d, f) || bad_gather(x, T, row_token, d) || bad_gather(dout, T, row_token, d) || bad_edges(edges))
    return MOE_ERR_INVALID;
  const void* ptrs[] = {dout, x, g, u, hw, expert_offsets, Wg, Wu, Wd, dxp, dWg, dWu, dWd, dgate, ws, row_weight, slot_row};
  for (const void* p : ptrs) if (!moe_aligned16(p)) return MOE_ERR_INVALID;
  if (ws_bytes < moe_grouped_gemm_bwd_folded_workspace_bytes(R_cap, f)) return MOE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const size_t one = moe_grouped_gemm_bwd_workspace_bytes(R_cap, f) / 2;
  uint16_t* dg = static_cast<uint16_t*>(ws);
  uint16_t* du = reinterpret_cast<uint16_t*>(static_cast<char*>(ws) + one);
  float* part = const_cast<float*>(moe_folded_part(ws, R_cap, f));

  // Two launches of two independent products each (the second list of a launch takes over the workgroups
  // that the first leaves idle at its end).
  // dh0 = dout[token] . Wd; dh = w dh0 -> dg, du; partial dot products of dh0 with h for the gate gradient
  // (first: its tiles are the long ones);
  // dWd = (w dout[token])^T h = dout[token]^T hw: rows of dout gathered by the loads of the A operand
  GemmArgs wd{};
  wd.offsets = expert_offsets; wd.E = E; wd.row_token = row_token;
  wd.A0 = U16(dout); wd.B0 = U16(hw); wd.O0 = dWd; wd.M = d; wd.N = f;
  GemmArgs a{};
  a.offsets = expert_offsets; a.E = E; a.row_token = row_token; a.row_weight = row_weight;
  a.dgate_part = part;
  a.A0 = U16(dout); a.B0 = U16(Wd); a.G = U16(g); a.U = U16(u); a.O0 = dg; a.O1 = du;
  a.K = d; a.N = f;
  int rc = run_gemm_pair<DGRAD_H_GATE, WGRAD_GATHER_A>(a, wd, R_cap, rows, s, "gemm_dgrad_h+wgrad_down", edges);
  if (rc != MOE_OK) return rc;
  if (dgate != nullptr) {
    const int n = T * k;
    MOE_LAUNCH("dgate_finish", dgate_finish_kernel, dim3((n + 255) / 256), dim3(256), 0, s, static_cast<const float*>(part),
               f / 64, slot_row, n, dgate);
  }
  // dWg = dg^T x[token] and dWu = du^T x[token] (one list: both read the same gathered rows of x), then
  // dxp = dg . Wg + du . Wu
  GemmArgs w{};
  w.offsets = expert_offsets; w.E = E; w.row_token = row_token;
  w.A0 = dg; w.A1 = du; w.B0 = U16(x); w.O0 = dWg; w.O1 = dWu; w.M = f; w.N = d;
  GemmArgs b{};
  b.offsets = expert_offsets; b.E = E;
  b.A0 = dg; b.A1 = du; b.B0 = U16(Wg); b.B1 = U16(Wu); b.O0 = dxp;
  b.K = f; b.N = d;
  // dgrad_x first: its tiles are the long ones, the weight gradients' many short tiles fill its tail.  (The other
  // order used to pay off through dxp still lying in the last-level cache when moe_permute_bwd read it; since that
  // kernel streams its rows with non-temporal loads it no longer depends on that.)
  return run_gemm_pair<DGRAD_X, WGRAD_GATHER>(b, w, R_cap, rows, s, "gemm_wgrad_gate_up+dgrad_x",
                                              edges != nullptr ? edges + 1 : nullptr);
}

extern "C" int moe_grouped_gemm_bwd_folded(const moe_bf16* dout, const moe_bf16* x, int T, int k,
                                           const int32_t* row_token, const float* row_weight, const int32_t* slot_row,
                                           const moe_bf16* g, const moe_bf16* u, const moe_bf16* hw,
                                           const int32_t* expert_offsets, const moe_bf16* Wg, const moe_bf16* Wu,
                                           const moe_bf16* Wd, int E, int R_cap, int d, int f, moe_bf16* dxp,
                                           moe_bf16* dWg, moe_bf16* dWu, moe_bf16* dWd, float* dgate, void* ws,
                                           size_t ws_bytes, void* stream) {
  if (!dgate) return MOE_ERR_INVALID;
  return moe_gemm_bwd_folded(dout, x, T, k, row_token, row_weight, slot_row, g, u, hw, expert_offsets, Wg, Wu, Wd, E, R_cap,
                             R_cap, d, f, dxp, dWg, dWu, dWd, dgate, ws, ws_bytes, stream);
}
