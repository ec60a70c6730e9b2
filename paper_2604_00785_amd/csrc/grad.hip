// The norm of all gradients of a model together, and their scaling to a largest norm:
//   norm = sqrt(sum over all tensors of g^2);   out = g min(1, largest / (norm + 1e-6))
// Bound by memory: one pass reads every gradient, the second reads it once more and writes it.  Squares and their sums are in 64 bits, so that gradients of any
// size have a norm; each workgroup leaves its sum, and whoever needs the norm adds these up in one order: no atomics, the same bits every time.
#include <algorithm>
#include <new>
#include "common.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
// (tensors may begin anywhere in a buffer of many: at multiples of their elements' size)
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t u32x4_any;

// What a launch knows of its tensors comes with its arguments, so that nothing has to be copied to the device first, in a graph or out of it.
constexpr int TENSORS = 120;                        // of a launch: 4 KB of arguments
constexpr int GRAD_GROUPS = 1024;                   // workgroups of a launch at most, each with its sum
constexpr int MAX_TENSORS = 1 << 20;
struct GradTable {
  const void* in[TENSORS];
  void* out[TENSORS];
  uint64_t count[TENSORS];                          // elements, and in the lowest bit whether they have 32 bits
  uint32_t first[TENSORS + 1];                      // first chunk
  uint32_t n;
};
static_assert(sizeof(GradTable) <= 3900, "kernel arguments");

__device__ __forceinline__ void add_squares(const u32x4& v, bool f32, double& s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (f32) {
      const double a = static_cast<double>(__uint_as_float(v[i]));
      s = __builtin_fma(a, a, s);
    } else {
      const double a = static_cast<double>(bf16lo(v[i])), b = static_cast<double>(bf16hi(v[i]));
      s = __builtin_fma(a, a, s);
      s = __builtin_fma(b, b, s);
    }
  }
}
__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
  for (int i = 1; i < MOE_WAVE; i *= 2) v += __shfl_xor(v, i);
  return v;
}
// The sum over 256 threads, in all of them.
__device__ __forceinline__ double group_total(double v, double (&part)[4]) {
  v = wave_total(v);
  if (threadIdx.x % MOE_WAVE == 0) part[threadIdx.x / MOE_WAVE] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

// f(tensor, is 32 bits, first piece of 16 bytes, pieces of the tensor, its elements, whether this is its last chunk) for the workgroup's chunks, a run of them: of
// 256 U pieces each.
template <int U, typename F> __device__ __forceinline__ void over_chunks(const GradTable& t, uint32_t total, bool backwards, F&& f) {
  const uint32_t b = backwards ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
  const uint32_t c0 = static_cast<uint32_t>(static_cast<uint64_t>(total) * b / gridDim.x), c1 = static_cast<uint32_t>(static_cast<uint64_t>(total) * (b + 1) / gridDim.x);
  if (c0 >= c1) return;
  uint32_t e = 0;                                   // the last tensor whose first chunk is not behind c0
  for (uint32_t step = 64; step > 0; step /= 2)
    if (e + step < t.n && t.first[e + step] <= c0) e += step;
  for (uint32_t c = c0; c < c1; ++e) {
    const uint32_t first = t.first[e], end = t.first[e + 1], to = end < c1 ? end : c1;
    const bool f32 = (t.count[e] & 1) != 0;
    const uint64_t count = t.count[e] >> 1, pieces = count / (f32 ? 4 : 8);
    for (; c < to; ++c) f(e, f32, static_cast<uint64_t>(c - first) * (256 * U), pieces, count, c + 1 == end);
  }
}

template <int U> __global__ __launch_bounds__(256) void grad_norm_kernel(GradTable t, double* __restrict__ sums) {
  __shared__ double part[4];
  double s = 0.0;
  over_chunks<U>(t, t.first[t.n], false, [&](uint32_t e, bool f32, uint64_t p0, uint64_t pieces, uint64_t count, bool last) __attribute__((always_inline)) {
    const u32x4_any* in = static_cast<const u32x4_any*>(t.in[e]);
    u32x4 v[U];
    if (p0 + 256 * U <= pieces) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = in[p0 + u * 256 + threadIdx.x];
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t p = p0 + u * 256 + threadIdx.x;
        v[u] = u32x4{0, 0, 0, 0};
        if (p < pieces) v[u] = in[p];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) add_squares(v[u], f32, s);
    const uint64_t at = pieces * (f32 ? 4 : 8) + threadIdx.x;
    if (last && at < count) {
      const float a = f32 ? static_cast<const float*>(t.in[e])[at] : bf16_to_f32(static_cast<const uint16_t*>(t.in[e])[at]);
      s = __builtin_fma(static_cast<double>(a), static_cast<double>(a), s);
    }
  });
  s = group_total(s, part);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

// sqrt of the workgroups' sums, in every thread of a workgroup of 256
__device__ __forceinline__ double norm_of(const double* sums, int n, double (&part)[4]) {
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += 256) s += sums[i];
  return sqrt(group_total(s, part));
}
__global__ __launch_bounds__(256) void grad_norm_finish_kernel(const double* __restrict__ sums, int n, float* __restrict__ norm) {
  __shared__ double part[4];
  const double v = norm_of(sums, n, part);
  if (threadIdx.x == 0) norm[0] = static_cast<float>(v);
}

// Backwards through the chunks, so that what the norm has read last, and the caches still hold, is read first.
template <int U> __global__ __launch_bounds__(256) void grad_clip_kernel(GradTable t, const double* __restrict__ sums, int n, double largest, float* __restrict__ norm) {
  __shared__ double part[4];
  const double v = norm_of(sums, n, part), ratio = largest / (v + 1e-6);
  if (norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = static_cast<float>(v);
  // As m 2^e with m in [1/2, 1): a scale may lie below what 32 bits hold where the gradients are as large.  (NaN stays NaN.)
  int e = 0;
  const float m = ratio >= 1.0 ? 1.f : static_cast<float>(frexp(ratio, &e));
  if (ratio >= 1.0) e = 0;
  const auto scaled1 = [&](float x) __attribute__((always_inline)) { return __builtin_amdgcn_ldexpf(x * m, e); };
  const bool same = m == 1.f && e == 0;
  over_chunks<U>(t, t.first[t.n], true, [&](uint32_t which, bool f32, uint64_t p0, uint64_t pieces, uint64_t count, bool last) __attribute__((always_inline)) {
    if (same && t.in[which] == t.out[which]) return;
    const u32x4_any* in = static_cast<const u32x4_any*>(t.in[which]);
    u32x4_any* out = static_cast<u32x4_any*>(t.out[which]);
    auto scaled = [&](u32x4 x) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x[i] = f32 ? __float_as_uint(scaled1(__uint_as_float(x[i]))) : pack_bf16(scaled1(bf16lo(x[i])), scaled1(bf16hi(x[i])));
      return x;
    };
    u32x4 v[U];
    if (p0 + 256 * U <= pieces) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = in[p0 + u * 256 + threadIdx.x];
#pragma unroll
      for (int u = 0; u < U; ++u) out[p0 + u * 256 + threadIdx.x] = scaled(v[u]);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint64_t p = p0 + u * 256 + threadIdx.x;
        if (p < pieces) out[p] = scaled(in[p]);
      }
    }
    const uint64_t at = pieces * (f32 ? 4 : 8) + threadIdx.x;
    if (last && at < count) {
      if (f32) static_cast<float*>(t.out[which])[at] = scaled1(static_cast<const float*>(t.in[which])[at]);
      else static_cast<uint16_t*>(t.out[which])[at] = f32_to_bf16(scaled1(bf16_to_f32(static_cast<const uint16_t*>(t.in[which])[at])));
    }
  });
}

// ---- host ---------------------------------------------------------------------------------------------------------------------

int bytes_of(const moe_grad& g) { return g.type == MOE_TYPE_F32 ? 4 : 2; }
bool bad_grads(const moe_grad* g, int n, bool clip) {
  if (g == nullptr || n <= 0 || n > MAX_TENSORS) return true;
  for (int i = 0; i < n; ++i) {
    if ((g[i].type != MOE_TYPE_BF16 && g[i].type != MOE_TYPE_F32) || g[i].count < 0 || g[i].count > (1ll << 40)) return true;
    if (g[i].count == 0) continue;
    const uintptr_t odd = bytes_of(g[i]) - 1;
    if (g[i].in == nullptr || (reinterpret_cast<uintptr_t>(g[i].in) & odd) != 0) return true;
    if (clip && (g[i].out == nullptr || (reinterpret_cast<uintptr_t>(g[i].out) & odd) != 0)) return true;
  }
  return false;
}
// Whether some output lies over an input other than its own, or over another output: what is there would depend on who comes first.
struct Range { uintptr_t from, to; bool out; };
int overlap(const moe_grad* g, int n) {
  Range few[2 * 256];
  Range* r = n <= 256 ? few : new (std::nothrow) Range[2 * static_cast<size_t>(n)];
  if (r == nullptr) return MOE_ERR_INVALID;
  int m = 0;
  for (int i = 0; i < n; ++i) {
    if (g[i].count == 0) continue;
    const uintptr_t in = reinterpret_cast<uintptr_t>(g[i].in), out = reinterpret_cast<uintptr_t>(g[i].out), bytes = static_cast<uintptr_t>(g[i].count) * bytes_of(g[i]);
    r[m++] = {out, out + bytes, true};
    if (in != out) r[m++] = {in, in + bytes, false};
  }
  std::sort(r, r + m, [](const Range& a, const Range& b) { return a.from < b.from; });
  uintptr_t outs = 0, all = 0;                      // where those so far end
  int rc = MOE_OK;
  for (int i = 0; i < m; ++i) {
    if (r[i].from < (r[i].out ? all : outs)) { rc = MOE_ERR_INVALID; break; }
    if (r[i].to > all) all = r[i].to;
    if (r[i].out && r[i].to > outs) outs = r[i].to;
  }
  if (r != few) delete[] r;
  return rc;
}
// Pieces of 16 bytes that a thread takes of a chunk: four, or one where there would be too few chunks for all compute units.
constexpr int WIDE = 4;
constexpr long long FEW_PIECES = 2ll * GRAD_GROUPS * 256 * WIDE;

// f(table, chunks) for the tensors, as many at a time as a table holds
template <typename F> int over_tables(const moe_grad* g, int n, int u, F&& f) {
  GradTable t;
  t.n = 0;
  unsigned long long chunks = 0;
  for (int i = 0; i <= n; ++i) {
    if (i == n || t.n == TENSORS) {
      t.first[t.n] = static_cast<uint32_t>(chunks);
      if (t.n > 0 && f(t, static_cast<long long>(chunks)) != MOE_OK) return MOE_ERR_LAUNCH;
      t.n = 0;
      chunks = 0;
    }
    if (i == n || g[i].count == 0) continue;
    const unsigned long long count = g[i].count, pieces = count / (16 / bytes_of(g[i])), c = (pieces + 256 * u - 1) / (256 * u);
    t.in[t.n] = g[i].in;
    t.out[t.n] = g[i].out;
    t.count[t.n] = count << 1 | (g[i].type == MOE_TYPE_F32 ? 1 : 0);
    t.first[t.n++] = static_cast<uint32_t>(chunks);
    chunks += c > 0 ? c : 1;
  }
  return MOE_OK;
}
int run_grads(const moe_grad* g, int n, bool clip, double largest, float* norm, void* ws, size_t ws_bytes, hipStream_t s) {
  if (bad_grads(g, n, clip) || norm == nullptr || !moe_aligned16(norm) || ws == nullptr || !moe_aligned16(ws)) return MOE_ERR_INVALID;
  if (ws_bytes < moe_grad_norm_workspace_bytes(n)) return MOE_ERR_WORKSPACE;
  unsigned long long pieces = 0;
  for (int i = 0; i < n; ++i) pieces += static_cast<unsigned long long>(g[i].count) / (16 / bytes_of(g[i])) + 1;
  if (pieces > 1ull << 40) return MOE_ERR_INVALID;   // chunks are counted in 32 bits
  if (clip && overlap(g, n) != MOE_OK) return MOE_ERR_INVALID;
  const bool wide = pieces >= FEW_PIECES;
  double* const sums = static_cast<double*>(ws);
  int parts = 0;
  auto groups = [](long long chunks) { return static_cast<int>(chunks < GRAD_GROUPS ? chunks : GRAD_GROUPS); };
  int rc = over_tables(g, n, wide ? WIDE : 1, [&](const GradTable& t, long long chunks) {
    const dim3 grid(groups(chunks));
    if (wide) MOE_LAUNCH("grad_norm", grad_norm_kernel<WIDE>, grid, dim3(256), 0, s, t, sums + parts);
    else MOE_LAUNCH("grad_norm", grad_norm_kernel<1>, grid, dim3(256), 0, s, t, sums + parts);
    parts += grid.x;
    return moe_check_launch();
  });
  if (rc != MOE_OK) return rc;
  float* left = norm;                                // the first launch that knows the norm writes it
  if (clip) {
    rc = over_tables(g, n, wide ? WIDE : 1, [&](const GradTable& t, long long chunks) {
      const dim3 grid(groups(chunks));
      if (wide) MOE_LAUNCH("grad_clip", grad_clip_kernel<WIDE>, grid, dim3(256), 0, s, t, sums, parts, largest, left);
      else MOE_LAUNCH("grad_clip", grad_clip_kernel<1>, grid, dim3(256), 0, s, t, sums, parts, largest, left);
      left = nullptr;
      return moe_check_launch();
    });
  }
  if (rc != MOE_OK || left == nullptr) return rc;
  MOE_LAUNCH("grad_norm_finish", grad_norm_finish_kernel, dim3(1), dim3(256), 0, s, sums, parts, norm);
  return moe_check_launch();
}

}  // namespace

extern "C" size_t moe_grad_norm_workspace_bytes(int n) {
  if (n <= 0 || n > MAX_TENSORS) return 0;
  return static_cast<size_t>((n + TENSORS - 1) / TENSORS) * GRAD_GROUPS * sizeof(double);
}

extern "C" int moe_grad_norm(const moe_grad* grads, int n, float* norm, void* ws, size_t ws_bytes, void* stream) {
  return run_grads(grads, n, false, 0.0, norm, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int moe_grad_clip(const moe_grad* grads, int n, double largest, float* norm, void* ws, size_t ws_bytes, void* stream) {
  if (!(largest > 0.0) || !(largest < __builtin_inff())) return MOE_ERR_INVALID;
  return run_grads(grads, n, true, largest, norm, ws, ws_bytes, static_cast<hipStream_t>(stream));
}
