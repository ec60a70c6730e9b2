// The norm of all gradients of a model together, and their scaling to a largest norm:
//   norm = sqrt(sum over all tensors of g^2);   out = g min(1, largest / (norm + 1e-6))
// Bound by memory: one pass reads every gradient, the second reads it once more and writes it, as more than the caches hold has to be: 298 MB take 54 + 90 us (5.5 and
// 6.6 TB/s), 1.22 GB 203 + 430 (6.0 and 5.7; a large copy runs at 4.9).  Squares and their sums are in 64 bits, so that gradients of any
// size have a norm; each workgroup leaves its sum, and whoever needs the norm adds these up in one order: no atomics, the same bits every time.
#include <algorithm>
#include <new>
#include <type_traits>
#include "common.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
// (tensors may begin anywhere in a buffer of many: at multiples of their elements' size)
typedef __attribute__((ext_vector_type(4), aligned(2))) uint32_t u32x4_any;

// What a launch knows of its tensors comes with its arguments, so that nothing has to be copied to the device first, in a graph or out of it: at most 4 KB of them, and
// less where there are few.  A tensor's chunks are CHUNK bytes each but for the last.
constexpr int GRAD_THREADS = 256, GRAD_GROUPS = 2048;   // workgroups of a launch at most, each with its sum
constexpr int FEW_TENSORS = 24, NORM_TENSORS = 240, CLIP_TENSORS = 160;
constexpr int MAX_TENSORS = 1 << 20;
template <int CAP, bool CLIP> struct GradTable {
  const void* in[CAP];
  void* out[CLIP ? CAP : 1];
  uint32_t first[CAP + 1];                          // first chunk
  uint32_t last[CAP];                               // elements of the last chunk, and in the lowest bit whether they have 32 bits
  uint32_t n, each, more;                           // chunks of a workgroup: each, and one more for the first `more` of them
};
static_assert(sizeof(GradTable<NORM_TENSORS, false>) <= 3968 && sizeof(GradTable<CLIP_TENSORS, true>) <= 3968, "kernel arguments");

template <bool F32> __device__ __forceinline__ void add_squares(const u32x4& v, double (&s)[2]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (F32) {
      const double a = static_cast<double>(__uint_as_float(v[i]));
      s[i & 1] = __builtin_fma(a, a, s[i & 1]);
    } else {
      const double a = static_cast<double>(bf16lo(v[i])), b = static_cast<double>(bf16hi(v[i]));
      s[0] = __builtin_fma(a, a, s[0]);
      s[1] = __builtin_fma(b, b, s[1]);
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

// One chunk as a workgroup has it: U pieces of 16 bytes a thread, 256 apart, and an element behind the last whole piece.
template <int U> struct Chunk {
  const void* in;
  void* out;
  uint32_t pieces, tail;
  bool f32;
  u32x4 v[U];
  float extra;
};
// Calls use(chunk) for each of the workgroup's chunks, one after the other whatever tensors they belong to, the next one being requested before; from the last to the first
// if BACKWARDS.
template <int U, bool BACKWARDS, int CAP, bool CLIP, typename Use> __device__ __forceinline__ void over_chunks(const GradTable<CAP, CLIP>& t, Use&& use) {
  constexpr uint32_t WHOLE = GRAD_THREADS * U;
  const uint32_t b = blockIdx.x, c0 = b * t.each + (b < t.more ? b : t.more), n = t.each + (b < t.more ? 1 : 0);
  if (n == 0) return;
  uint32_t c = BACKWARDS ? c0 + n - 1 : c0, e = 0;
#pragma unroll
  for (uint32_t step = 128; step > 0; step /= 2)      // the last tensor whose first chunk is not behind c
    if (e + step < t.n && t.first[e + step] <= c) e += step;
  const auto request = [&](Chunk<U>& x) __attribute__((always_inline)) {
    const uint32_t first = t.first[e], last = t.last[e], at = c - first;
    x.f32 = (last & 1) != 0;
    const uint32_t per = x.f32 ? 4 : 8, count = c + 1 == t.first[e + 1] ? last >> 1 : WHOLE * per;
    x.pieces = count / per;
    x.tail = count % per;
    x.in = static_cast<const u32x4_any*>(t.in[e]) + static_cast<size_t>(at) * WHOLE;
    if constexpr (CLIP) x.out = static_cast<u32x4_any*>(t.out[e]) + static_cast<size_t>(at) * WHOLE;
    const u32x4_any* const p = static_cast<const u32x4_any*>(x.in);
    if (x.pieces == WHOLE) {
#pragma unroll
      for (int u = 0; u < U; ++u) x.v[u] = CLIP && U > 1 ? __builtin_nontemporal_load(p + u * GRAD_THREADS + threadIdx.x) : p[u * GRAD_THREADS + threadIdx.x];
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x.v[u] = u32x4{0, 0, 0, 0};
        if (u * GRAD_THREADS + threadIdx.x < x.pieces) x.v[u] = p[u * GRAD_THREADS + threadIdx.x];
      }
    }
    x.extra = 0.f;
    if (threadIdx.x < x.tail) {
      const uint32_t i = x.pieces * per + threadIdx.x;
      x.extra = x.f32 ? static_cast<const float*>(x.in)[i] : bf16_to_f32(static_cast<const uint16_t*>(x.in)[i]);
    }
  };
  const auto step = [&]() __attribute__((always_inline)) {
    if constexpr (BACKWARDS) { if (c-- == t.first[e]) --e; }
    else { if (++c == t.first[e + 1]) ++e; }
  };
  Chunk<U> one, two;
  request(one);
  for (uint32_t left = n;;) {
    if (--left == 0) { use(one); break; }
    step();
    request(two);
    use(one);
    if (--left == 0) { use(two); break; }
    step();
    request(one);
    use(two);
  }
}

template <int U, int CAP> __global__ __launch_bounds__(GRAD_THREADS) void grad_norm_kernel(GradTable<CAP, false> t, double* __restrict__ sums) {
  __shared__ double part[4];
  double s[2] = {0.0, 0.0};
  over_chunks<U, false>(t, [&](const Chunk<U>& x) __attribute__((always_inline)) {
    if (x.f32) {
#pragma unroll
      for (int u = 0; u < U; ++u) add_squares<true>(x.v[u], s);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) add_squares<false>(x.v[u], s);
    }
    const double a = x.extra;
    s[0] = __builtin_fma(a, a, s[0]);
  });
  const double total = group_total(s[0] + s[1], part);
  if (threadIdx.x == 0) sums[blockIdx.x] = total;
}

// sqrt of the workgroups' sums, in every thread of a workgroup of 256
__device__ __forceinline__ double norm_of(const double* sums, int n, double (&part)[4]) {
  double s = 0.0;
#pragma unroll 8
  for (int i = threadIdx.x; i < n; i += GRAD_THREADS) s += sums[i];
  return sqrt(group_total(s, part));
}
__global__ __launch_bounds__(GRAD_THREADS) void grad_norm_finish_kernel(const double* __restrict__ sums, int n, float* __restrict__ norm, double* __restrict__ total) {
  __shared__ double part[4];
  const double v = norm_of(sums, n, part);
  if (threadIdx.x == 0) {
    norm[0] = static_cast<float>(v);
    total[0] = v * v;
  }
}

// Each workgroup goes backwards through the chunks that it had for the norm, so that what the caches still hold is read first (1.22 GB: 445 -> 430 us).
// What it writes is past what the caches hold anyway, and so is what it reads for the last time: with non-temporal stores the next pass reads from memory without
// waiting for the writes of this one, and so does the norm (us, ordinary / non-temporal: norm of 298 MB in 126 tensors 87 / 54, of 1.22 GB in 8 245 / 203, clip 95 / 91 and
// 460 / 441).  Where there is a megabyte or two, they stay ordinary: the update that comes next finds them in the caches.
template <int U, int CAP> __global__ __launch_bounds__(GRAD_THREADS) void grad_clip_kernel(GradTable<CAP, true> t, const double* __restrict__ sums, int n_sums, double largest,
                                                                                           float* __restrict__ norm) {
  __shared__ double part[4];
  const double v = norm_of(sums, n_sums, part), ratio = largest / (v + 1e-6);
  if (norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = static_cast<float>(v);
  // As m 2^e with m in [1/2, 1): a scale may lie below what 32 bits hold where the gradients are as large.  (NaN stays NaN.)
  int exponent = 0;
  const float m = ratio >= 1.0 ? 1.f : static_cast<float>(frexp(ratio, &exponent));
  if (ratio >= 1.0) exponent = 0;
  const bool same = m == 1.f && exponent == 0;
  const auto scaled = [&](float x) __attribute__((always_inline)) { return __builtin_amdgcn_ldexpf(x * m, exponent); };
  over_chunks<U, true>(t, [&](const Chunk<U>& x) __attribute__((always_inline)) {
    if (same && x.in == x.out) return;
    u32x4_any* const o = static_cast<u32x4_any*>(x.out);
    const auto put = [&](auto f32, bool whole) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        u32x4 v = x.v[u];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (decltype(f32)::value) v[i] = __float_as_uint(scaled(__uint_as_float(v[i])));
          else v[i] = pack_bf16(scaled(bf16lo(v[i])), scaled(bf16hi(v[i])));
        }
        if (!whole && u * GRAD_THREADS + threadIdx.x >= x.pieces) continue;
        if constexpr (U > 1) __builtin_nontemporal_store(v, o + u * GRAD_THREADS + threadIdx.x);
        else o[u * GRAD_THREADS + threadIdx.x] = v;
      }
    };
    const bool whole = x.pieces == GRAD_THREADS * U;
    if (x.f32) { if (whole) put(std::true_type{}, true); else put(std::true_type{}, false); }
    else { if (whole) put(std::false_type{}, true); else put(std::false_type{}, false); }
    if (threadIdx.x < x.tail) {
      const uint32_t i = x.pieces * (x.f32 ? 4 : 8) + threadIdx.x;
      if (x.f32) static_cast<float*>(x.out)[i] = scaled(x.extra);
      else static_cast<uint16_t*>(x.out)[i] = f32_to_bf16(scaled(x.extra));
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
// Whether some output lies over an input other than its own, or over another output (the norm and the workspace are such): what is there would depend on who comes first.
struct Range { uintptr_t from, to; bool out; };
// The norm alone: its inputs are read while the workgroups' sums are written.
bool norm_overlaps(const moe_grad* g, int n, const float* norm, const void* ws, size_t ws_bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(norm), sums = reinterpret_cast<uintptr_t>(ws);
  const auto meet = [](uintptr_t a, uintptr_t a_bytes, uintptr_t b, uintptr_t b_bytes) { return a < b + b_bytes && b < a + a_bytes; };
  bool some = meet(at, sizeof(float), sums, ws_bytes);
  for (int i = 0; i < n; ++i) {
    const uintptr_t in = reinterpret_cast<uintptr_t>(g[i].in), bytes = static_cast<uintptr_t>(g[i].count) * bytes_of(g[i]);
    some |= g[i].count > 0 && (meet(in, bytes, at, sizeof(float)) || meet(in, bytes, sums, ws_bytes));
  }
  return some;
}
int overlap(const moe_grad* g, int n, const float* norm, const void* ws, size_t ws_bytes) {
  Range few[2 * 256 + 2];
  Range* r = n <= 256 ? few : new (std::nothrow) Range[2 * static_cast<size_t>(n) + 2];
  if (r == nullptr) return MOE_ERR_INVALID;
  const uintptr_t at[2] = {reinterpret_cast<uintptr_t>(norm), reinterpret_cast<uintptr_t>(ws)};
  r[0] = {at[0], at[0] + sizeof(float), true};
  r[1] = {at[1], at[1] + ws_bytes, true};
  int m = 2;
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
constexpr long long FEW_PIECES = 1ll * GRAD_GROUPS * GRAD_THREADS * WIDE;

int tables_for(int n, int cap) { return (n + cap - 1) / cap; }
int groups_for(unsigned long long chunks) { return chunks < GRAD_GROUPS ? static_cast<int>(chunks > 0 ? chunks : 1) : GRAD_GROUPS; }
// f(table, chunks) for all tensors, CAP of them at a time or, if that takes several tables, as many in each
template <int U, int CAP, bool CLIP, typename F> int over_tables(const moe_grad* g, int n, F&& f) {
  const int tables = tables_for(n, CAP), each = (n + tables - 1) / tables;
  GradTable<CAP, CLIP> t;
  for (int at = 0; at < n; at += each) {
    unsigned long long chunks = 0;
    t.n = 0;
    for (int i = at; i < n && i < at + each; ++i) {
      if (g[i].count == 0) continue;
      const unsigned long long count = g[i].count, chunk = static_cast<unsigned long long>(GRAD_THREADS) * U * (16 / bytes_of(g[i])), c = (count + chunk - 1) / chunk;
      t.in[t.n] = g[i].in;
      if constexpr (CLIP) t.out[t.n] = g[i].out;
      t.last[t.n] = static_cast<uint32_t>(count - (c - 1) * chunk) << 1 | (g[i].type == MOE_TYPE_F32 ? 1 : 0);
      t.first[t.n++] = static_cast<uint32_t>(chunks);
      chunks += c;
    }
    t.first[t.n] = static_cast<uint32_t>(chunks);
    const unsigned long long groups = groups_for(chunks);
    t.each = static_cast<uint32_t>(chunks / groups);
    t.more = static_cast<uint32_t>(chunks % groups);
    if (f(t, static_cast<int>(groups)) != MOE_OK) return MOE_ERR_LAUNCH;
  }
  return MOE_OK;
}
struct GradCall {
  const moe_grad* g;
  int n;
  double* sums;
  double largest;
  float* norm;
  hipStream_t s;
};
template <int U, int CAP> int launch_norms(const GradCall& c, int& parts) {
  return over_tables<U, CAP, false>(c.g, c.n, [&](const GradTable<CAP, false>& t, int groups) {
    MOE_LAUNCH("grad_norm", (grad_norm_kernel<U, CAP>), dim3(groups), dim3(GRAD_THREADS), 0, c.s, t, c.sums + parts);
    parts += groups;
    return moe_check_launch();
  });
}
template <int U, int CAP> int launch_clips(const GradCall& c, int parts) {
  float* norm = c.norm;                              // the first launch writes it, if it is to be written
  return over_tables<U, CAP, true>(c.g, c.n, [&](const GradTable<CAP, true>& t, int groups) {
    MOE_LAUNCH("grad_clip", (grad_clip_kernel<U, CAP>), dim3(groups), dim3(GRAD_THREADS), 0, c.s, t, c.sums, parts, c.largest, norm);
    norm = nullptr;
    return moe_check_launch();
  });
}
int run_grads(const moe_grad* g, int n, bool clip, double largest, float* norm, void* ws, size_t ws_bytes, hipStream_t s) {
  if (bad_grads(g, n, clip) || norm == nullptr || !moe_aligned16(norm) || ws == nullptr || !moe_aligned16(ws)) return MOE_ERR_INVALID;
  if (ws_bytes < moe_grad_norm_workspace_bytes(n)) return MOE_ERR_WORKSPACE;
  unsigned long long pieces = 0;
  for (int i = 0; i < n; ++i) pieces += static_cast<unsigned long long>(g[i].count) / (16 / bytes_of(g[i])) + 1;
  if (pieces > 1ull << 40) return MOE_ERR_INVALID;   // chunks are counted in 32 bits
  const size_t used = moe_grad_norm_workspace_bytes(n);
  if (clip ? overlap(g, n, norm, ws, used) != MOE_OK : norm_overlaps(g, n, norm, ws, used)) return MOE_ERR_INVALID;
  const bool wide = pieces >= FEW_PIECES, few = n <= FEW_TENSORS;
  GradCall c{g, n, static_cast<double*>(ws), largest, norm, s};
  int parts = 0;
  int rc = wide ? (few ? launch_norms<WIDE, FEW_TENSORS>(c, parts) : launch_norms<WIDE, NORM_TENSORS>(c, parts))
                : (few ? launch_norms<1, FEW_TENSORS>(c, parts) : launch_norms<1, NORM_TENSORS>(c, parts));
  if (rc != MOE_OK) return rc;
  // Every workgroup that scales adds the sums up by itself, unless there are more of them than that is worth another launch for (us from a graph, by themselves / by a
  // launch: 8 bf16 tensors of 4 million 33 / 44; 5 tables, 1000 of 150001, 184 / 147; 11 tables, 2500 of them, 706 / 363 to 507).
  double* const total = c.sums + static_cast<size_t>(tables_for(n, few ? FEW_TENSORS : NORM_TENSORS)) * GRAD_GROUPS;
  if (!clip || parts > 2 * GRAD_GROUPS) {
    MOE_LAUNCH("grad_norm_finish", grad_norm_finish_kernel, dim3(1), dim3(GRAD_THREADS), 0, s, c.sums, parts, norm, total);
    if ((rc = moe_check_launch()) != MOE_OK || !clip) return rc;
    c.sums = total;
    c.norm = nullptr;
    parts = 1;
  }
  return wide ? (few ? launch_clips<WIDE, FEW_TENSORS>(c, parts) : launch_clips<WIDE, CLIP_TENSORS>(c, parts))
              : (few ? launch_clips<1, FEW_TENSORS>(c, parts) : launch_clips<1, CLIP_TENSORS>(c, parts));
}

}  // namespace

extern "C" size_t moe_grad_norm_workspace_bytes(int n) {
  if (n <= 0 || n > MAX_TENSORS) return 0;
  return static_cast<size_t>(tables_for(n, n <= FEW_TENSORS ? FEW_TENSORS : NORM_TENSORS)) * GRAD_GROUPS * sizeof(double) + 16;
}

extern "C" int moe_grad_norm(const moe_grad* grads, int n, float* norm, void* ws, size_t ws_bytes, void* stream) {
  return run_grads(grads, n, false, 0.0, norm, ws, ws_bytes, static_cast<hipStream_t>(stream));
}

extern "C" int moe_grad_clip(const moe_grad* grads, int n, double largest, float* norm, void* ws, size_t ws_bytes, void* stream) {
  if (!(largest > 0.0) || !(largest < __builtin_inff())) return MOE_ERR_INVALID;
  return run_grads(grads, n, true, largest, norm, ws, ws_bytes, static_cast<hipStream_t>(stream));
}
