// Joins the strips of the vocabulary head's logits into log probabilities, entropies and likeliest alternatives.
//
// With o_j the distance of logit j from the largest, over the temperature, R the sum of exp(-o) over all columns but the largest's and Q that of o exp(-o):
//   log p of the largest = -log(1 + R);   of any other -log(1 + R) - o;   entropy = log(1 + R) + Q / (1 + R)
// All terms are positive: a token that the model is sure of keeps the digits of its log probability and entropy, which a difference of the two usual sums would not.
//
// Which of two logits is larger is told in 64 bits (products of two bf16 numbers are exact in 32 bits, their sums in 64 are off by 1e-16): the chain of additions of the
// matrix product would put one in some 10^4 alternatives in the wrong place.  So the K + SCORE_SPARE largest by the product are formed anew, a row of W each, and ordered by that.
// Candidates: the columns of a lane of the product (16 or 32) have their largest apart.  None of the C largest logits lies in another lane's columns than
// those with the C largest of these; where the second largest of such a lane may be among them too, all of its columns are candidates.  That is one lane in six
// tokens for 24 of 50304 columns, and no more than C of them whatever the logits are.
#include <type_traits>
#include "head_score.h"

namespace {

constexpr int SCORE_CANDIDATES = 512, SCORE_FEW = 256, SCORE_SOME = 1024;
constexpr int SCORE_ROW = 1 << 20;                 // workgroups of a row of the grid (a launch may have 2^32 threads in a row)

__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) != 0 ? 0x80000000u : 0xFFFFFFFFu)); }
// Sums of 2^t and t 2^t relative to 2^e, e a whole number.
struct ScoreSum {
  float e = -3.0e38f, sum = 0.f, moment = 0.f;
  __device__ __forceinline__ void raise(float n) {                        // n >= e
    const float f = __builtin_amdgcn_exp2f(e - n);
    moment = f * __builtin_fmaf(sum, e - n, moment);
    sum *= f;
    e = n;
  }
  __device__ __forceinline__ void add(float E, float s, float m) {        // E <= e
    const float g = __builtin_amdgcn_exp2f(E - e);
    sum = __builtin_fmaf(g, s, sum);
    moment = __builtin_fmaf(g, __builtin_fmaf(s, E - e, m), moment);
  }
  __device__ __forceinline__ void add_logit(float z, float c1) {          // z c1 <= e
    const float t = __builtin_fmaf(z, c1, -e), s = __builtin_amdgcn_exp2f(t);
    sum += s;
    moment = __builtin_fmaf(s, t, moment);
  }
};

// Logits of N columns in 64 bits by each LANES lanes of a wave; AHEAD pieces of each row requested together.
template <int LANES, int N, int AHEAD>
__device__ __forceinline__ void exact_logits(const moe_bf16* x, const moe_bf16* W, int d, const int (&col)[N], double (&z)[N]) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u4;
  constexpr int STEP = LANES * 8;
  const moe_bf16* row[N];
#pragma unroll
  for (int k = 0; k < N; ++k) { z[k] = 0.0; row[k] = W + static_cast<size_t>(col[k]) * d; }
  for (int c0 = threadIdx.x % LANES * 8; c0 < d; c0 += AHEAD * STEP) {
    u4 p[AHEAD], w[AHEAD][N];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int c = c0 + u * STEP < d ? c0 + u * STEP : c0;
      p[u] = *reinterpret_cast<const u4*>(x + c);
#pragma unroll
      for (int k = 0; k < N; ++k) w[u][k] = *reinterpret_cast<const u4*>(row[k] + c);
    }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (c0 + u * STEP >= d) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double lo = bf16lo(p[u][i]), hi = bf16hi(p[u][i]);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          z[k] = __builtin_fma(lo, static_cast<double>(bf16lo(w[u][k][i])), z[k]);
          z[k] = __builtin_fma(hi, static_cast<double>(bf16hi(w[u][k][i])), z[k]);
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const auto from = [&](auto ctrl) __attribute__((always_inline)) {
      const uint64_t b = __builtin_bit_cast(uint64_t, z[k]);
      return __builtin_bit_cast(double, static_cast<uint64_t>(dpp_u32<decltype(ctrl)::value>(static_cast<uint32_t>(b >> 32))) << 32 | dpp_u32<decltype(ctrl)::value>(static_cast<uint32_t>(b)));
    };
    z[k] += from(std::integral_constant<int, 0xB1>{});                     // (the steps of group_reduce)
    z[k] += from(std::integral_constant<int, 0x4E>{});
    z[k] += from(std::integral_constant<int, 0x141>{});
    z[k] += from(std::integral_constant<int, 0x140>{});
#pragma unroll
    for (int i = 16; i < LANES; i *= 2) z[k] += __shfl_xor(z[k], i);
  }
}
__device__ __forceinline__ int64_t ordered_i64(double v) {
  const int64_t b = __builtin_bit_cast(int64_t, v == 0.0 ? 0.0 : v);          // (-0 and +0 are equal)
  return b >= 0 ? b : b ^ 0x7FFFFFFFFFFFFFFFll;
}

// Maximum over groups of G threads (a power of two up to a wave), in all of them.
template <int G> __device__ __forceinline__ uint64_t group_most(uint64_t v) {
#pragma unroll
  for (int i = 1; i < G; i *= 2) {
    const uint64_t o = __shfl_xor(v, i);
    v = o > v ? o : v;
  }
  return v;
}

constexpr uint32_t NONE = 0xFF800000u;              // -infinity
// What the sums over all columns but the largest come to.  The largest by the product is what they leave out: the formulas hold whether it is the largest in 64 bits
// or next to it.  NaN where a logit is no number or infinite, and where a scale of 2^30 or more leaves its exponent without digits.
struct ScoreResult { double log_1R; float entropy; };
__device__ __forceinline__ ScoreResult result_of(const ScoreSum& all, bool there, double z_top, float c1) {
  const double from = static_cast<double>(all.e) - z_top * static_cast<double>(c1);
  const bool alone = all.e == -3.0e38f;                                    // no other column
  const bool fine = there && fabs(z_top * static_cast<double>(c1)) < 0x1p30 && (alone || fabsf(all.e) < 0x1p30f);
  const double whole = fmax(rint(from), -10000.0);
  const float scale = fine ? __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(static_cast<float>(from - whole)), static_cast<int>(whole)) : __builtin_nanf("");
  const float R = alone ? 0.f : all.sum * scale;
  const float Q = alone ? 0.f : -0.693147180559945309f * scale * __builtin_fmaf(static_cast<float>(from), all.sum, all.moment);
  const float log_1R = fine ? log1pf(R) : __builtin_nanf("");
  return {static_cast<double>(log_1R), log_1R + Q / (1.f + R)};
}
__device__ __forceinline__ void put_scores(const ScoreJoinArgs& a, int t, const ScoreResult& r, bool at_top, double z, double z_top) {
  a.logp[t] = at_top ? -static_cast<float>(r.log_1R) : static_cast<float>((z - z_top) * a.over_tau - r.log_1R);
  a.entropy[t] = r.entropy;
  a.lse[t] = static_cast<float>(z_top * a.over_tau + r.log_1R);
}

// Without alternatives: a wave for each token, or (FEW) four (V 50304, us, one / four: 256 tokens 6.4 / 5.5, 1000 8.0 / 8.1, 4000 15 / 21; 8192 23).  HALF: columns of a strip.
// SURES: for rows of the backward pass.
template <int HALF, bool FEW, bool SURES> __global__ __launch_bounds__(256) void head_score_kernel(ScoreJoinArgs a) {
  constexpr int AT_ONCE = 4, STEP = FEW ? 4 * MOE_WAVE : MOE_WAVE;
  typedef __attribute__((ext_vector_type(4))) uint32_t u4;
  __shared__ uint64_t tops[FEW ? 4 : 1];
  __shared__ float parts[FEW ? 4 : 1][3];
  const int lane = threadIdx.x % MOE_WAVE, wave = threadIdx.x / MOE_WAVE, group = blockIdx.y * SCORE_ROW + blockIdx.x;
  const int at = __builtin_amdgcn_readfirstlane(FEW ? group : group * 4 + wave);
  if (at >= a.T || (SURES && at >= a.sure_rows[0])) return;
  const int t = SURES ? a.row_token[at] : at, y = a.target[t];
  if (y < 0 || y >= a.V) {
    if (lane == 0) { a.logp[t] = 0.f; a.entropy[t] = 0.f; a.lse[t] = 0.f; }
    return;
  }
  const int row = !SURES && a.control != nullptr ? a.token_row[t] : at;
  const u4* const strip = static_cast<const u4*>(a.part) + static_cast<size_t>(row) * a.strips;
  const float c1 = a.c1;
  uint64_t best = 0;
  ScoreSum total;
  for (int s0 = FEW ? threadIdx.x : lane; s0 < a.strips; s0 += AT_ONCE * STEP) {
    u4 x[AT_ONCE];
    float E[AT_ONCE], most = total.e;
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int s = s0 + i * STEP;
      x[i] = u4{NONE, 0, 0, 0};
      if (s < a.strips) x[i] = strip[s];
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      E[i] = x[i][0] == NONE ? total.e : ceilf(__uint_as_float(x[i][0]) * c1);
      most = fmaxf(most, E[i]);
    }
    total.raise(most);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const float sum = __uint_as_float(x[i][2]);
      total.add(x[i][0] == NONE && sum == 0.f ? total.e : E[i], sum, __uint_as_float(x[i][3]));
      const int col = (s0 + i * STEP) * HALF + static_cast<int>(x[i][1]);
      const uint64_t key = x[i][0] == NONE ? 0 : static_cast<uint64_t>(ordered_u32(x[i][0])) << 32 | ~static_cast<uint32_t>(col), less = key < best ? key : best;
      best = key < best ? best : key;
      if (less != 0) total.add_logit(from_ordered(static_cast<uint32_t>(less >> 32)), c1);
    }
  }
  uint64_t top_key = group_most<MOE_WAVE>(best);
  if constexpr (FEW) {
    if (lane == 0) tops[wave] = top_key;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) top_key = tops[w] > top_key ? tops[w] : top_key;
  }
  if (best != top_key && best != 0) total.add_logit(from_ordered(static_cast<uint32_t>(best >> 32)), c1);
  total.raise(group_max<MOE_WAVE>(total.e));
  total.sum = group_sum<MOE_WAVE>(total.sum);
  total.moment = group_sum<MOE_WAVE>(total.moment);
  if constexpr (FEW) {
    if (lane == 0) { parts[wave][0] = total.e; parts[wave][1] = total.sum; parts[wave][2] = total.moment; }
    __syncthreads();
    if (wave != 0) return;
    total = ScoreSum{};
#pragma unroll
    for (int w = 0; w < 4; ++w) total.e = fmaxf(total.e, parts[w][0]);
#pragma unroll
    for (int w = 0; w < 4; ++w) total.add(parts[w][0], parts[w][1], parts[w][2]);
  }
  const int top_col = top_key != 0 ? static_cast<int>(~__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(top_key))) : y;
  const int col[2] = {top_col, y};
  double z[2];
  exact_logits<MOE_WAVE, 2, 4>(a.x + static_cast<size_t>(t) * a.d, a.W, a.d, col, z);
  if (lane != 0) return;
  const ScoreResult r = result_of(total, top_key != 0, z[0], c1);
  if constexpr (SURES) reinterpret_cast<float*>(a.of_row + row)[3] = static_cast<float>(r.log_1R * -1.4426950408889634);
  else put_scores(a, t, r, y == top_col, z[1], z[0]);
}

// put(i, number of k with above(k, i)) for i and k below n, sixteen threads to an i.
template <int THREADS, typename Above, typename Put> __device__ __forceinline__ void ranked(int n, Above&& above, Put&& put) {
  const int l16 = threadIdx.x % 16;
  for (int i = threadIdx.x / 16; i - static_cast<int>(threadIdx.x / 16) < n; i += THREADS / 16) {
    uint32_t count = 0;
    if (i < n) for (int k = l16; k < n; k += 16) count += above(k, i) ? 1 : 0;
    count = group_reduce<16>(count, [](uint32_t u, uint32_t v) __attribute__((always_inline)) { return u + v; });
    if (i < n && l16 == 0) put(i, static_cast<int>(count));
  }
}

// The logits of columns[0 .. m], in 64 bits.  Sixteen lanes take a row of W, or, where there are few tokens or (TWO) rows and these are long, a wave: one latency then instead of several.
template <int THREADS, bool TWO> __device__ __forceinline__ void form_exact(const moe_bf16* x, const moe_bf16* W, int d, const int32_t* columns, double* exact, int m) {
  const int tid = threadIdx.x, wave = tid / MOE_WAVE;
  const auto form = [&](auto lanes, auto at_once, auto ahead) __attribute__((always_inline)) {
    constexpr int LANES = decltype(lanes)::value, N = decltype(at_once)::value, SETS = THREADS / LANES;
    const int set = tid / LANES;
    for (int i = 0; i + wave * (MOE_WAVE / LANES) <= m; i += SETS * N) {
      int col[N];
      double z[N];
#pragma unroll
      for (int k = 0; k < N; ++k) col[k] = columns[i + k * SETS + set < m ? i + k * SETS + set : m];
      exact_logits<LANES, N, decltype(ahead)::value>(x, W, d, col, z);
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (tid % LANES == 0 && i + k * SETS + set <= m) exact[i + k * SETS + set] = z[k];
    }
  };
  constexpr bool FEW = THREADS > 256;
  if ((FEW || TWO) && d > 512) form(std::integral_constant<int, MOE_WAVE>{}, std::integral_constant<int, 2>{}, std::integral_constant<int, 4>{});
  else form(std::integral_constant<int, 16>{}, std::integral_constant<int, FEW ? 1 : 2>{}, std::integral_constant<int, 4>{});
}
// The K largest of m of these, in the order of their logits, of equal ones the lower column first.
template <int THREADS>
__device__ __forceinline__ void put_alternatives(const ScoreJoinArgs& a, int t, const ScoreResult& r, const int32_t* columns, const double* exact, int m, int top_col, double z_top) {
  const size_t out = static_cast<size_t>(t) * a.K;
  for (int k = m + threadIdx.x; k < a.K; k += THREADS) {                   // (logits of -infinity: columns that are not there)
    a.ids[out + k] = -1;
    a.top[out + k] = __builtin_nanf("");
  }
  ranked<THREADS>(m, [&](int k, int i) __attribute__((always_inline)) {
    const int64_t one = ordered_i64(exact[k]), two = ordered_i64(exact[i]);
    return one > two || (one == two && columns[k] < columns[i]);
  }, [&](int i, int above) __attribute__((always_inline)) {
    if (above >= a.K) return;
    const bool there = exact[i] != -static_cast<double>(__builtin_inff());
    a.ids[out + above] = there ? columns[i] : -1;
    a.top[out + above] = !there ? __builtin_nanf("") : columns[i] == top_col ? -static_cast<float>(r.log_1R) : static_cast<float>((exact[i] - z_top) * a.over_tau - r.log_1R);
  });
}

// From the logits themselves: a thread has PIECES times four of them in registers.  LISTS: with alternatives.
template <int THREADS, int PIECES, bool LISTS> __global__ __launch_bounds__(THREADS) void head_score_whole_kernel(ScoreJoinArgs a) {
  // Groups of threads have 4, 8 or 16 columns side by side, and there are at least as many groups as logits are wanted; where fewer of them have any, all columns are
  // candidates.
  constexpr int WAVES = THREADS / MOE_WAVE, SIZE = THREADS <= 128 ? 1 : THREADS == 256 ? 2 : 4, GROUPS = THREADS / SIZE, WANTED = score_wanted(SCORE_MAX_K);
  constexpr int CANDIDATES = WANTED * SIZE * 4;
  __shared__ uint64_t keys[GROUPS], found[CANDIDATES], s_top, s_least;
  __shared__ double exact[WANTED + 1];
  __shared__ int32_t columns[WANTED + 1];
  __shared__ float part[WAVES][2];
  __shared__ int s_found;
  const int tid = threadIdx.x, lane = tid % MOE_WAVE, wave = tid / MOE_WAVE, K = a.K, wanted = score_wanted(K);
  const int t = blockIdx.y * SCORE_ROW + blockIdx.x;
  if (t >= a.T) return;
  const int y = a.target[t];
  if (y < 0 || y >= a.V) {
    if (tid == 0) { a.logp[t] = 0.f; a.entropy[t] = 0.f; a.lse[t] = 0.f; }
    for (int k = tid; k < K; k += THREADS) { a.ids[static_cast<size_t>(t) * K + k] = -1; a.top[static_cast<size_t>(t) * K + k] = 0.f; }
    return;
  }
  const int row = a.control != nullptr ? a.token_row[t] : t, ld = score_ld(a.V);
  const float* const z_row = static_cast<const float*>(a.part) + static_cast<size_t>(row) * ld;
  const float c1 = a.c1;
  float z[PIECES][4];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int c = (p * THREADS + tid) * 4;
    f32x4_t v = {};
    if (c < ld) v = *reinterpret_cast<const f32x4_t*>(z_row + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) z[p][i] = c + i < a.V ? v[i] : -__builtin_inff();
  }
  for (int part = 1; part < a.parts; ++part) {
    const float* const more = z_row + static_cast<size_t>(part) * a.T * ld;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int c = (p * THREADS + tid) * 4;
      f32x4_t v = {};
      if (c < ld) v = *reinterpret_cast<const f32x4_t*>(more + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) if (c + i < a.V) z[p][i] += v[i];
    }
  }
  // (as in the other kernel; of 0 and -0 either may be called the larger, the order in 64 bits knows no difference)
  const auto key_of = [&](int p, int i) __attribute__((always_inline)) -> uint64_t {
    const uint32_t bits = __float_as_uint(z[p][i]);
    return bits == NONE ? 0 : static_cast<uint64_t>(ordered_u32(bits)) << 32 | ~static_cast<uint32_t>((p * THREADS + tid) * 4 + i);
  };
  uint64_t best = 0;
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) { const uint64_t k = key_of(p, i); best = k > best ? k : best; }
  if (tid == 0) { s_top = s_least = 0; s_found = 0; }
  const uint64_t of_group = group_most<LISTS ? SIZE : MOE_WAVE>(best);
  uint64_t top_key = 0, least = 0;
  if constexpr (LISTS) {
    if (tid % SIZE == 0) keys[tid / SIZE] = of_group;
    __syncthreads();
    ranked<THREADS>(GROUPS, [&](int k, int i) __attribute__((always_inline)) { return keys[k] > keys[i]; }, [&](int i, int above) __attribute__((always_inline)) {
      if (above == 0 && keys[i] != 0) s_top = keys[i];
      if (above == wanted - 1 && keys[i] != 0) s_least = keys[i];
    });
    __syncthreads();
    top_key = s_top;
    least = s_least;
  } else {
    if (lane == 0) keys[wave] = of_group;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top_key = keys[w] > top_key ? keys[w] : top_key;
  }
  const int top_col = static_cast<int>(~static_cast<uint32_t>(top_key));
  const float most = from_ordered(static_cast<uint32_t>(top_key >> 32)), e = ceilf(most * c1);
  float sum = 0.f, moment = 0.f;
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = (p * THREADS + tid) * 4 + i;
      const float x = __builtin_elementwise_maximum(__builtin_fmaf(z[p][i], c1, -e), -1000.f), s = col == top_col ? 0.f : __builtin_amdgcn_exp2f(x);
      sum += s;
      moment = __builtin_fmaf(s, x, moment);
      if constexpr (LISTS) {
        const uint64_t key = key_of(p, i);
        if (key >= least && key != 0) {
          const int at = atomicAdd(&s_found, 1);
          if (at < CANDIDATES) found[at] = key;
        }
      }
    }
  sum = group_sum<MOE_WAVE>(sum);
  moment = group_sum<MOE_WAVE>(moment);
  if (lane == 0) { part[wave][0] = sum; part[wave][1] = moment; }
  __syncthreads();
  int m = LISTS ? s_found : top_key != 0;
  if (!LISTS) {
    if (tid == 0) columns[0] = top_col;
  } else if (m <= CANDIDATES) {
    ranked<THREADS>(m, [&](int k, int i) __attribute__((always_inline)) { return found[k] > found[i]; }, [&](int i, int above) __attribute__((always_inline)) {
      if (above < wanted) columns[above] = static_cast<int>(~static_cast<uint32_t>(found[i]));
    });
    m = m < wanted ? m : wanted;
  } else {
    // (large logits in few threads: one after the other)
    m = 0;
    for (uint64_t last = ~0ull; m < wanted; ++m) {
      uint64_t next = 0;
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) { const uint64_t k = key_of(p, i); next = k < last && k > next ? k : next; }
      next = group_most<MOE_WAVE>(next);
      __syncthreads();
      if (lane == 0) keys[wave] = next;
      __syncthreads();
      uint64_t whole = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) whole = keys[w] > whole ? keys[w] : whole;
      if (whole == 0) break;
      if (tid == 0) columns[m] = static_cast<int>(~static_cast<uint32_t>(whole));
      last = whole;
    }
  }
  if (tid == 0) columns[m] = y;
  __syncthreads();
  form_exact<THREADS, !LISTS>(a.x + static_cast<size_t>(t) * a.d, a.W, a.d, columns, exact, m);
  __syncthreads();
  ScoreSum all;
  all.e = e;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) { all.sum += part[w][0]; all.moment += part[w][1]; }
  const double z_top = exact[0];                                           // (columns[0] is top_col)
  const ScoreResult r = result_of(all, top_key != 0, z_top, c1);
  if (tid == 0) put_scores(a, t, r, y == top_col, exact[m], z_top);
  if constexpr (LISTS) put_alternatives<THREADS>(a, t, r, columns, exact, m, top_col, z_top);
}

// With alternatives: a workgroup of THREADS for each token, 1024 where there are few (d 2048, V 50304, 20 alternatives, us, 256 / 1024: 1 token 18.5 / 12.7, 256 tokens
// 31.6 / 20.5, 600 tokens 35 / 41; the whole call 257 to 512 tokens 111 / 112.5 to 142 / 140.5; 300 tokens, d 128, V 20000, 4 alternatives 24 / 29, d 512, V 32003, 64 83 / 65).  HALF: columns of a strip.  3074 tokens take 95 to 107 us, most of it for some 30 rows of W each, 390 MB at 4 TB/s.
template <int HALF, int THREADS>
__global__ __launch_bounds__(THREADS) void head_score_join_kernel(ScoreJoinArgs a) {
  constexpr int GROUPS = 256, WAVES = THREADS / MOE_WAVE, AT_ONCE = THREADS > 256 ? 4 : 8, STEP = THREADS / 4;
  extern __shared__ double exact[];
  __shared__ uint64_t keys[GROUPS], found[SCORE_CANDIDATES], chosen[score_wanted(SCORE_MAX_K)], s_top, s_least;
  __shared__ uint32_t found_next[SCORE_CANDIDATES], chosen_next[score_wanted(SCORE_MAX_K)];
  __shared__ float part[WAVES][3];
  __shared__ int s_found, s_columns, s_top_at;
  __shared__ uint32_t s_border;
  constexpr uint32_t LOW = HALF / 4 - 1;
  constexpr uint32_t LEAST = 0x00800000u;                                 // the order of the lowest number
  const int tid = threadIdx.x, lane = tid % MOE_WAVE, wave = tid / MOE_WAVE, lq = tid & 3, K = a.K, wanted = score_wanted(K);
  const int t = blockIdx.y * SCORE_ROW + blockIdx.x;
  if (t >= a.T) return;
  const int y = a.target[t];
  if (y < 0 || y >= a.V) {
    if (tid == 0) { a.logp[t] = 0.f; a.entropy[t] = 0.f; a.lse[t] = 0.f; }
    for (int k = tid; k < K; k += THREADS) { a.ids[static_cast<size_t>(t) * K + k] = -1; a.top[static_cast<size_t>(t) * K + k] = 0.f; }
    return;
  }
  const int row = a.control != nullptr ? a.token_row[t] : t;
  const HeadStrip* const strip = static_cast<const HeadStrip*>(a.part) + static_cast<size_t>(row) * a.strips;
  const float c1 = a.c1;
  int32_t* const columns = reinterpret_cast<int32_t*>(exact + wanted * (HALF / 4) + 1);

  // the larger logit, of equal ones the lower column, has the larger key; 0: none
  const auto key_of = [&](const HeadTop& x, int s) __attribute__((always_inline)) -> uint64_t {
    const int place = static_cast<int>(x.next & LOW), col = s * HALF + 16 * (place >> 2) + 4 * lq + (place & 3);
    return __float_as_uint(x.top) == NONE ? 0 : static_cast<uint64_t>(ordered_u32(__float_as_uint(x.top))) << 32 | ~static_cast<uint32_t>(col);
  };
  const auto load = [&](int s0, HeadTop (&x)[AT_ONCE]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int s = s0 + i * STEP;
      x[i] = HeadTop{-__builtin_inff(), 0};
      if (s < a.strips) x[i] = strip[s].lane[lq];
    }
  };
  // All logits but a thread's largest are summed up at once; the largest of all is left out.  (A sum's NaN reaches all that is made of it.)
  constexpr bool KEEP = THREADS > 256;
  HeadTop kept[KEEP ? AT_ONCE : 1];                                       // of the first round
  uint64_t best = 0;
  ScoreSum total;
  for (int s0 = tid >> 2; s0 < a.strips; s0 += AT_ONCE * STEP) {
    HeadTop x[AT_ONCE];
    float sum[AT_ONCE], moment[AT_ONCE], E[AT_ONCE], most = total.e;
    load(s0, x);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      sum[i] = moment[i] = 0.f;
      if (lq == 0 && s0 + i * STEP < a.strips) {
        const HeadStrip* const at = strip + s0 + i * STEP;
        sum[i] = at->sum;
        moment[i] = at->moment;
      }
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if constexpr (KEEP) { if (s0 == tid >> 2) kept[i] = x[i]; }
      float whole = x[i].top;
      whole = __builtin_elementwise_maximum(whole, __uint_as_float(dpp_u32<0xB1>(__float_as_uint(whole))));
      whole = __builtin_elementwise_maximum(whole, __uint_as_float(dpp_u32<0x4E>(__float_as_uint(whole))));
      E[i] = __float_as_uint(whole) == NONE ? total.e : ceilf(whole * c1);
      most = fmaxf(most, E[i]);
    }
    total.raise(fmaxf(most, -3.0e38f));
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      total.add(__float_as_uint(x[i].top) == NONE && sum[i] == 0.f ? total.e : E[i], sum[i], moment[i]);
      const uint64_t key = key_of(x[i], s0 + i * STEP), less = key < best ? key : best;
      best = key < best ? best : key;
      if (less != 0) total.add_logit(from_ordered(static_cast<uint32_t>(less >> 32)), c1);
    }
  }
  if (tid == 0) { s_top = s_least = 0; s_found = s_columns = 0; s_top_at = 0; s_border = 0; }
  {
    // The largest of every few threads, and of these the one that `wanted` - 1 are above: no smaller logit is among the `wanted` largest.
    const bool coarse = wanted <= 32;                                     // 64 groups are enough
    constexpr int FINE = THREADS / GROUPS;
    uint64_t mine = group_most<FINE>(best);
    if (coarse) mine = group_most<FINE * 4>(mine);
    const int size = coarse ? FINE * 4 : FINE, groups = THREADS / size;
    if (tid % size == 0) keys[tid / size] = mine;
    __syncthreads();
    ranked<THREADS>(groups, [&](int k, int i) __attribute__((always_inline)) { return keys[k] > keys[i]; }, [&](int i, int above) __attribute__((always_inline)) {
      if (above == 0 && keys[i] != 0) s_top = keys[i];
      if (above == wanted - 1 && keys[i] != 0) s_least = keys[i];
    });
    __syncthreads();
    if (best != s_top && best != 0) total.add_logit(from_ordered(static_cast<uint32_t>(best >> 32)), c1);
  }
  {
    const float e = group_max<MOE_WAVE>(total.e);
    total.raise(e);
    const float moment = group_sum<MOE_WAVE>(total.moment), sum = group_sum<MOE_WAVE>(total.sum);
    if (lane == 0) { part[wave][0] = e; part[wave][1] = sum; part[wave][2] = moment; }
  }
  __syncthreads();
  const uint64_t top_key = s_top, least = s_least;
  const int top_col = static_cast<int>(~static_cast<uint32_t>(top_key));
  int m;                                                                  // columns whose logits are formed anew, beside the target
  {
    int n;                                                                // lanes of the product whose columns are looked at
    const auto look = [&](const HeadTop& x, int s) __attribute__((always_inline)) {
      const uint64_t key = key_of(x, s);
      if (key == 0 || key < least) return;
      const int at = atomicAdd(&s_found, 1);
      if (at < SCORE_CANDIDATES) { found[at] = key; found_next[at] = x.next | LOW; }
    };
    if constexpr (KEEP) {
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) if ((tid >> 2) + i * STEP < a.strips) look(kept[i], (tid >> 2) + i * STEP);
    }
    for (int s0 = (tid >> 2) + (KEEP ? AT_ONCE * STEP : 0); s0 < a.strips; s0 += AT_ONCE * STEP) {
      HeadTop x[AT_ONCE];
      load(s0, x);
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) look(x[i], s0 + i * STEP);
    }
    __syncthreads();
    n = s_found;
    if (n <= SCORE_CANDIDATES) {
      ranked<THREADS>(n, [&](int k, int i) __attribute__((always_inline)) { return found[k] > found[i]; }, [&](int i, int above) __attribute__((always_inline)) {
        if (above < wanted) { chosen[above] = found[i]; chosen_next[above] = found_next[i]; }
      });
      n = n < wanted ? n : wanted;
    } else {
      // (large logits in few threads' strips: one after the other)
      n = 0;
      for (uint64_t last = ~0ull; n < wanted; ++n) {
        uint64_t most = 0;
        uint32_t next = 0;
        for (int s = tid >> 2; s < a.strips; s += STEP) {
          const HeadTop x = strip[s].lane[lq];
          const uint64_t key = key_of(x, s);
          if (key < last && key > most) { most = key; next = x.next | LOW; }
        }
        const uint64_t of_wave = group_most<MOE_WAVE>(most);
        __syncthreads();
        if (lane == 0) keys[wave] = of_wave;
        __syncthreads();
        uint64_t whole = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) whole = keys[w] > whole ? keys[w] : whole;
        if (whole == 0) break;
        if (most == whole) { chosen[n] = most; chosen_next[n] = next; }
        last = whole;
      }
    }
    __syncthreads();
    // No logit below the `wanted`-th of the largest and second largest of these lanes is among the `wanted` largest of all.  The columns to look at: the lanes' largest down
    // to that, and all of a lane whose second largest may be as large (it is known but for its low bits).
    const auto value = [&](int i) __attribute__((always_inline)) { return i < n ? static_cast<uint32_t>(chosen[i] >> 32) : chosen_next[i - n] & ~LOW; };
    uint32_t border = n == wanted ? value(n - 1) : 0;
    // (Finding it costs as much as looking at one lane more.  One token, 17 of 213 columns: 28 -> 18 us.)
    if (__syncthreads_count(tid < n && chosen_next[tid] >= LEAST && chosen_next[tid] >= border) > 1) {
      ranked<THREADS>(2 * n, [&](int k, int i) __attribute__((always_inline)) { return value(k) > value(i) || (value(k) == value(i) && k < i); },
                      [&](int i, int above) __attribute__((always_inline)) { if (above == wanted - 1) s_border = value(i); });
      __syncthreads();
      border = s_border > border ? s_border : border;
    }
    for (int i = tid; i < n * (HALF / 4); i += THREADS) {
      const int which = i / (HALF / 4), place = i % (HALF / 4), own = static_cast<int>(~static_cast<uint32_t>(chosen[which]));
      const int col = own / HALF * HALF + 16 * (place >> 2) + (own & 12) + (place & 3);
      const uint32_t next = chosen_next[which];
      const bool all_of_it = next >= LEAST && next >= border;
      if (col == own ? own == top_col || static_cast<uint32_t>(chosen[which] >> 32) >= border : all_of_it && col < a.V) {
        const int at = atomicAdd(&s_columns, 1);
        columns[at] = col;
        if (col == top_col) s_top_at = at;
      }
    }
    __syncthreads();
    m = s_columns;
    if (tid == 0) columns[m] = y;
    __syncthreads();
  }
  form_exact<THREADS, false>(a.x + static_cast<size_t>(t) * a.d, a.W, a.d, columns, exact, m);
  __syncthreads();
  ScoreSum all;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) all.e = fmaxf(all.e, part[w][0]);
#pragma unroll
  for (int w = 0; w < WAVES; ++w) all.add(part[w][0], part[w][1], part[w][2]);
  const double z_top = exact[s_top_at];
  const ScoreResult r = result_of(all, top_key != 0, z_top, c1);
  if (tid == 0) put_scores(a, t, r, y == top_col, exact[m], z_top);
  put_alternatives<THREADS>(a, t, r, columns, exact, m, top_col, z_top);
}

// The logits' gradient from their summands: what the epilogue of the product of HEAD_SCORE_DZ does with whole logits, and, as all of a row is at hand, what head_sure_kernel does
// behind it.  THREADS to a row, eight columns each at a time.
template <int THREADS> __global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void head_score_dz_kernel(ScoreDzArgs a) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u4;
  constexpr int ROWS = THREADS < 256 ? 256 / THREADS : 1, WAVES = THREADS / MOE_WAVE;
  __shared__ float part[WAVES];
  const int tid = threadIdx.x % THREADS, row = blockIdx.x * ROWS + threadIdx.x / THREADS, rows = a.control[1];
  if (row >= rows) return;
  const int z_ld = score_ld(a.V), y = a.target[row];
  const f32x4_t p = a.row[row];
  const float at_target = a.terms[row][0];
  const float* const z_row = a.part + static_cast<size_t>(row) * z_ld;
  const auto rounded = [](float x) __attribute__((always_inline)) { return bf16_to_f32(f32_to_bf16(x)); };
  float sum = 0.f;
  int found = 0, top = 0;
  for (int c = tid * 8; c < a.ld; c += THREADS * 8) {
    float g[8] = {};
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      if (c + h >= z_ld) continue;
      const float* z_at = z_row + c + h;
      f32x4_t z = *reinterpret_cast<const f32x4_t*>(z_at);
      for (int part = 1; part < a.parts; ++part) z += *reinterpret_cast<const f32x4_t*>(z_at += static_cast<size_t>(a.T) * z_ld);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = c + h + i;
        const float t = __builtin_fmaf(z[i], a.c1, -p[0]);
        float v = __builtin_amdgcn_exp2f(t) * __builtin_fmaf(p[2], t, p[1]);
        if (col >= a.V) v = 0.f;
        else if (col == y) v = at_target;
        else if (score_apart(z[i], a.c1, p)) { ++found; top = col; v = __builtin_nanf(""); }
        g[h + i] = v;
        if (v == v) sum += v;
      }
    }
    const auto put = [&](int r) __attribute__((always_inline)) {
      *reinterpret_cast<u4*>(a.dz + static_cast<size_t>(r) * a.ld + c) = u4{pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]), pack_bf16(g[4], g[5]), pack_bf16(g[6], g[7])};
    };
    put(row);
    if (rows <= a.low) {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] -= rounded(g[i]);
      put(rows + row);
    }
  }
  if (tid == 0) a.item[row] = at_target - rounded(at_target);
  if (!(p[3] <= 0.f)) return;                                             // (the same for all threads of a row)
  sum = group_sum<MOE_WAVE>(sum);
  bool one = __popcll(__ballot(found == 1)) == 1 && __ballot(found > 1) == 0;
  if constexpr (WAVES > 1) {
    if (threadIdx.x % MOE_WAVE == 0) part[threadIdx.x / MOE_WAVE] = sum;
    one = __syncthreads_count(found != 0) == 1;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += part[w];
  }
  if (!one || found != 1) return;                                         // (NaN for a row that has more of it)
  a.dz[static_cast<size_t>(row) * a.ld + top] = f32_to_bf16(-sum);
  if (rows <= a.low) a.dz[static_cast<size_t>(rows + row) * a.ld + top] = f32_to_bf16(-sum - rounded(-sum));
}

// Threads for a token whose logits are all looked at, each with 32 of them at most: many where there are few tokens, few where there are many (d 832, us of the whole call,
// 64 / 128 / 256 threads: V 697, 8 alternatives, 500 tokens 36 / 35 / 32, 2000 42 / 44 / 53, 8000 84 / 102 / 145; V 4000, 20 alternatives, 128 / 256: 500 44 / 40, 8000 188 / 214).
// Short rows in registers for them alone: 8192 tokens, d 2048, V 256, 20 alternatives, with 8 / 2 pieces a thread 146 / 131; 300, 704, 697 33 / 31.
// A few tokens, their rows formed anew by waves, 256 / 1024 threads: 16, 4096, 5000 39 / 35.5; 200, 2048, 3001 36 / 34; 1, 4096, 256 29.5 / 35.  At the borders (from a graph):
// 256, 2048, 8192 33.6 / 32.6; 256, 256, 2049 17.7 / 17.4; 256, 512, 8192 20.1 / 20.2; 1, 512, 2049, one alternative 14.4 / 14.7; 64 alternatives 256, 512, 4096 28.9 / 23.3;
// 64, 2048, 5000 38 / 28; past 256 tokens 300, 256, 5000 25.5 / 32, 500, 2048, 3000 36.5 / 45.
// (64 threads are 64 groups: with as many alternatives wanted nearly every column would be a candidate.)
void launch_whole(const ScoreJoinArgs& a, dim3 grid, hipStream_t s) {
  const auto launch = [&](auto threads, auto pieces) {
    constexpr int THREADS = decltype(threads)::value, PIECES = decltype(pieces)::value;
    // (1024 threads are for alternatives)
    if constexpr (THREADS > 512) MOE_LAUNCH("head_score_whole", (head_score_whole_kernel<THREADS, PIECES, true>), grid, dim3(THREADS), 0, s, a);
    else if (a.K > 0) MOE_LAUNCH("head_score_whole", (head_score_whole_kernel<THREADS, PIECES, true>), grid, dim3(THREADS), 0, s, a);
    else MOE_LAUNCH("head_score_whole", (head_score_whole_kernel<THREADS, PIECES, false>), grid, dim3(THREADS), 0, s, a);
  };
  using std::integral_constant;
  const bool few = a.T <= SCORE_SOME;
  if (a.K > 0 && a.T <= SCORE_FEW && a.V > 2048 && a.V <= 8192) launch(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  else if (!few && a.V <= 512 && score_wanted(a.K) <= 32) launch(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (!few && a.V <= 2048 && score_wanted(a.K) <= 32) launch(integral_constant<int, 64>{}, integral_constant<int, 8>{});
  else if (few && a.V <= 2048) launch(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (!few && a.V <= 4096) launch(integral_constant<int, 128>{}, integral_constant<int, 8>{});
  else if (a.V <= 8192) launch(integral_constant<int, 256>{}, integral_constant<int, 8>{});
  else launch(integral_constant<int, 512>{}, integral_constant<int, 8>{});
}
template <int HALF> void launch_join(const ScoreJoinArgs& a, hipStream_t s) {
  const auto rows = [](int n) { return dim3(n < SCORE_ROW ? n : SCORE_ROW, (n + SCORE_ROW - 1) / SCORE_ROW); };
  if (a.K == 0 && !a.whole) {
    const bool few = a.T <= SCORE_FEW;
    const dim3 grid = few ? dim3(a.T) : rows((a.T + 3) / 4);
    if (a.of_row != nullptr) {
      if (few) MOE_LAUNCH("head_score_sure", (head_score_kernel<HALF, true, true>), grid, dim3(256), 0, s, a);
      else MOE_LAUNCH("head_score_sure", (head_score_kernel<HALF, false, true>), grid, dim3(256), 0, s, a);
    } else if (few) MOE_LAUNCH("head_score", (head_score_kernel<HALF, true, false>), grid, dim3(256), 0, s, a);
    else MOE_LAUNCH("head_score", (head_score_kernel<HALF, false, false>), grid, dim3(256), 0, s, a);
    return;
  }
  if (a.whole) {
    launch_whole(a, rows(a.T), s);
    return;
  }
  const int lds = (score_wanted(a.K) * (HALF / 4) + 1) * 12;
  const dim3 grid = rows(a.T);
  if (a.T <= SCORE_FEW) MOE_LAUNCH("head_score_join", (head_score_join_kernel<HALF, 1024>), grid, dim3(1024), lds, s, a);
  else MOE_LAUNCH("head_score_join", (head_score_join_kernel<HALF, 256>), grid, dim3(256), lds, s, a);
}

}  // namespace

int moe_head_score_dz(const ScoreDzArgs& a, hipStream_t s) {
  if (a.ld <= 8 * MOE_WAVE) MOE_LAUNCH("head_score_dz", head_score_dz_kernel<MOE_WAVE>, dim3((a.T + 3) / 4), dim3(256), 0, s, a);
  else if (a.ld <= 4096) MOE_LAUNCH("head_score_dz", head_score_dz_kernel<256>, dim3(a.T), dim3(256), 0, s, a);
  else MOE_LAUNCH("head_score_dz", head_score_dz_kernel<1024>, dim3(a.T), dim3(1024), 0, s, a);
  return moe_check_launch();
}
int moe_head_score_join(const ScoreJoinArgs& a, int edge, hipStream_t s) {
  if (edge == 128) launch_join<64>(a, s);
  else launch_join<128>(a, s);
  return moe_check_launch();
}
