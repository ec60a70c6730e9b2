// Joins the strips of the vocabulary head's logits into log probabilities, entropies and likeliest alternatives.
//
// With o_j the distance of logit j from the largest, over the temperature, R the sum of exp(-o) over all columns but the largest's and Q that of o exp(-o):
//   log p of the largest = -log(1 + R);   of any other -log(1 + R) - o;   entropy = log(1 + R) + Q / (1 + R)
// All terms are positive: a token that the model is sure of keeps the digits of its log probability and entropy, which a difference of the two usual sums would not.
//
// Which of two logits is larger is told in 64 bits (products of two bf16 numbers are exact in 32 bits, their sums in 64 are off by 1e-16): the chain of additions of the
// matrix product would put one in some 10^4 alternatives in the wrong place.  So the K + SCORE_SPARE largest by the product are formed anew, a row of W each, and ordered by that.
// Candidates: the columns of a lane of the product (16 or 32) have their largest apart.  None of the C largest logits lies in another lane's columns than
// those with the C largest of these; where the second largest of such a lane may be among them too, all of its columns are candidates.  That is one lane in four
// tokens for 28 of 50304 columns, and no more than C of them whatever the logits are.
#include "head_score.h"

namespace {

constexpr int SCORE_THREADS = 256, SCORE_CANDIDATES = 512;

__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) != 0 ? 0x80000000u : 0xFFFFFFFFu)); }
// Sums of 2^t and t 2^t relative to 2^e, e a whole number.
struct ScoreSum {
  float e = -3.0e38f, sum = 0.f, moment = 0.f;
  __device__ __forceinline__ void add(float E, float s, float m) {
    const float n = fmaxf(e, E), f = __builtin_amdgcn_exp2f(e - n), g = __builtin_amdgcn_exp2f(E - n);
    moment = f * __builtin_fmaf(sum, e - n, moment) + g * __builtin_fmaf(s, E - n, m);
    sum = f * sum + g * s;
    e = n;
  }
  __device__ __forceinline__ void add_logit(float z, float c1) {
    const float E = ceilf(z * c1), t = __builtin_fmaf(z, c1, -E), s = __builtin_amdgcn_exp2f(t);
    add(E, s, s * t);
  }
};

// Logits of up to four columns in 64 bits, by a wave.
__device__ __forceinline__ void exact_logits(const moe_bf16* x, const moe_bf16* W, int d, const int (&col)[4], double (&z)[4]) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u4;
  const int lane = threadIdx.x % MOE_WAVE;
#pragma unroll
  for (int k = 0; k < 4; ++k) z[k] = 0.0;
#pragma unroll 2
  for (int c = lane * 8; c < d; c += MOE_WAVE * 8) {
    u4 w[4];
    const u4 p = *reinterpret_cast<const u4*>(x + c);
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const u4*>(W + static_cast<size_t>(col[k]) * d + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float lo = bf16lo(p[i]), hi = bf16hi(p[i]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        z[k] += static_cast<double>(lo * bf16lo(w[k][i]));
        z[k] += static_cast<double>(hi * bf16hi(w[k][i]));
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int i = 1; i < MOE_WAVE; i *= 2) z[k] += __shfl_xor(z[k], i);
}
__device__ __forceinline__ int64_t ordered_i64(double v) {
  const int64_t b = __builtin_bit_cast(int64_t, v == 0.0 ? 0.0 : v);          // (-0 and +0 are equal)
  return b >= 0 ? b : b ^ 0x7FFFFFFFFFFFFFFFll;
}

// A workgroup for each token.  HALF: columns of a strip.
template <int HALF>
__global__ __launch_bounds__(SCORE_THREADS) void head_score_join_kernel(ScoreJoinArgs a) {
  extern __shared__ double exact[];
  __shared__ uint64_t keys[SCORE_THREADS], found[SCORE_CANDIDATES], chosen[score_wanted(SCORE_MAX_K)], s_top, s_least;
  __shared__ uint32_t found_next[SCORE_CANDIDATES], chosen_next[score_wanted(SCORE_MAX_K)];
  __shared__ float part[4][3];
  __shared__ int s_found, s_columns;
  constexpr uint32_t LOW = HALF / 4 - 1;
  constexpr uint32_t NONE = 0xFF800000u, LEAST = 0x00800000u;             // -infinity; the order of the lowest number
  const int tid = threadIdx.x, lane = tid % MOE_WAVE, wave = tid / MOE_WAVE, lq = tid & 3, t = blockIdx.x, K = a.K, wanted = score_wanted(K);
  const int y = a.target[t];
  if (y < 0 || y >= a.V) {
    if (tid == 0) { a.logp[t] = 0.f; a.entropy[t] = 0.f; a.lse[t] = 0.f; }
    for (int k = tid; k < K; k += SCORE_THREADS) { a.ids[static_cast<size_t>(t) * K + k] = -1; a.top[static_cast<size_t>(t) * K + k] = 0.f; }
    return;
  }
  const int row = a.control != nullptr ? a.token_row[t] : t;
  const HeadStrip* const strip = a.part + static_cast<size_t>(row >> 4) * a.strips * 16 + (row & 15);
  const float c1 = a.c1;
  int32_t* const columns = reinterpret_cast<int32_t*>(exact + wanted * (HALF / 4) + 1);

  // the larger logit, of equal ones the lower column, has the larger key; 0: none
  const auto key_of = [&](const HeadTop& x, int s) __attribute__((always_inline)) -> uint64_t {
    const int place = static_cast<int>(x.next & LOW), col = s * HALF + 16 * (place >> 2) + 4 * lq + (place & 3);
    return __float_as_uint(x.top) == NONE ? 0 : static_cast<uint64_t>(ordered_u32(__float_as_uint(x.top))) << 32 | ~static_cast<uint32_t>(col);
  };
  uint64_t best = 0;
  ScoreSum total;
#pragma unroll 4
  for (int s = tid >> 2; s < a.strips; s += SCORE_THREADS / 4) {
    const HeadTop x = strip[static_cast<size_t>(s) * 16].lane[lq];
    float sum = 0.f, moment = 0.f;
    if (lq == 0) { sum = strip[static_cast<size_t>(s) * 16].sum; moment = strip[static_cast<size_t>(s) * 16].moment; }
    float whole = x.top;
    whole = __builtin_elementwise_maximum(whole, __uint_as_float(dpp_u32<0xB1>(__float_as_uint(whole))));
    whole = __builtin_elementwise_maximum(whole, __uint_as_float(dpp_u32<0x4E>(__float_as_uint(whole))));
    if (lq == 0 && !(__float_as_uint(whole) == NONE)) total.add(whole == whole ? ceilf(whole * c1) : whole, sum, moment);
    const uint64_t key = key_of(x, s), less = key < best ? key : best;
    best = key < best ? best : key;
    if (less != 0) total.add_logit(from_ordered(static_cast<uint32_t>(less >> 32)), c1);
  }
  keys[tid] = best;
  if (tid == 0) { s_top = s_least = 0; s_found = s_columns = 0; }
  __syncthreads();
  int rank = 0;
#pragma unroll 8
  for (int i = 0; i < SCORE_THREADS; ++i) rank += keys[i] > best;
  if (rank == 0 && best != 0) s_top = best;
  if (rank == wanted - 1 && best != 0) s_least = best;
  if (rank != 0 && best != 0) total.add_logit(from_ordered(static_cast<uint32_t>(best >> 32)), c1);
  {
    const float e = group_max<MOE_WAVE>(total.e), f = __builtin_amdgcn_exp2f(total.e - e);
    const float moment = group_sum<MOE_WAVE>(f * __builtin_fmaf(total.sum, total.e - e, total.moment)), sum = group_sum<MOE_WAVE>(f * total.sum);
    if (lane == 0) { part[wave][0] = e; part[wave][1] = sum; part[wave][2] = moment; }
  }
  __syncthreads();
  ScoreSum all;
#pragma unroll
  for (int w = 0; w < 4; ++w) all.add(part[w][0], part[w][1], part[w][2]);
  const uint64_t top_key = s_top, least = s_least;
  int n = top_key != 0 ? 1 : 0;                                           // lanes of the product whose columns are looked at
  if (K == 0) {
    if (tid == 0) { chosen[0] = top_key; chosen_next[0] = 0; }
  } else {
    for (int s = tid >> 2; s < a.strips; s += SCORE_THREADS / 4) {
      const HeadTop x = strip[static_cast<size_t>(s) * 16].lane[lq];
      const uint64_t key = key_of(x, s);
      if (key == 0 || key < least) continue;
      const int at = atomicAdd(&s_found, 1);
      if (at < SCORE_CANDIDATES) { found[at] = key; found_next[at] = x.next | LOW; }
    }
    __syncthreads();
    n = s_found;
    if (n <= SCORE_CANDIDATES) {
      for (int i = tid; i < n; i += SCORE_THREADS) {
        const uint64_t mine = found[i];
        int above = 0;
        for (int k = 0; k < n; ++k) above += found[k] > mine;
        if (above < wanted) { chosen[above] = mine; chosen_next[above] = found_next[i]; }
      }
      n = n < wanted ? n : wanted;
    } else {
      // (large logits in few threads' strips: one after the other)
      n = 0;
      for (uint64_t last = ~0ull; n < wanted; ++n) {
        uint64_t most = 0;
        uint32_t next = 0;
        for (int s = tid >> 2; s < a.strips; s += SCORE_THREADS / 4) {
          const HeadTop x = strip[static_cast<size_t>(s) * 16].lane[lq];
          const uint64_t key = key_of(x, s);
          if (key < last && key > most) { most = key; next = x.next | LOW; }
        }
        __syncthreads();
        keys[tid] = most;
        __syncthreads();
        uint64_t whole = 0;
        for (int i = 0; i < SCORE_THREADS; ++i) whole = keys[i] > whole ? keys[i] : whole;
        if (whole == 0) break;
        if (most == whole) { chosen[n] = most; chosen_next[n] = next; }
        last = whole;
      }
    }
  }
  __syncthreads();
  // the columns to look at: those, and all of a lane whose second largest may be among the `wanted` largest
  const uint32_t border = n == wanted ? static_cast<uint32_t>(chosen[n - 1] >> 32) : 0;
  for (int i = tid; i < n * (HALF / 4); i += SCORE_THREADS) {
    const int which = i / (HALF / 4), place = i % (HALF / 4), own = static_cast<int>(~static_cast<uint32_t>(chosen[which]));
    const int col = own / HALF * HALF + 16 * (place >> 2) + (own & 12) + (place & 3);
    const uint32_t next = chosen_next[which];
    if (col == own || (K > 0 && next >= LEAST && next >= border && col < a.V)) columns[atomicAdd(&s_columns, 1)] = col;
  }
  __syncthreads();
  const int m = s_columns;
  if (tid == 0) columns[m] = y;
  __syncthreads();
  for (int i = wave * 4; i <= m; i += 16) {
    int col[4];
    double z[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) col[k] = __builtin_amdgcn_readfirstlane(columns[i + k <= m ? i + k : m]);
    exact_logits(a.x + static_cast<size_t>(t) * a.d, a.W, a.d, col, z);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane == 0 && i + k <= m) exact[i + k] = z[k];
  }
  __syncthreads();
  // the largest logit by the product is what the sums leave out: the formulas hold whether it is the largest in 64 bits or next to it
  const int top_col = static_cast<int>(~static_cast<uint32_t>(top_key));
  double z_top = 0.0;
  for (int i = 0; i < m; ++i) z_top = columns[i] == top_col ? exact[i] : z_top;
  const double from = static_cast<double>(all.e) - z_top * static_cast<double>(c1);
  // (NaN where a logit is no number or infinite, and where a scale of 2^30 or more leaves its exponent without digits)
  const bool alone = all.e == -3.0e38f;                                    // no other column
  const bool fine = top_key != 0 && fabs(z_top * static_cast<double>(c1)) < 0x1p30 && (alone || fabsf(all.e) < 0x1p30f);
  const double whole = fmax(rint(from), -10000.0);
  const float scale = fine ? __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(static_cast<float>(from - whole)), static_cast<int>(whole)) : __builtin_nanf("");
  const float R = alone ? 0.f : all.sum * scale;
  const float Q = alone ? 0.f : -0.693147180559945309f * scale * __builtin_fmaf(static_cast<float>(from), all.sum, all.moment);
  const double log_1R = static_cast<double>(fine ? log1pf(R) : __builtin_nanf(""));
  if (tid == 0) {
    a.logp[t] = y == top_col ? -static_cast<float>(log_1R) : static_cast<float>((exact[m] - z_top) * a.over_tau - log_1R);
    a.entropy[t] = static_cast<float>(log_1R) + Q / (1.f + R);
    a.lse[t] = static_cast<float>(z_top * a.over_tau + log_1R);
  }
  if (K == 0) return;
  for (int k = m + tid; k < K; k += SCORE_THREADS) {                       // (logits of -infinity)
    a.ids[static_cast<size_t>(t) * K + k] = -1;
    a.top[static_cast<size_t>(t) * K + k] = __builtin_nanf("");
  }
  for (int i = tid; i < m; i += SCORE_THREADS) {
    const int64_t mine = ordered_i64(exact[i]);
    const int col = columns[i];
    int above = 0;
    for (int k = 0; k < m; ++k) {
      const int64_t other = ordered_i64(exact[k]);
      above += other > mine || (other == mine && columns[k] < col);
    }
    if (above >= K) continue;
    a.ids[static_cast<size_t>(t) * K + above] = col;
    a.top[static_cast<size_t>(t) * K + above] = col == top_col ? -static_cast<float>(log_1R) : static_cast<float>((exact[i] - z_top) * a.over_tau - log_1R);
  }
}

}  // namespace

int moe_head_score_join(const ScoreJoinArgs& a, int edge, hipStream_t s) {
  const int lds = (score_wanted(a.K) * (edge / 8) + 1) * 12;
  if (edge == 128) MOE_LAUNCH("head_score_join", head_score_join_kernel<64>, dim3(a.T), dim3(SCORE_THREADS), lds, s, a);
  else MOE_LAUNCH("head_score_join", head_score_join_kernel<128>, dim3(a.T), dim3(SCORE_THREADS), lds, s, a);
  return moe_check_launch();
}
