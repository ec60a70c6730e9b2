// The vocabulary head's losses and their gradients.  With logits z = x W^T of a token, its target y and a teacher's logits l on a few entries:
//   loss = log sum exp z - z_y                                        dz += dloss (softmax z - [y])
//   kd   = sum over entries of q (log q - log p), q = softmax(l / tau), p = softmax(z / tau)     dz += dkd / tau (p - q)
//   dx = dz W;   dW = dz^T x
// The logits are never in memory.  Forward: the product's epilogue leaves a row's maximum and sum of exponentials for every strip of columns, and
// the logits that count by themselves (target, entries); a last kernel joins them.  Backward: the logits once more, their gradient
// rounded to bf16 (the products read it as their operand; half a step is 2^-9 of each element, against the 2^-9 of dx and dW themselves), then
// the two products.  What bounds it is the matrix pipe: four products of 2 T V d operations, one of them for the logits a second time.
//
// Tokens without a loss are left out of all products: a first kernel finds the others, copies their rows of x side by side, and lists by blocks of
// 16 rows and strips of 64 columns which logits count by themselves.
#include <initializer_list>
#include "gemm_tile.h"

namespace {

constexpr int HEAD_MAX_V = 1 << 20, HEAD_MAX_K = 1024;
constexpr int HEAD_CUS = 256;                       // what the workspace's size is laid out for
constexpr int SELF_MASK_TOKENS = 4096;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Teacher { const int32_t* ids; const float* logits; float temperature; int K; };

__device__ __forceinline__ bool entry_there(int id, float l, int V) { return id >= 0 && id < V && l > -__builtin_inff(); }
__device__ __forceinline__ bool target_there(int y, int V) { return y >= 0 && y < V; }

// Which tokens have a loss, a bit each: a target, or (K > 0) an entry.  A wave takes 64 tokens.
__global__ __launch_bounds__(256) void head_mask_kernel(const int32_t* __restrict__ target, Teacher t, int T, int V, uint64_t* __restrict__ mask) {
  __shared__ int some[4][MOE_WAVE];
  const int lane = threadIdx.x % MOE_WAVE, wave = threadIdx.x / MOE_WAVE;
  const int word = blockIdx.x * 4 + wave, t0 = word * 64;
  if (t0 >= T) return;
  some[wave][lane] = t0 + lane < T && target_there(target[t0 + lane], V);
  __builtin_amdgcn_wave_barrier();
  const size_t n = static_cast<size_t>(T - t0 < 64 ? T - t0 : 64) * t.K, at = static_cast<size_t>(t0) * t.K;
#pragma unroll 4
  for (size_t i = lane; i < n; i += MOE_WAVE)
    if (entry_there(t.ids[at + i], t.logits[at + i], V)) some[wave][static_cast<int>(i) / t.K] = 1;
  __builtin_amdgcn_wave_barrier();
  const uint64_t bits = __ballot(some[wave][lane] != 0);
  if (lane == 0) mask[word] = bits;
}

struct HeadPrepArgs {
  const moe_bf16* x;
  const int32_t* target;
  Teacher t;
  const uint64_t* mask;            // null: up to SELF_MASK_TOKENS tokens, and no teacher
  int T, d, V, strips;             // strips: of 64 columns
  int32_t *offsets, *row_token, *token_row;
  moe_bf16* xc;
  int32_t* list_start;
  HeadItem* items;
  int32_t* target_slot;
  float *loss, *lse, *kd, *lse_t;  // forward: zeros for tokens without a loss
  const float *in_loss, *in_lse, *in_lse_t, *dloss, *dkd;   // backward: the rows' factors
  f32x4_t* row;
};

// Workgroup b: rows 16 b to 16 b + 15 of those with a loss, in the order of their tokens; and tokens 16 b to 16 b + 15, if they have none.
__global__ __launch_bounds__(256) void head_prep_kernel(HeadPrepArgs a) {
  extern __shared__ int count[];                     // [strips + 1]
  __shared__ uint64_t own[SELF_MASK_TOKENS / 64];
  __shared__ int wave_sum[4], s_token[16], s_target[16], s_slot[16], s_taught[16];
  const int tid = threadIdx.x, lane = tid % MOE_WAVE, wave = tid / MOE_WAVE;
  const int words = (a.T + 63) / 64, per = (words + 255) / 256, K = a.t.K, V = a.V, slots = K + 1;
  const uint64_t* mask = a.mask;
  if (mask == nullptr) {
    for (int w = wave; w < words; w += 4) {
      const int t = w * 64 + lane;
      const uint64_t bits = __ballot(t < a.T && target_there(a.target[t], V));
      if (lane == 0) own[w] = bits;
    }
    mask = own;
  }
  if (tid < 16) { s_token[tid] = -1; s_slot[tid] = K; s_taught[tid] = 0; }
  for (int i = tid; i <= a.strips; i += 256) count[i] = 0;
  __syncthreads();
  // rank of each thread's first token among those with a loss
  const int w0 = tid * per < words ? tid * per : words, w1 = w0 + per < words ? w0 + per : words;
  int mine = 0;
  for (int w = w0; w < w1; ++w) mine += __builtin_popcountll(mask[w]);
  int rank = wave_incl_scan(mine);
  if (lane == 63) wave_sum[wave] = rank;
  __syncthreads();
  int live = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) { rank += w < wave ? wave_sum[w] : 0; live += wave_sum[w]; }
  rank -= mine;
  const int first = blockIdx.x * 16;
  if (blockIdx.x == 0 && tid == 0) { a.offsets[0] = 0; a.offsets[1] = live; }
  if (tid < 16 && first + tid < a.T) {
    const int t = first + tid;
    if ((mask[t >> 6] >> (t & 63) & 1) == 0) {
      a.token_row[t] = -1;
      if (a.loss != nullptr) {
        a.loss[t] = 0.f;
        a.lse[t] = 0.f;
        if (K > 0) { a.kd[t] = 0.f; a.lse_t[t] = 0.f; }
      }
    }
  }
  if (first >= live) return;
  for (int w = w0; w < w1 && rank < first + 16; ++w) {
    uint64_t bits = mask[w];
    const int n = __builtin_popcountll(bits);
    if (rank + n <= first) { rank += n; continue; }
    for (; bits != 0; bits &= bits - 1, ++rank) {
      if (rank < first || rank >= first + 16) continue;
      const int t = w * 64 + __builtin_ctzll(bits);
      s_token[rank - first] = t;
      s_target[rank - first] = a.target[t];
      a.row_token[rank] = t;
      a.token_row[t] = rank;
    }
  }
  __syncthreads();
  const int n = live - first < 16 ? live - first : 16, pieces = a.d / 8;
  for (int i = tid; i < n * pieces; i += 256) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u4;
    const int r = i / pieces, c = (i - r * pieces) * 8;
    *reinterpret_cast<u4*>(a.xc + static_cast<size_t>(first + r) * a.d + c) = *reinterpret_cast<const u4*>(a.x + static_cast<size_t>(s_token[r]) * a.d + c);
  }
  auto entry = [&](int i, int& r, int& j, int& id) __attribute__((always_inline)) {
    r = i / K;
    j = i - r * K;
    const size_t at = static_cast<size_t>(s_token[r]) * K + j;
    id = a.t.ids[at];
    return entry_there(id, a.t.logits[at], V);
  };
  for (int i = tid; i < n * K; i += 256) {
    int r, j, id;
    if (!entry(i, r, j, id)) continue;
    s_taught[r] = 1;
    if (id == s_target[r]) atomicMin(&s_slot[r], j);     // the target's logit is that of an entry
    atomicAdd(&count[id >> 6], 1);
  }
  __syncthreads();
  const bool own_target = tid < n && s_slot[tid] == K && target_there(s_target[tid], V);
  if (own_target) atomicAdd(&count[s_target[tid] >> 6], 1);
  __syncthreads();
  // exclusive sums over the strips
  const int chunk = (a.strips + 255) / 256, c0 = tid * chunk, c1 = c0 + chunk < a.strips ? c0 + chunk : a.strips;
  int sum = 0;
  for (int i = c0; i < c1; ++i) sum += count[i];
  int before = wave_incl_scan(sum);
  if (lane == 63) wave_sum[wave] = before;
  __syncthreads();
  before -= sum;
#pragma unroll
  for (int w = 0; w < 3; ++w) before += w < wave ? wave_sum[w] : 0;
  int32_t* start = a.list_start + static_cast<size_t>(blockIdx.x) * (a.strips + 1);
  for (int i = c0; i < c1; ++i) {
    const int c = count[i];
    count[i] = before;
    start[i] = before;
    before += c;
  }
  if (tid == 255) start[a.strips] = before;
  __syncthreads();
  HeadItem* items = a.items + static_cast<size_t>(blockIdx.x) * 16 * slots;
  auto put = [&](int r, int col, int slot) __attribute__((always_inline)) {   // (the order inside a strip does not matter)
    items[atomicAdd(&count[col >> 6], 1)] = HeadItem{static_cast<uint32_t>(r) | static_cast<uint32_t>(col) << 4, static_cast<uint32_t>(slot)};
  };
  for (int i = tid; i < n * K; i += 256) {
    int r, j, id;
    if (entry(i, r, j, id)) put(r, id, j);
  }
  if (own_target) put(tid, s_target[tid], K);
  if (tid < n) {
    const int t = s_token[tid];
    const bool has = target_there(s_target[tid], V), taught = s_taught[tid] != 0;
    a.target_slot[first + tid] = has ? s_slot[tid] : -1;
    if (a.row != nullptr) {
      const float none = __builtin_inff(), tau = a.t.temperature;
      f32x4_t p = {none, 0.f, none, 0.f};
      if (has) { p[0] = a.in_lse[t] * LOG2E; p[1] = a.dloss[t]; }
      if (taught) {
        const float l = a.in_lse_t[t] * LOG2E, g = a.dkd[t] / tau;
        if (tau != 1.f) { p[2] = l; p[3] = g; }
        else { if (!has) p[0] = l; p[1] += g; }                       // one sum serves both
      }
      a.row[first + tid] = p;
    }
  }
}

__device__ __forceinline__ float wave_sum_of(float v) { return group_sum<MOE_WAVE>(v); }
__device__ __forceinline__ float wave_max_of(float v) { return group_max<MOE_WAVE>(v); }

// log sum exp of a token's teacher logits over the temperature (all lanes of a wave)
__device__ __forceinline__ float teacher_lse(const Teacher& t, size_t at, int V, int lane) {
  float top = -__builtin_inff();
  for (int j = lane; j < t.K; j += MOE_WAVE) if (entry_there(t.ids[at + j], t.logits[at + j], V)) top = fmaxf(top, t.logits[at + j] / t.temperature);
  top = wave_max_of(top);
  float sum = 0.f;
  for (int j = lane; j < t.K; j += MOE_WAVE)
    if (entry_there(t.ids[at + j], t.logits[at + j], V)) sum += expf(t.logits[at + j] / t.temperature - top);
  return top + logf(wave_sum_of(sum));
}

struct HeadJoinArgs {
  const float* part;
  const int32_t *offsets, *row_token, *target_slot;
  const float* z_item;
  Teacher t;
  int strips, rows_cap, V;
  float *loss, *lse, *kd, *lse_t;
  float c1, c2;
};
// 16 rows: their strips' maxima and sums joined, then the losses.  Sums of exponentials have the scale 2^E of gemm_tile.h.
__global__ __launch_bounds__(256) void head_join_kernel(HeadJoinArgs a) {
  __shared__ float part[16][16][4], joined[16][2];
  const int tid = threadIdx.x, lane = tid % MOE_WAVE, wave = tid / MOE_WAVE;
  const int first = blockIdx.x * 16, live = a.offsets[1], K = a.t.K;
  const bool two = K > 0 && a.t.temperature != 1.f;
  if (first >= live) return;
  constexpr float NONE = -__builtin_inff(), LOW = -3.0e38f;
  {
    const int r = tid % 16, g = tid / 16, row = first + r < live ? first + r : live - 1;
    const size_t plane = static_cast<size_t>(a.strips) * a.rows_cap;
    float e1 = LOW, s1 = 0.f, e2 = LOW, s2 = 0.f;
#pragma unroll 4
    for (int s = g; s < a.strips; s += 16) {
      const float* p = a.part + static_cast<size_t>(s) * a.rows_cap + row;
      const float m = p[0], v1 = p[plane], v2 = two ? p[2 * plane] : 0.f;
      const float f1 = m > NONE ? ceilf(m * a.c1) : LOW, f2 = m > NONE ? ceilf(m * a.c2) : LOW;
      const float n1 = fmaxf(e1, f1), n2 = fmaxf(e2, f2);
      s1 = s1 * exp2f(e1 - n1) + v1 * exp2f(f1 - n1);
      s2 = s2 * exp2f(e2 - n2) + v2 * exp2f(f2 - n2);
      e1 = n1; e2 = n2;
    }
    part[r][g][0] = e1; part[r][g][1] = s1; part[r][g][2] = e2; part[r][g][3] = s2;
  }
  __syncthreads();
  if (tid < 32) {
    const int r = tid % 16, h = tid / 16 * 2;
    float e = LOW, s = 0.f;
#pragma unroll
    for (int g = 0; g < 16; ++g) e = fmaxf(e, part[r][g][h]);
#pragma unroll
    for (int g = 0; g < 16; ++g) s += part[r][g][h + 1] * exp2f(part[r][g][h] - e);
    joined[r][tid / 16] = s > 0.f ? __builtin_fmaf(e, LN2, logf(s)) : NONE;    // log of the sum over the columns that are no item
  }
  __syncthreads();
  for (int r = wave; r < 16 && first + r < live; r += 4) {
    const int row = first + r, t = a.row_token[row], slot = a.target_slot[row];
    const float* z = a.z_item + static_cast<size_t>(row) * (K + 1);
    const float rest1 = joined[r][0], rest2 = two ? joined[r][1] : rest1, tau = a.t.temperature;
    const size_t at = static_cast<size_t>(t) * K;
    const float zy = slot >= 0 ? z[slot] : 0.f;
    float loss = 0.f, lse = 0.f, kd = 0.f, lse_t = 0.f;
    // loss = log(1 + exp(away)), away = log of the sum over all columns but the target, less the target's logit
    if (slot >= 0) {
      float top = rest1;
      for (int j = lane; j < K; j += MOE_WAVE)
        if (j != slot && entry_there(a.t.ids[at + j], a.t.logits[at + j], a.V)) top = fmaxf(top, z[j]);
      top = wave_max_of(top);
      float sum = 0.f;
      for (int j = lane; j < K; j += MOE_WAVE)
        if (j != slot && entry_there(a.t.ids[at + j], a.t.logits[at + j], a.V)) sum += expf(z[j] - top);
      sum = wave_sum_of(sum);
      const float away = top > NONE ? top + logf(sum + expf(rest1 - top)) - zy : NONE;
      loss = fmaxf(away, 0.f) + log1pf(expf(-fabsf(away)));
      lse = loss + zy;
    }
    // With b_j = z_j / tau - log q_j on the entries, b their mean under q, u_j = b_j - b, and R the sum over the columns that are no entry:
    // kd = log(R e^-b + sum q e^u), where sum q e^u = 1 + sum q (e^u - 1 - u) tells a student that is nearly the teacher from the teacher
    if (K > 0) {
      const float lq = teacher_lse(a.t, at, a.V, lane);
      float mean = 0.f;
      for (int j = lane; j < K; j += MOE_WAVE) {
        if (!entry_there(a.t.ids[at + j], a.t.logits[at + j], a.V)) continue;
        const float log_q = a.t.logits[at + j] / tau - lq;
        mean += expf(log_q) * (z[j] / tau - log_q);
      }
      mean = wave_sum_of(mean);
      float rest = rest2;
      if (slot == K) {                                                   // the target is no entry
        const float b = zy / tau, top = fmaxf(rest, b);
        rest = top + logf(expf(rest - top) + expf(b - top));
      }
      float far = rest - mean, sum = 0.f;
      for (int j = lane; j < K; j += MOE_WAVE) {
        if (!entry_there(a.t.ids[at + j], a.t.logits[at + j], a.V)) continue;
        const float log_q = a.t.logits[at + j] / tau - lq, u = z[j] / tau - log_q - mean;
        far = fmaxf(far, u);
        sum += expf(log_q) * (expm1f(fminf(u, 80.f)) - u);
      }
      far = wave_max_of(far);
      sum = wave_sum_of(sum);
      if (far < 40.f) {
        kd = log1pf(expf(rest - mean) + sum);
      } else {                                                           // the same with the largest term in front
        sum = 0.f;
        for (int j = lane; j < K; j += MOE_WAVE) {
          if (!entry_there(a.t.ids[at + j], a.t.logits[at + j], a.V)) continue;
          sum += expf(z[j] / tau - mean - far);                          // q e^u
        }
        kd = far + logf(expf(rest - mean - far) + wave_sum_of(sum));
      }
      lse_t = kd + mean;
      if (!(lq > NONE)) kd = lse_t = 0.f;                                // no entry
    }
    if (lane == 0) {
      a.loss[t] = loss;
      a.lse[t] = lse;
      if (K > 0) { a.kd[t] = kd; a.lse_t[t] = lse_t; }
    }
  }
}

struct HeadPatchArgs {
  const int32_t *offsets, *row_token, *target, *target_slot;
  const float* z_item;
  Teacher t;
  const float *loss, *lse, *lse_t, *dloss, *dkd;
  moe_bf16* dz;
  int ld, V, v0, v1;               // columns v0 to v1 are in dz
};
// The gradient where it is no plain softmax: at the target and at the entries, from their logits.  p - 1 at the target is exp(-loss) - 1, p - q at an
// entry q (exp(log p - log q) - 1).  A wave takes a row.
__global__ __launch_bounds__(256) void head_patch_kernel(HeadPatchArgs a) {
  const int row = blockIdx.x * 4 + threadIdx.x / MOE_WAVE, lane = threadIdx.x % MOE_WAVE;
  if (row >= a.offsets[1]) return;
  const int t = a.row_token[row], slot = a.target_slot[row], K = a.t.K, y = a.target[t];
  const size_t at = static_cast<size_t>(t) * K;
  const float* z = a.z_item + static_cast<size_t>(row) * (K + 1);
  const float tau = a.t.temperature, at_target = slot >= 0 ? expm1f(-a.loss[t]) * a.dloss[t] : 0.f;
  moe_bf16* out = a.dz + static_cast<size_t>(row) * a.ld;
  const float lq = K > 0 ? teacher_lse(a.t, at, a.V, lane) : 0.f;
  const bool taught = K > 0 && lq > -__builtin_inff();
  const float gk = taught ? a.dkd[t] / tau : 0.f, lt = taught ? a.lse_t[t] : 0.f;
  for (int j = lane; j < K; j += MOE_WAVE) {
    const int id = a.t.ids[at + j];
    if (!entry_there(id, a.t.logits[at + j], a.V) || id < a.v0 || id >= a.v1) continue;
    const float log_q = a.t.logits[at + j] / tau - lq;
    float g = expf(log_q) * expm1f(z[j] / tau - lt - log_q) * gk;
    if (id == y) g += at_target;
    else if (slot >= 0) g = __builtin_fmaf(expf(z[j] - a.lse[t]), a.dloss[t], g);
    out[id - a.v0] = f32_to_bf16(g);
  }
  if (slot == K && lane == 0 && y >= a.v0 && y < a.v1) {
    float g = at_target;
    if (taught) g = __builtin_fmaf(expf(z[K] / tau - lt), gk, g);
    out[y - a.v0] = f32_to_bf16(g);
  }
}

// dx of a token: the parts' sums in their order, rounded once; zeros without a loss.
__global__ __launch_bounds__(256) void head_dx_kernel(const float* __restrict__ part, int parts, const int32_t* __restrict__ token_row, int T, int d,
                                                      moe_bf16* __restrict__ dx) {
  const int pieces = d / 8;
  const size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<size_t>(T) * pieces) return;
  const int t = static_cast<int>(i / pieces), c = static_cast<int>(i - static_cast<size_t>(t) * pieces) * 8, row = token_row[t];
  f32x4_t v[2] = {};
  if (row >= 0) {
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const float* q = part + (static_cast<size_t>(p) * T + row) * d + c;
      v[0] += *reinterpret_cast<const f32x4_t*>(q);
      v[1] += *reinterpret_cast<const f32x4_t*>(q + 4);
    }
  }
  typedef __attribute__((ext_vector_type(4))) uint32_t u4;
  *reinterpret_cast<u4*>(dx + static_cast<size_t>(t) * d + c) =
      u4{pack_bf16(v[0][0], v[0][1]), pack_bf16(v[0][2], v[0][3]), pack_bf16(v[1][0], v[1][1]), pack_bf16(v[1][2], v[1][3])};
}

// ---- host ---------------------------------------------------------------------------------------------------------------------

bool bad_head_dims(int T, int d, int V, int K) {
  return T <= 0 || d <= 0 || d % 64 != 0 || d > (1 << 20) || V <= 0 || V > HEAD_MAX_V || K < 0 || K > HEAD_MAX_K ||
         static_cast<long long>(T) * (K + 1) > 0x7FFFFFFFll / 2 || T > (1 << 26);
}
// Columns of a piece of the vocabulary in the backward pass: what the caller asks for, or as many as keep the logits' gradient under 2 GiB.
int head_piece(int T, int V, int asked) {
  const int whole = (V + 63) & ~63;
  if (asked > 0) return asked < whole ? asked : whole;
  const long long most = (1ll << 30) / T & ~2047ll;
  return most >= whole ? whole : static_cast<int>(most < 2048 ? 2048 : most);
}
// The edge of a product's tiles and (HEAD_DX) the parts of its reduction, by the model of gemm_tile.h on the compute units that the workspace is
// laid out for.
template <int S> double head_time(double tiles, double steps, double fixed) {
  const double rounds = tiles / (HEAD_CUS * Tile<S>::PER_CU);
  const double whole = static_cast<double>(static_cast<long long>(rounds + 0.95));
  const double each = fixed + TileCost<S>::STEP * steps;
  return (0.5 * rounds + 0.5 * (whole < 1.0 ? 1.0 : whole)) * each;
}
struct HeadShape { int edge, parts; };
template <int S> void head_parts(int T, int d, int cols, double& best, HeadShape& shape) {
  const double tiles = static_cast<double>(ceil_div(T, S)) * ceil_div(d, S);
  const int steps = ceil_div(cols, BK);
  for (int p = 1; p <= 64 && (p == 1 || steps / p >= 4); ++p) {
    // each part's sums are written and read: T d 8 bytes at some 4 bytes per compute unit and cycle
    const double time = head_time<S>(tiles * p, static_cast<double>(steps) / p, TileCost<S>::FIXED) + p * (static_cast<double>(T) * d / 4.0e6);
    if (time < best) { best = time; shape = {S, p}; }
  }
}
HeadShape head_dx_shape(int T, int d, int cols) {
  HeadShape shape{128, 1};
  double best = 1e300;
  head_parts<256>(T, d, cols, best, shape);
  head_parts<128>(T, d, cols, best, shape);
  return shape;
}
template <int S> double head_plain_time(int rows, int cols, int depth, double fixed) {
  return head_time<S>(static_cast<double>(ceil_div(rows, S)) * ceil_div(cols, S), ceil_div(depth, BK), fixed);
}
int head_edge(int rows, int cols, int depth, double more256, double more128) {
  return head_plain_time<128>(rows, cols, depth, TileCost<128>::FIXED + more128) <
                 head_plain_time<256>(rows, cols, depth, TileCost<256>::FIXED + more256) ? 128 : 256;
}

// What the workspace holds, by offset.
struct HeadLayout {
  size_t offsets, mask, row_token, token_row, target_slot, xc, list_start, items, z_item, row, big, bytes;
  int strips64, blocks, slots;
};
HeadLayout head_layout(int T, int d, int V, int K) {
  HeadLayout l{};
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t p = at; at += (bytes + 255) & ~static_cast<size_t>(255); return p; };
  const size_t n = T;
  l.strips64 = (V + 63) / 64;
  l.blocks = (T + 15) / 16;
  l.slots = K + 1;
  l.offsets = take(8);
  l.mask = take((n + 63) / 64 * 8);
  l.row_token = take(4 * n);
  l.token_row = take(4 * n);
  l.target_slot = take(4 * n);
  l.xc = take(2 * n * d);
  l.list_start = take(static_cast<size_t>(l.blocks) * (l.strips64 + 1) * 4);
  l.items = take(static_cast<size_t>(l.blocks) * 16 * l.slots * sizeof(HeadItem));
  l.z_item = take(n * l.slots * 4);
  l.row = take(16 * n);
  l.big = l.bytes = at;
  return l;
}
size_t head_part_bytes(int T, int V) { return static_cast<size_t>(3) * ((V + 63) / 64) * T * sizeof(float); }
size_t head_dz_bytes(int T, int piece) { return (static_cast<size_t>(T) * ((piece + 63) & ~63) * 2 + 255) & ~static_cast<size_t>(255); }

struct HeadCall {
  const moe_bf16 *x, *W;
  const int32_t* target;
  Teacher t;
  int T, d, V;
  float *loss, *lse, *kd, *lse_t;                                  // forward: out
  const float *in_loss, *in_lse, *in_lse_t, *dloss, *dkd;          // backward
  moe_bf16 *dx, *dW;
  char* ws;
  hipStream_t s;
};

int run_prep(const HeadCall& c, const HeadLayout& l) {
  uint64_t* mask = nullptr;
  if (c.t.K > 0 || c.T > SELF_MASK_TOKENS) {
    mask = reinterpret_cast<uint64_t*>(c.ws + l.mask);
    MOE_LAUNCH("head_mask", head_mask_kernel, dim3((c.T + 255) / 256), dim3(256), 0, c.s, c.target, c.t, c.T, c.V, mask);
  }
  HeadPrepArgs p{};
  p.x = c.x; p.target = c.target; p.t = c.t; p.mask = mask; p.T = c.T; p.d = c.d; p.V = c.V; p.strips = l.strips64;
  p.offsets = reinterpret_cast<int32_t*>(c.ws + l.offsets);
  p.row_token = reinterpret_cast<int32_t*>(c.ws + l.row_token);
  p.token_row = reinterpret_cast<int32_t*>(c.ws + l.token_row);
  p.target_slot = reinterpret_cast<int32_t*>(c.ws + l.target_slot);
  p.xc = reinterpret_cast<moe_bf16*>(c.ws + l.xc);
  p.list_start = reinterpret_cast<int32_t*>(c.ws + l.list_start);
  p.items = reinterpret_cast<HeadItem*>(c.ws + l.items);
  p.loss = c.loss; p.lse = c.lse; p.kd = c.kd; p.lse_t = c.lse_t;
  p.in_loss = c.in_loss; p.in_lse = c.in_lse; p.in_lse_t = c.in_lse_t; p.dloss = c.dloss; p.dkd = c.dkd;
  p.row = c.dx != nullptr ? reinterpret_cast<f32x4_t*>(c.ws + l.row) : nullptr;
  const int lds = (l.strips64 + 1) * 4;
  static bool configured[MAX_DEVICES] = {};
  if (configure_lds(&head_prep_kernel, (HEAD_MAX_V / 64 + 1) * 4, configured) != MOE_OK) return MOE_ERR_LAUNCH;
  MOE_LAUNCH("head_prep", head_prep_kernel, dim3(l.blocks), dim3(256), lds, c.s, p);
  return moe_check_launch();
}

void fill_head(const HeadCall& c, const HeadLayout& l, GemmArgs& a, HeadArgs& h) {
  a.offsets = reinterpret_cast<const int32_t*>(c.ws + l.offsets);
  a.E = 1;
  h.list_start = reinterpret_cast<const int32_t*>(c.ws + l.list_start);
  h.items = reinterpret_cast<const HeadItem*>(c.ws + l.items);
  h.z_item = reinterpret_cast<float*>(c.ws + l.z_item);
  h.row = reinterpret_cast<const f32x4_t*>(c.ws + l.row);
  h.c1 = LOG2E;
  h.c2 = LOG2E / c.t.temperature;
  h.two = c.t.K > 0 && c.t.temperature != 1.f;
  h.rows_cap = c.T;
  h.list_ld = l.strips64 + 1;
  h.slots = l.slots;
}
template <int MODE> int launch_head(GemmArgs& a, const HeadArgs& h, int edge, int rows, int cols, const char* name, hipStream_t s) {
  a.n_tiles = ceil_div(cols, edge);
  a.m_tiles_cap = ceil_div(rows, edge);
  const long long tiles = static_cast<long long>(a.n_tiles) * a.m_tiles_cap * a.E;
  if (tiles > 0x7FFFFFFFll / 2) return MOE_ERR_INVALID;
  return edge == 128 ? launch_gemm_head<MODE, 128>(a, h, tiles, s, name) : launch_gemm_head<MODE, 256>(a, h, tiles, s, name);
}

int run_head_fwd(const HeadCall& c) {
  const HeadLayout l = head_layout(c.T, c.d, c.V, c.t.K);
  int rc = run_prep(c, l);
  if (rc != MOE_OK) return rc;
  GemmArgs a{};
  HeadArgs h{};
  fill_head(c, l, a, h);
  a.A0 = reinterpret_cast<const uint16_t*>(c.ws + l.xc); a.B0 = c.W; a.K = c.d; a.N = c.V;
  const int edge = head_edge(c.T, c.V, c.d, 6.0, 3.0);
  h.strips = ceil_div(c.V, edge / 2);
  h.part = reinterpret_cast<float*>(c.ws + l.big);
  if ((rc = launch_head<HEAD_STATS>(a, h, edge, c.T, c.V, "gemm_head_stats", c.s)) != MOE_OK) return rc;
  const HeadJoinArgs j{h.part, a.offsets, reinterpret_cast<const int32_t*>(c.ws + l.row_token), reinterpret_cast<const int32_t*>(c.ws + l.target_slot),
                       h.z_item, c.t, h.strips, c.T, c.V, c.loss, c.lse, c.kd, c.lse_t, h.c1, h.c2};
  MOE_LAUNCH("head_join", head_join_kernel, dim3(l.blocks), dim3(256), 0, c.s, j);
  return moe_check_launch();
}

int run_head_bwd(const HeadCall& c, int v_piece) {
  const HeadLayout l = head_layout(c.T, c.d, c.V, c.t.K);
  const int piece = head_piece(c.T, c.V, v_piece);
  uint16_t* dz = reinterpret_cast<uint16_t*>(c.ws + l.big);
  float* part = reinterpret_cast<float*>(c.ws + l.big + head_dz_bytes(c.T, piece));
  int rc = run_prep(c, l);
  if (rc != MOE_OK) return rc;
  const HeadShape dxs = head_dx_shape(c.T, c.d, piece);
  int parts = 0;
  for (int v0 = 0; v0 < c.V; v0 += piece) {
    const int cols = c.V - v0 < piece ? c.V - v0 : piece, ld = (cols + 63) & ~63;
    GemmArgs a{};
    HeadArgs h{};
    fill_head(c, l, a, h);
    h.col0 = v0;
    const uint16_t* W = c.W + static_cast<size_t>(v0) * c.d;
    a.A0 = reinterpret_cast<const uint16_t*>(c.ws + l.xc); a.B0 = W; a.O0 = dz; a.K = c.d; a.N = cols; a.M = ld;
    rc = launch_head<HEAD_DZ>(a, h, head_edge(c.T, cols, c.d, 6.0, 3.0), c.T, cols, "gemm_head_dz", c.s);
    if (rc != MOE_OK) return rc;
    const HeadPatchArgs p{a.offsets, reinterpret_cast<const int32_t*>(c.ws + l.row_token), c.target, reinterpret_cast<const int32_t*>(c.ws + l.target_slot),
                          h.z_item, c.t, c.in_loss, c.in_lse, c.in_lse_t, c.dloss, c.dkd, dz, ld, c.V, v0, v0 + cols};
    MOE_LAUNCH("head_patch", head_patch_kernel, dim3((c.T + 3) / 4), dim3(256), 0, c.s, p);
    if ((rc = moe_check_launch()) != MOE_OK) return rc;
    GemmArgs b{};
    b.offsets = a.offsets;
    b.A0 = dz; b.B0 = W; b.O0 = reinterpret_cast<uint16_t*>(part); b.K = ld; b.M = cols; b.N = c.d;
    b.E = dxs.parts < ld / 64 ? dxs.parts : ld / 64;
    if (v0 == 0) parts = b.E;
    h.add = v0 > 0;
    if ((rc = launch_head<HEAD_DX>(b, h, dxs.edge, c.T, c.d, "gemm_head_dx", c.s)) != MOE_OK) return rc;
    GemmArgs w{};
    w.offsets = a.offsets; w.E = 1;
    w.A0 = dz; w.B0 = a.A0; w.O0 = c.dW + static_cast<size_t>(v0) * c.d; w.M = ld; w.K = cols; w.N = c.d;
    rc = launch_head<HEAD_DW>(w, h, head_edge(cols, c.d, c.T, 0.8, 1.1), cols, c.d, "gemm_head_dw", c.s);
    if (rc != MOE_OK) return rc;
  }
  const size_t n = static_cast<size_t>(c.T) * (c.d / 8);
  MOE_LAUNCH("head_dx", head_dx_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, c.s, static_cast<const float*>(part), parts,
             reinterpret_cast<const int32_t*>(c.ws + l.token_row), c.T, c.d, c.dx);
  return moe_check_launch();
}

bool bad_ptrs(std::initializer_list<const void*> needed) {
  for (const void* p : needed) if (p == nullptr || !moe_aligned16(p)) return true;
  return false;
}
bool bad_temperature(float t) { return !(t > 0.f) || !(t < __builtin_inff()); }

}  // namespace

extern "C" size_t moe_head_fwd_workspace_bytes(int T, int d, int V, int K) {
  if (bad_head_dims(T, d, V, K)) return 0;
  return head_layout(T, d, V, K).bytes + head_part_bytes(T, V);
}

extern "C" size_t moe_head_bwd_workspace_bytes(int T, int d, int V, int K, int v_piece) {
  if (bad_head_dims(T, d, V, K) || v_piece < 0 || v_piece % 256 != 0) return 0;
  const int piece = head_piece(T, V, v_piece);
  return head_layout(T, d, V, K).bytes + head_dz_bytes(T, piece) + static_cast<size_t>(head_dx_shape(T, d, piece).parts) * T * d * sizeof(float);
}

extern "C" int moe_head_ce_fwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, int T, int d, int V, float* loss, float* lse,
                               void* ws, size_t ws_bytes, void* stream) {
  if (bad_head_dims(T, d, V, 0) || bad_ptrs({x, W, target, loss, lse, ws})) return MOE_ERR_INVALID;
  if (ws_bytes < moe_head_fwd_workspace_bytes(T, d, V, 0)) return MOE_ERR_WORKSPACE;
  HeadCall c{};
  c.x = x; c.W = W; c.target = target; c.t = {nullptr, nullptr, 1.f, 0}; c.T = T; c.d = d; c.V = V; c.loss = loss; c.lse = lse;
  c.ws = static_cast<char*>(ws); c.s = static_cast<hipStream_t>(stream);
  return run_head_fwd(c);
}

extern "C" int moe_head_ce_bwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const float* loss, const float* lse,
                               const float* dloss, int T, int d, int V, int v_piece, moe_bf16* dx, moe_bf16* dW, void* ws, size_t ws_bytes,
                               void* stream) {
  if (bad_head_dims(T, d, V, 0) || v_piece < 0 || v_piece % 256 != 0) return MOE_ERR_INVALID;
  if (bad_ptrs({x, W, target, loss, lse, dloss, dx, dW, ws})) return MOE_ERR_INVALID;
  if (ws_bytes < moe_head_bwd_workspace_bytes(T, d, V, 0, v_piece)) return MOE_ERR_WORKSPACE;
  HeadCall c{};
  c.x = x; c.W = W; c.target = target; c.t = {nullptr, nullptr, 1.f, 0}; c.T = T; c.d = d; c.V = V;
  c.in_loss = loss; c.in_lse = lse; c.dloss = dloss; c.dx = dx; c.dW = dW;
  c.ws = static_cast<char*>(ws); c.s = static_cast<hipStream_t>(stream);
  return run_head_bwd(c, v_piece);
}

extern "C" int moe_head_distill_fwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const int32_t* ids, const float* teacher,
                                    float temperature, int T, int d, int V, int K, float* loss, float* lse, float* kd, float* lse_t, void* ws,
                                    size_t ws_bytes, void* stream) {
  if (bad_head_dims(T, d, V, K) || K == 0 || bad_temperature(temperature)) return MOE_ERR_INVALID;
  if (bad_ptrs({x, W, target, ids, teacher, loss, lse, kd, lse_t, ws})) return MOE_ERR_INVALID;
  if (ws_bytes < moe_head_fwd_workspace_bytes(T, d, V, K)) return MOE_ERR_WORKSPACE;
  HeadCall c{};
  c.x = x; c.W = W; c.target = target; c.t = {ids, teacher, temperature, K}; c.T = T; c.d = d; c.V = V;
  c.loss = loss; c.lse = lse; c.kd = kd; c.lse_t = lse_t;
  c.ws = static_cast<char*>(ws); c.s = static_cast<hipStream_t>(stream);
  return run_head_fwd(c);
}

extern "C" int moe_head_distill_bwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const int32_t* ids, const float* teacher,
                                    float temperature, const float* loss, const float* lse, const float* lse_t, const float* dloss,
                                    const float* dkd, int T, int d, int V, int K, int v_piece, moe_bf16* dx, moe_bf16* dW, void* ws,
                                    size_t ws_bytes, void* stream) {
  if (bad_head_dims(T, d, V, K) || K == 0 || bad_temperature(temperature) || v_piece < 0 || v_piece % 256 != 0) return MOE_ERR_INVALID;
  if (bad_ptrs({x, W, target, ids, teacher, loss, lse, lse_t, dloss, dkd, dx, dW, ws})) return MOE_ERR_INVALID;
  if (ws_bytes < moe_head_bwd_workspace_bytes(T, d, V, K, v_piece)) return MOE_ERR_WORKSPACE;
  HeadCall c{};
  c.x = x; c.W = W; c.target = target; c.t = {ids, teacher, temperature, K}; c.T = T; c.d = d; c.V = V;
  c.in_loss = loss; c.in_lse = lse; c.in_lse_t = lse_t; c.dloss = dloss; c.dkd = dkd; c.dx = dx; c.dW = dW;
  c.ws = static_cast<char*>(ws); c.s = static_cast<hipStream_t>(stream);
  return run_head_bwd(c, v_piece);
}
