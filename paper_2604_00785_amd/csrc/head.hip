// The vocabulary head's losses and their gradients.  With logits z = x W^T of a token, its target y and a teacher's logits l on a few entries:
//   loss = log sum exp z - z_y                                        dz += dloss (softmax z - [y])
//   kd   = sum over entries of q (log q - log p), q = softmax(l / tau), p = softmax(z / tau)     dz += dkd / tau (p - q)
//   dx = dz W;   dW = dz^T x
// The logits are never in memory.  Forward: the product's epilogue leaves a row's maximum and sum of exponentials for every strip of columns, and
// the logits that count by themselves (target, entries); a last kernel joins them.  Backward: the logits once more, their gradient
// rounded to bf16 (the products read it as their operand; half a step is at most 2^-8 of each element, as it is of those of dx and dW themselves), then
// the two products.  What bounds it is the matrix pipe: four products of 2 T V d operations, one of them for the logits a second time, as the two calls share no memory
// but the losses.  dx and dW are 0.0023 of their norm from 64 bits, 0.0017 of it their own rounding and as much that of dz: products of 32-bit
// operands take eight times as long (the plain form), dz in two parts would, by count, take 45 % longer.
//
// us, with the library's products for the same sizes (no losses in them): 8192 tokens, d 2048, V 50304: logits and sums 1220 to 1260 (1350), logits and gradient 1330 to 1390,
// dx and dW 2110 to 2180 (1220 + 1610); all of the training step 4720 to 4940, by card.  The chip is at its power limit there (clock 1.7 to 1.96 GHz, matrix pipe busy 0.61 to 0.82).
// One token: 40 for 206 MB of weights (5.2 TB/s), 57 tokens of d 4096, V 32003 46 for 262 MB (5.7 TB/s).
//
// Tokens without a loss are left out of all products: a first kernel finds the others, copies their rows of x side by side, and lists by blocks of
// 16 rows and strips of 64 columns which logits count by themselves.
#include <initializer_list>
#include "gemm_tile.h"

namespace {

constexpr int HEAD_MAX_V = 1 << 20, HEAD_MAX_K = 1024;
constexpr int HEAD_CUS = 256;                       // what the workspace's size is laid out for
// Without a teacher each workgroup of head_prep finds out by itself which of up to so many tokens have a target; entries are looked through by a
// kernel in front (300 tokens, 20 entries each, d 704, V 14000: training step 103 -> 90 us against doing the same with those)
constexpr int SELF_MASK_TOKENS = 4096;
// Up to these many tokens all are taken for rows, with a loss or not, as the products are one pass over W in any case: a forward pass without a
// teacher then needs no kernel in front (ALL_TOKENS), and with one nothing has to be known of all tokens before the rows are laid out
// (ALL_TAUGHT: 40 tokens, 22 entries each, 21.6 -> 19.2 us; beyond, masked tokens cost more than the kernel: 256, 30 % of them masked, 257 -> 270).
constexpr int ALL_TOKENS = 256, ALL_TAUGHT = 128;
// Up to these many tokens with a loss dW takes what rounding dz loses as well, as further rows of its reduction (and of up to these many tokens dx what
// it loses at the teacher's entries).  The rounding of a token's gradient at its target is one number for a whole row of dW: over many tokens such
// errors average out to the size of dW's own rounding, over a few they need not (84 tokens, 80 % of them masked: 0.0027 of dW's norm, 0.0017 with it).
// Training steps without / with, us: 100 tokens of d 2048, V 50304 216 / 222; 128, 1088, 32003 99 / 105; 90, 320, 500 37 / 39; up to 32 the same, as the
// reduction is padded to 64 rows.
constexpr int LOW_TOKENS = 128;
constexpr float LOG2E = 1.4426950408889634f;

struct Teacher { const int32_t* ids; const float* logits; float temperature; int K; };

__device__ __forceinline__ bool entry_there(int id, float l, int V) { return id >= 0 && id < V && l > -__builtin_inff(); }
__device__ __forceinline__ bool target_there(int y, int V) { return y >= 0 && y < V; }

// Which tokens have a loss, a bit each: a target, or (K > 0) an entry.  A workgroup takes 16 tokens, sixteen threads each.
__global__ __launch_bounds__(256) void head_mask_kernel(const int32_t* __restrict__ target, Teacher t, int T, int V, uint16_t* __restrict__ mask) {
  __shared__ uint32_t bits[4];
  const int tid = threadIdx.x, l16 = tid & 15, token = blockIdx.x * 16 + (tid >> 4);
  bool some = false;
  if (token < T) {
    some = l16 == 0 && target_there(target[token], V);
    const size_t at = static_cast<size_t>(token) * t.K;
#pragma unroll 4
    for (int j = l16; j < t.K; j += 16) {
      const int id = t.ids[at + j];
      const float l = t.logits[at + j];
      some = some || entry_there(id, l, V);
    }
  }
  const uint64_t any = __ballot(some);
  uint32_t four = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) four |= (any >> (16 * k) & 0xFFFFu) != 0 ? 1u << k : 0u;
  if (tid % MOE_WAVE == 0) bits[tid / MOE_WAVE] = four;
  __syncthreads();
  if (tid == 0) mask[blockIdx.x] = static_cast<uint16_t>(bits[0] | bits[1] << 4 | bits[2] << 8 | bits[3] << 12);
}

// What head_prep leaves for the kernels behind it, as integers: rows of the products from 0 to LIVE; those of dW, with the low parts, from 0
// to DW_ROWS; whether x itself holds the rows.
enum { ROWS = 0, LIVE = 1, DW_ROWS = 3, DIRECT = 4, DX_PARTS = 5, CONTROL_INTS = 6 };

// Parts of dx's reduction for `rows` rows, at most `most`: the number with which dx and dW together take least time (head_bwd_time), each part's sums
// being written and read besides (8 bytes an element, 7 MB in the model's unit of time).  Lane p - 1 of a wave weighs p parts.
struct BwdRule { int edge, places, d, steps, most, dw_tiles, dw_parts, low; float fixed, wgrad, step; };
__device__ __forceinline__ float bwd_time_of(const BwdRule& x, int rows, int p) {
  const int tiles = (rows + x.edge - 1) / x.edge * ((x.d + x.edge - 1) / x.edge) * p;
  return head_bwd_time(tiles, x.fixed + x.step * x.steps / p, x.dw_tiles, x.wgrad + 1.1f * x.step * (((x.low ? 2 : 1) * rows + BK - 1) / BK) / x.dw_parts, x.places) +
         p * (static_cast<float>(rows) * x.d / 1.0e6f);
}
__device__ __forceinline__ int dx_parts(const BwdRule& x, int rows, int lane) {
  const int p = lane + 1;
  const float time = bwd_time_of(x, rows, p);
  const uint32_t key = p <= x.most && (p == 1 || x.steps / p >= 4) ? (__float_as_uint(time) & ~63u) | static_cast<uint32_t>(lane) : ~0u;
  return 1 + (group_reduce<MOE_WAVE>(key, [](uint32_t u, uint32_t v) __attribute__((always_inline)) { return u < v ? u : v; }) & 63u);
}

struct HeadPrepArgs {
  const moe_bf16* x;
  const int32_t* target;
  Teacher t;
  const uint64_t* mask;            // null: found here (no teacher), or all
  int all;                         // every token is a row (with a teacher); rows without a loss are zeros
  int T, d, V, strips;             // strips: of 64 columns
  int low;                         // up to so many rows: rows of x twice
  BwdRule dx;
  long long dx_room;               // rows that the parts' sums have room for, together
  int32_t* target_row;             // the rows' targets
  int32_t *control, *row_token, *token_row;
  moe_bf16* xc;
  int32_t* list_start;
  HeadItem* items;
  f32x4_t* terms;                  // backward, as is what follows
  int32_t* target_slot;
  float *loss, *lse, *kd, *lse_t;  // forward: zeros for tokens without a loss
  const float *in_loss, *in_lse, *in_lse_t, *dloss, *dkd;
  f32x4_t* row;
};

// Workgroup (b, 0): rows 16 b to 16 b + 15 of those with a loss, in the order of their tokens; and tokens 16 b to 16 b + 15, if they have none.
// Workgroups (b, 1 ..) help with the rows of x.  Sixteen threads share a row and its entries.  A workgroup behind those of the rows writes down what is
// found for all.  (The kernel is one chain of a few us, and short code is part of that: it is fetched cold.)
__global__ __launch_bounds__(256) void head_prep_kernel(HeadPrepArgs a) {
  extern __shared__ int count[];                     // [strips + 1]
  __shared__ uint64_t own[SELF_MASK_TOKENS / 64];
  __shared__ int wave_sum[4], s_token[16], s_slot[16], s_zero[16];
  const int tid = threadIdx.x, lane = tid % MOE_WAVE, wave = tid / MOE_WAVE;
  const int words = (a.T + 63) / 64, per = (words + 255) / 256, K = a.t.K, V = a.V, slots = K + 1;
  const bool lists = blockIdx.y == 0;
  const uint64_t* mask = a.mask;
  if (mask == nullptr && !a.all) {
    constexpr int WORDS = SELF_MASK_TOKENS / 256;        // of a wave, requested together
    int y[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      const int t = (wave + 4 * i) * 64 + lane;
      y[i] = t < a.T ? a.target[t] : -1;
    }
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      const uint64_t bits = __ballot(target_there(y[i], V));
      if (lane == 0) own[wave + 4 * i] = bits;
    }
    mask = own;
  }
  if (tid < 16) { s_token[tid] = a.all && static_cast<int>(blockIdx.x) * 16 + tid < a.T ? blockIdx.x * 16 + tid : -1; s_slot[tid] = K; }
  if (lists && K > 0) for (int i = tid; i <= a.strips; i += 256) count[i] = 0;
  __syncthreads();
  // rank of each thread's first token among those with a loss
  const int w0 = tid * per < words ? tid * per : words, w1 = w0 + per < words ? w0 + per : words;
  int mine = 0;
  if (!a.all) for (int w = w0; w < w1; ++w) mine += __builtin_popcountll(mask[w]);
  int rank = wave_incl_scan(mine);
  if (lane == 63) wave_sum[wave] = rank;
  __syncthreads();
  int live = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) { rank += w < wave ? wave_sum[w] : 0; live += wave_sum[w]; }
  rank -= mine;
  if (a.all) live = a.T;
  const int first = blockIdx.x * 16;
  const bool low = live <= a.low, direct = a.all ? a.row == nullptr : live == a.T && !low;
  if (blockIdx.x == gridDim.x - 1) {
    if (!lists || wave != 0) return;
    int parts = 1;
    if (a.row != nullptr) {
      BwdRule x = a.dx;
      x.low = low;
      const long long room = live > 0 ? a.dx_room / live : 1;
      x.most = room < 64 ? static_cast<int>(room) : 64;
      parts = dx_parts(x, live > 0 ? live : 1, lane);
    }
    if (lane == 0) {
      a.control[ROWS] = 0; a.control[LIVE] = live;
      a.control[DW_ROWS - 1] = 0; a.control[DW_ROWS] = low ? 2 * live : live;
      a.control[DIRECT] = direct;
      a.control[DX_PARTS] = parts;
    }
    return;
  }
  if (lists && !a.all && tid < 16 && first + tid < a.T) {
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
  if (first >= live || (direct && !lists)) return;
  // the words that hold ranks first to first + 15, a bit a lane
  for (uint64_t hit = __ballot(mine > 0 && rank < first + 16 && rank + mine > first); hit != 0; hit &= hit - 1) {
    const int l = __builtin_ctzll(hit), from = (wave * MOE_WAVE + l) * per, to = from + per < words ? from + per : words;
    int at = wave_lane(rank, l);
    for (int w = from; w < to; ++w) {
      const uint64_t bits = mask[w];
      const int rk = at + __builtin_popcountll(bits & ((1ull << lane) - 1));
      if ((bits >> lane & 1) != 0 && rk >= first && rk < first + 16) s_token[rk - first] = w * 64 + lane;
      at += __builtin_popcountll(bits);
    }
  }
  __syncthreads();
  const int n = live - first < 16 ? live - first : 16;
  const int r = tid >> 4, l16 = tid & 15, t = s_token[r], y = r < n ? a.target[t] : -1;
  if (lists && l16 == 0 && r < n) {
    a.row_token[first + r] = t;
    a.token_row[t] = first + r;
  }
  const bool has = r < n && target_there(y, V);
  float in_loss = 0.f, in_lse = 0.f, in_lse_t = 0.f, gl = 0.f, in_dkd = 0.f;      // requested ahead of the rows
  if (a.row != nullptr && lists && r < n) {
    in_loss = a.in_loss[t]; in_lse = a.in_lse[t]; gl = has ? a.dloss[t] : 0.f;
    if (K > 0) { in_lse_t = a.in_lse_t[t]; in_dkd = a.dkd[t]; }
  }
  if (a.all && !direct) {                                // (not the numbers of a token that counts for nothing)
    bool some = has;
    for (int j = l16; j < (r < n ? K : 0); j += 16) {
      const int id = a.t.ids[static_cast<size_t>(t) * K + j];
      const float l = a.t.logits[static_cast<size_t>(t) * K + j];
      some = some || entry_there(id, l, V);
    }
    const uint64_t any = __ballot(some);
    if (l16 == 0) s_zero[r] = (any >> (lane & 48) & 0xFFFFu) == 0;
    __syncthreads();
  }
  if (!direct && r < n) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u4;
    const bool zero = a.all && s_zero[r];
    const int pieces = a.d / 8, step = 16 * gridDim.y;
    const u4* from = reinterpret_cast<const u4*>(a.x + static_cast<size_t>(t) * a.d);
    u4* to = reinterpret_cast<u4*>(a.xc + static_cast<size_t>(first + r) * a.d);
    u4* again = low ? reinterpret_cast<u4*>(a.xc + static_cast<size_t>(live + first + r) * a.d) : to;
    for (int p0 = l16 + 16 * blockIdx.y; p0 < pieces; p0 += 8 * step) {
      u4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = from[p0 + k * step < pieces ? p0 + k * step : p0];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int p = p0 + k * step;
        if (p >= pieces) break;
        if (zero) v[k] = u4{0, 0, 0, 0};
        to[p] = v[k];
        if (low) again[p] = v[k];
      }
    }
  }
  if (!lists) return;
  const size_t at = static_cast<size_t>(t < 0 ? 0 : t) * K;
  const int mine_K = r < n ? K : 0;
  const float tau = a.t.temperature;
  // The gradient at the target and at the entries, where it is no plain softmax: p - 1 = exp(-loss) - 1 at the target; p - q = q (exp(log p - log q) - 1)
  // at an entry.  What does not depend on the logit is put down here (q by the hardware's exponential: 1e-6 of what is rounded to 2^-8).  Where q is small
  // (below e^-20), q times a number is no way to p: by and by it has few bits, then none.  There the entry's p comes from the row's factors, like any other
  // column's, and q alone stands in its terms; what the difference of the two loses is 1e-6 of e^-20 at most.
  constexpr float SMALL_LOG_Q = -20.f;
  const float at_target = has && a.row != nullptr ? expm1f(-in_loss) * gl : 0.f;
  if (K == 0) {                                          // every row has a target, its only item
    if (l16 == 0 && r < n) {
      a.target_row[first + r] = y;
      if (a.row != nullptr) {
        a.row[first + r] = f32x4_t{in_lse * LOG2E, gl, 0.f, 0.f};
        a.terms[first + r] = f32x4_t{at_target, 0.f, 0.f, 0.f};
      }
    }
    return;
  }
  float top = -__builtin_inff();
#pragma unroll 2
  for (int j = l16; j < mine_K; j += 16) {
    const int id = a.t.ids[at + j];
    const float l = a.t.logits[at + j];
    if (!entry_there(id, l, V)) continue;
    top = fmaxf(top, l);
    if (id == y) atomicMin(&s_slot[r], j);               // the target's logit is that of an entry
    atomicAdd(&count[id >> 6], 1);
  }
  top = group_max<16>(top);
  const bool taught = top > -__builtin_inff();
  __syncthreads();
  const bool own_target = l16 == 0 && has && s_slot[r] == K;
  if (own_target) atomicAdd(&count[y >> 6], 1);
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
  const size_t list = static_cast<size_t>(blockIdx.x) * 16 * slots;
  auto put = [&](int col, int slot, const f32x4_t& term) __attribute__((always_inline)) {   // (the order inside a strip does not matter)
    const int i = atomicAdd(&count[col >> 6], 1);
    a.items[list + i] = HeadItem{static_cast<uint32_t>(r) | static_cast<uint32_t>(col) << 4, static_cast<uint32_t>(slot)};
    if (a.terms != nullptr) a.terms[list + i] = term;
  };
  float lq = 0.f, lt = 0.f, gk = 0.f;
  if (a.terms != nullptr && r < n) {
    if (taught) {
      float e = 0.f;
      for (int j = l16; j < mine_K; j += 16) {
        const float l = a.t.logits[at + j];
        if (entry_there(a.t.ids[at + j], l, V)) e += __builtin_amdgcn_exp2f((l - top) / tau * LOG2E);
      }
      lq = logf(group_sum<16>(e));
      lt = in_lse_t;
      gk = in_dkd / tau;
    }
    if (l16 == 0) {
      const float none = __builtin_inff();
      f32x4_t p = {none, 0.f, none, 0.f};
      if (has) { p[0] = in_lse * LOG2E; p[1] = gl; }
      if (taught) {
        if (tau != 1.f) { p[2] = lt * LOG2E; p[3] = gk; }
        else { if (!has) p[0] = lt * LOG2E; p[1] += gk; }             // one exponential serves both
      }
      a.row[first + r] = p;
    }
  }
  for (int j = l16; j < mine_K; j += 16) {
    const int id = a.t.ids[at + j];
    const float l = a.t.logits[at + j];
    if (!entry_there(id, l, V)) continue;
    f32x4_t term = {};
    if (a.terms != nullptr) {
      const float log_q = (l - top) / tau - lq, of_q = __builtin_amdgcn_exp2f(log_q * LOG2E) * gk;
      term = f32x4_t{id == y ? at_target : 0.f, of_q, lt + log_q, id == y ? 0.f : gl};
      if (log_q < SMALL_LOG_Q) {
        term[0] -= of_q;
        term[1] = term[2] = 0.f;
        if (tau == 1.f) term[3] += gk;                   // (exp(z - lse) is p; otherwise the epilogue adds gk p where term[1] is zero)
      }
    }
    put(id, j, term);
  }
  if (own_target) put(y, K, f32x4_t{at_target, 0.f, 0.f, tau == 1.f ? gk : 0.f});      // (and gk p, as below the least q)
  if (l16 == 0 && r < n) a.target_slot[first + r] = has ? s_slot[r] : -1;
}

__device__ __forceinline__ float wave_sum_of(float v) { return group_sum<MOE_WAVE>(v); }
__device__ __forceinline__ float wave_max_of(float v) { return group_max<MOE_WAVE>(v); }

struct HeadJoinArgs {
  const float* part;
  const int32_t *control, *row_token, *target_slot, *target;   // control null: rows are tokens, all T of them
  int T;
  const float* z_item;
  Teacher t;
  const moe_bf16 *x, *W;
  int d, strips, V;
  float *loss, *lse, *kd, *lse_t;
  float c1, c2;
};
// Four rows of a block of 16 (blockIdx.y: which): their strips' maxima and sums joined by 256 threads, then the losses, a wave for each row with its
// entries in registers (EPL a lane).  Sums of exponentials have the scale 2^E of gemm_tile.h.  (All 16 rows of a block by one workgroup of 1024 threads, us: 57
// tokens of d 4096 11.2 instead of 8.5, 129 with 16 entries 13.3 instead of 9.6; 4096 tokens with 64 entries and V 131072 24.7 instead of 31.)
constexpr int JOIN_THREADS = 256, JOIN_GROUPS = JOIN_THREADS, JOIN_ROWS = JOIN_THREADS / MOE_WAVE;
template <int EPL>
__global__ __launch_bounds__(JOIN_THREADS) void head_join_kernel(HeadJoinArgs a) {
  __shared__ float part[4][JOIN_ROWS][JOIN_GROUPS + 1];
  const int tid = threadIdx.x, lane = tid % MOE_WAVE;
  const int first = blockIdx.x * 16 + blockIdx.y * JOIN_ROWS, live = a.control != nullptr ? a.control[LIVE] : a.T, K = a.t.K;
  const bool two = K > 0 && a.t.temperature != 1.f;
  if (first >= live) return;
  constexpr float NONE = -__builtin_inff(), LOW = -3.0e38f;
  // what belongs to the wave's row is requested first
  const int r = tid / MOE_WAVE, row = first + r < live ? first + r : live - 1;
  const int t = a.control != nullptr ? a.row_token[row] : row;
  const int slot = K > 0 ? a.target_slot[row] : target_there(a.target[t], a.V) ? 0 : -1;
  const float* z = a.z_item + static_cast<size_t>(row) * (K + 1);
  const size_t at = static_cast<size_t>(t) * K;
  // The target's logit stands against the sum over all others, whose errors average out, and its own in the product is that of a chain of d / 32 additions.
  // It is formed anew, in 64 bits: with logits of 100 that are sums over 8192 columns the losses are 5e-6 off instead of 4e-5 (300 tokens, root mean square).  That is a row of x and one of W for
  // every token with a target (us: 57 tokens of d 4096 52.7 -> 53.1, 8192 of d 2048 4920 -> 4930).
  double zy = 0.0;
  if (slot >= 0) {
    const moe_bf16 *xr = a.x + static_cast<size_t>(t) * a.d, *wr = a.W + static_cast<size_t>(a.target[t]) * a.d;
#pragma unroll 4
    for (int c = lane * 8; c < a.d; c += MOE_WAVE * 8) {
      typedef __attribute__((ext_vector_type(4))) uint32_t u4;
      const u4 p = *reinterpret_cast<const u4*>(xr + c), q = *reinterpret_cast<const u4*>(wr + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        zy = __builtin_fma(static_cast<double>(bf16lo(p[i])), static_cast<double>(bf16lo(q[i])), zy);
        zy = __builtin_fma(static_cast<double>(bf16hi(p[i])), static_cast<double>(bf16hi(q[i])), zy);
      }
    }
#pragma unroll
    for (int i = 1; i < MOE_WAVE; i *= 2) zy += __shfl_xor(zy, i);
  }
  const float tau = a.t.temperature;
  bool on[EPL];
  float zj[EPL], l[EPL];                                 // an entry's logit and the teacher's
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int j = lane + i * MOE_WAVE;
    on[i] = j < K && entry_there(a.t.ids[at + j], a.t.logits[at + j], a.V);
    zj[i] = on[i] ? z[j] : 0.f;
    l[i] = on[i] ? a.t.logits[at + j] : NONE;
  }
  {
    const int planes = two ? 3 : 2;
    const float* base = a.part + static_cast<size_t>(blockIdx.x) * a.strips * planes * 16 + blockIdx.y * JOIN_ROWS;
    float e1[4], s1[4], e2[4], s2[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { e1[i] = e2[i] = LOW; s1[i] = s2[i] = 0.f; }
#pragma unroll 2
    for (int s = tid; s < a.strips; s += JOIN_GROUPS) {
      const float* p = base + s * planes * 16;
      const f32x4_t m = *reinterpret_cast<const f32x4_t*>(p), v1 = *reinterpret_cast<const f32x4_t*>(p + 16);
      const f32x4_t v2 = two ? *reinterpret_cast<const f32x4_t*>(p + 32) : f32x4_t{};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f1 = m[i] > NONE ? ceilf(m[i] * a.c1) : LOW, n1 = fmaxf(e1[i], f1);
        s1[i] = s1[i] * __builtin_amdgcn_exp2f(e1[i] - n1) + v1[i] * __builtin_amdgcn_exp2f(f1 - n1);
        e1[i] = n1;
        if (two) {
          const float f2 = m[i] > NONE ? ceilf(m[i] * a.c2) : LOW, n2 = fmaxf(e2[i], f2);
          s2[i] = s2[i] * __builtin_amdgcn_exp2f(e2[i] - n2) + v2[i] * __builtin_amdgcn_exp2f(f2 - n2);
          e2[i] = n2;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      part[0][i][tid] = e1[i]; part[1][i][tid] = s1[i];
      if (two) { part[2][i][tid] = e2[i]; part[3][i][tid] = s2[i]; }
    }
  }
  __syncthreads();
  if (first + r >= live) return;
  // log of the sum over the columns that are no item, less `from`.  The exponents are products with LOG2E as 32 bits have it, so its inverse leads back from them (with log 2
  // a loss would have 1.3e-8 of the logits' size in it; kd, whose terms are differences in 32 bits, does not notice).  A sum is zero where there are no such columns (or all are -infinity); one that is NaN
  // stays NaN, and so does what an item that is NaN or infinite makes of a row without others.  Where a scale 2^E has E of 2^30 or more, the product that
  // E is rounded up from is off by 64 or more, which sums of powers do not bear for long (2^31: zero or infinity): NaN as well.
  const double lost = zy < static_cast<double>(__builtin_inff()) ? 0.0 : static_cast<double>(__builtin_nanf(""));
  auto joined = [&](int h, double from, double unit) __attribute__((always_inline)) {
    float e[JOIN_GROUPS / MOE_WAVE], top = LOW, s = 0.f;
#pragma unroll
    for (int i = 0; i < JOIN_GROUPS / MOE_WAVE; ++i) { e[i] = part[h][r][lane + i * MOE_WAVE]; top = fmaxf(top, e[i]); }
    top = wave_max_of(top);
#pragma unroll
    for (int i = 0; i < JOIN_GROUPS / MOE_WAVE; ++i) s += part[h + 1][r][lane + i * MOE_WAVE] * __builtin_amdgcn_exp2f(e[i] - top);
    s = wave_sum_of(s);
    const float log_s = fabsf(top) < 0x1p30f ? logf(s) : __builtin_nanf("");
    return static_cast<float>((s == 0.f && top == LOW ? static_cast<double>(NONE) : static_cast<double>(top) * unit - from + static_cast<double>(log_s)) + lost);
  };
  const float rest1 = joined(0, zy, 1.0 / static_cast<double>(LOG2E)), rest2 = two ? joined(2, 0.0, 0.693147180559945309) : static_cast<float>(rest1 + zy);     // rest1: less the target's logit
  float loss = 0.f, lse = 0.f, kd = 0.f, lse_t = 0.f;
  // loss = log(1 + exp(away)), away = log of the sum over all columns but the target, less the target's logit
  if (slot >= 0) {
    float away = rest1;
    if (K > 0) {
      float top = rest1, sum = 0.f, far[EPL];
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        far[i] = on[i] && lane + i * MOE_WAVE != slot ? static_cast<float>(zj[i] - zy) : NONE;
        top = fmaxf(top, far[i]);
      }
      top = fmaxf(wave_max_of(top), LOW);                // (a maximum passes over NaN, the sum does not; no other column at all: log 0)
#pragma unroll
      for (int i = 0; i < EPL; ++i) sum += expf(far[i] - top);
      away = top + logf(wave_sum_of(sum) + expf(rest1 - top));
    }
    loss = fmaxf(away, 0.f) + log1pf(expf(-fabsf(away)));
    lse = static_cast<float>(loss + zy);
  }
  // With b_j = z_j / tau - log q_j on the entries, b their mean under q, t_j = z_j / tau - b, u_j = t_j - log q_j, and R the sum over the columns that
  // are no entry: kd = log(R e^-b + sum e^t), where sum e^t = 1 + sum q (e^u - 1 - u) tells a student that is nearly the teacher from the teacher.
  // Logits are taken from their largest before they are divided: the type's lowest value is a logit like others, whatever the temperature.  An entry
  // that is next to nothing to the teacher has a u that says nothing of its e^t = q e^u, which is then formed by itself; q = 0 leaves e^t alone.
  float top = NONE;
#pragma unroll
  for (int i = 0; i < EPL; ++i) top = fmaxf(top, l[i]);
  if (K > 0) top = wave_max_of(top);
  if (top > NONE) {                                      // there is an entry
    float sum = 0.f, mean = 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      l[i] = (l[i] - top) / tau;
      sum += on[i] ? expf(l[i]) : 0.f;
    }
    const float log_sum = logf(wave_sum_of(sum));
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      l[i] -= log_sum;                                   // log q
      const float q = on[i] ? expf(l[i]) : 0.f;
      if (q != 0.f) mean += q * (zj[i] / tau - l[i]);
    }
    mean = wave_sum_of(mean);
    float rest = rest2;
    if (slot == K) {                                     // the target is no entry
      const float zt = static_cast<float>(zy) / tau, m = fmaxf(rest, zt);
      rest = m + logf(expf(rest - m) + expf(zt - m));
    }
    float far = rest - mean;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const float e = zj[i] / tau - mean, u = e - l[i], q = expf(l[i]);
      if (!on[i]) continue;
      far = fmaxf(far, e);
      sum += u < 20.f ? q * (expm1f(u) - u) : expf(e) - (q != 0.f ? q * (1.f + u) : 0.f);
    }
    far = wave_max_of(far);
    sum = wave_sum_of(sum);
    if (far < 40.f) {
      kd = log1pf(expf(rest - mean) + sum);
    } else {                                             // the same with the largest term in front
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) sum += on[i] ? expf(zj[i] / tau - mean - far) : 0.f;
      kd = far + logf(expf(rest - mean - far) + wave_sum_of(sum));
    }
    lse_t = kd + mean;
  }
  if (lane == 0) {
    a.loss[t] = loss;
    a.lse[t] = lse;
    if (K > 0) { a.kd[t] = kd; a.lse_t[t] = lse_t; }
  }
}

__device__ __forceinline__ void store8(moe_bf16* to, const f32x4_t (&v)[2]) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u4;
  *reinterpret_cast<u4*>(to) = u4{pack_bf16(v[0][0], v[0][1]), pack_bf16(v[0][2], v[0][3]), pack_bf16(v[1][0], v[1][1]), pack_bf16(v[1][2], v[1][3])};
}

struct HeadDxArgs {
  const float* part;
  const int32_t* control;
  const int32_t *token_row, *target_slot, *target;
  const float* item;               // what dz lost at the items
  Teacher t;
  const moe_bf16* W;
  int T, d, V;
  moe_bf16* dx;
  const float* dw_part;            // dW's sums, [dw_parts][V][d], if they are in parts
  int dw_parts, dx_groups;         // workgroups from dx_groups on are for them
  moe_bf16* dW;
};
// v += e W[id, c .. c + 7]
__device__ __forceinline__ void add_row(const HeadDxArgs& a, float e, int id, int c, f32x4_t (&v)[2]) {
  typedef __attribute__((ext_vector_type(4))) uint32_t u4;
  const u4 w = *reinterpret_cast<const u4*>(a.W + static_cast<size_t>(id) * a.d + c);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[k >> 1][2 * (k & 1)] = __builtin_fmaf(e, bf16lo(w[k]), v[k >> 1][2 * (k & 1)]);
    v[k >> 1][2 * (k & 1) + 1] = __builtin_fmaf(e, bf16hi(w[k]), v[k >> 1][2 * (k & 1) + 1]);
  }
}
__device__ __forceinline__ void add_parts(const float* part, size_t stride, int parts, f32x4_t (&v)[2]) {
#pragma unroll 4
  for (int p = 0; p < parts; ++p) {
    v[0] += *reinterpret_cast<const f32x4_t*>(part + p * stride);
    v[1] += *reinterpret_cast<const f32x4_t*>(part + p * stride + 4);
  }
}
__device__ __forceinline__ void head_dw_sum(const HeadDxArgs& a) {
  const size_t i = static_cast<size_t>(blockIdx.x - a.dx_groups) * 256 + threadIdx.x, n = static_cast<size_t>(a.V) * (a.d / 8);
  if (i >= n) return;
  f32x4_t v[2] = {};
  add_parts(a.dw_part + i * 8, n * 8, a.dw_parts, v);
  store8(a.dW + i * 8, v);
}
// dx of a token: the parts' sums in their order and what rounding dz took from them at the target, rounded once; zeros without a loss.  And dW
// likewise, where its reduction over the tokens is in parts.
__global__ __launch_bounds__(256) void head_dx_kernel(HeadDxArgs a) {
  if (static_cast<int>(blockIdx.x) >= a.dx_groups) { head_dw_sum(a); return; }
  const int pieces = a.d / 8, K = a.t.K;
  const size_t i = static_cast<size_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<size_t>(a.T) * pieces) return;
  const int t = static_cast<int>(i / pieces), c = static_cast<int>(i - static_cast<size_t>(t) * pieces) * 8, row = a.token_row[t];
  f32x4_t v[2] = {};
  if (row >= 0) {
    const int slot = K > 0 ? a.target_slot[row] : 0, live = a.control[LIVE];
    if (slot >= 0) add_row(a, a.item[static_cast<size_t>(row) * (K + 1) + slot], a.target[t], c, v);
    add_parts(a.part + static_cast<size_t>(row) * a.d + c, static_cast<size_t>(live) * a.d, a.control[DX_PARTS], v);
  }
  store8(a.dx + static_cast<size_t>(t) * a.d + c, v);
}
// The same for a few tokens with a teacher, with what rounding took at the entries too: a workgroup has 256 columns of a token, eight threads share the
// items of eight columns.
constexpr int FEW_PIECES = 32, FEW_SHARES = 256 / FEW_PIECES;
__global__ __launch_bounds__(256) void head_dx_few_kernel(HeadDxArgs a) {
  __shared__ f32x4_t sums[FEW_SHARES][FEW_PIECES][2];
  if (static_cast<int>(blockIdx.x) >= a.dx_groups) { head_dw_sum(a); return; }
  const int wide = (a.d / 8 + FEW_PIECES - 1) / FEW_PIECES, t = blockIdx.x / wide, K = a.t.K;
  const int share = threadIdx.x / FEW_PIECES, piece = threadIdx.x % FEW_PIECES, c = ((blockIdx.x - t * wide) * FEW_PIECES + piece) * 8;
  const int row = a.token_row[t];
  f32x4_t v[2] = {};
  if (row >= 0 && c < a.d) {
    const float* item = a.item + static_cast<size_t>(row) * (K + 1);
    const size_t at = static_cast<size_t>(t) * K;
    if (share == 0 && a.target_slot[row] == K) add_row(a, item[K], a.target[t], c, v);     // (a target that is an entry is among them)
#pragma unroll 4
    for (int j = share; j < K; j += FEW_SHARES) {
      const int id = a.t.ids[at + j];
      const float l = a.t.logits[at + j], e = item[j];
      const bool on = entry_there(id, l, a.V);
      add_row(a, on ? e : 0.f, on ? id : 0, c, v);
    }
  }
  sums[share][piece][0] = v[0];
  sums[share][piece][1] = v[1];
  __syncthreads();
  if (share != 0 || c >= a.d) return;
#pragma unroll
  for (int i = 1; i < FEW_SHARES; ++i) { v[0] += sums[i][piece][0]; v[1] += sums[i][piece][1]; }
  if (row >= 0) add_parts(a.part + static_cast<size_t>(row) * a.d + c, static_cast<size_t>(a.control[LIVE]) * a.d, a.control[DX_PARTS], v);
  store8(a.dx + static_cast<size_t>(t) * a.d + c, v);
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
// The backward products of `cols` columns: their tiles' edge and the parts of either reduction, dW's in more than one only where its tiles do not fill the
// chip, and not in pieces of the vocabulary (`whole`), whose sums would have to be rounded one by one.  The parts of dx are those for all T
// tokens; they are chosen again for the tokens that have a loss, in the room that these leave.
struct BwdShape { int edge, dx_parts, dw_parts; };
template <int S> void weigh_bwd(int T, int d, int cols, int depth, bool whole, double& best, BwdShape& shape) {
  const int places = HEAD_CUS * Tile<S>::PER_CU, wide = ceil_div(d, S), steps = ceil_div(cols, BK), dw_steps = ceil_div(depth, BK);
  const long long dx_tiles = static_cast<long long>(ceil_div(T, S)) * wide, dw_tiles = static_cast<long long>(ceil_div(cols, S)) * wide;
  int q = 1;
  if (whole) while (dw_tiles * (q + 1) <= places && dw_steps / (q + 1) >= 4) ++q;
  constexpr int some[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48, 56, 64};
  for (int p : some) {
    if (p > 1 && (steps / p < 4 || dx_tiles * p > 8ll * places)) break;
    const double time = head_bwd_time(static_cast<int>(dx_tiles * p), head_dx_each<S>(steps, p), static_cast<int>(dw_tiles * q), head_dw_each<S>(dw_steps, q), places) +
                        (static_cast<double>(p) * T + (q > 1 ? static_cast<double>(q) * cols : 0.0)) * d / 1.0e6;
    if (time < best) { best = time; shape = {S, p, q}; }
  }
}
BwdShape head_bwd_shape(int T, int d, int cols, bool whole) {
  BwdShape shape{128, 1, 1};
  double best = 1e300;
  const int depth = T <= LOW_TOKENS ? 2 * T : T;
  // One reduction step of dW, all of it waiting for memory: two workgroups on a compute unit wait better.  256 / 128 in us: 10 tokens, d 2048, V 50304 110 / 94;
  // 8, 2880, 35317 117 / 96; 1, 832, 61930 62 / 50; 22, 1216, 178071 248 / 257.  (100, 2048, 50304: 119 / 118, as the model has it.)
  if (depth > 64) weigh_bwd<256>(T, d, cols, depth, whole, best, shape);
  weigh_bwd<128>(T, d, cols, depth, whole, best, shape);
  return shape;
}
// The logits' products.  Their epilogues take the vector unit, which a tile of 256 leaves idle matrix cores beside and two of 128 share a compute unit for:
// so narrow rows take 128 (more: what the epilogue of a tile of 256 costs beside that of a plain product, 3.0 at 128; K steps of 1.4 us).  256 / 128 in us,
// sums (gradient): 3799 tokens, d 256, V 50524 169 / 160 (215 / 191); 1597, 64, 25439 34 / 29 (48 / 37); 3372, 576, 43471 202 / 197 (239 / 217);
// 1420, 3968, 58453 516 / 728 (541 / 749); 8192, 2048, 50304 1201 / 1535 (1331 / 1736).
int logits_edge(int rows, int cols, int d, double more) {
  const auto time = [&](auto edge, double fixed) {
    constexpr int S = decltype(edge)::value;
    return head_time<S>(static_cast<double>(ceil_div(rows, S)) * ceil_div(cols, S), ceil_div(d, BK), fixed);
  };
  return time(IC<128>{}, TileCost<128>::FIXED + 3.0) < time(IC<256>{}, TileCost<256>::FIXED + more) ? 128 : 256;
}

// What the workspace holds, by offset.
struct HeadLayout {
  size_t control, mask, row_token, token_row, target_row, target_slot, xc, list_start, items, terms, item, row, big;   // terms, row: of the backward pass
  int strips64, blocks, slots, low;
};
// Rows of dz, and of x beside it: those of all tokens, or twice as many as take what rounding loses.
int head_dz_rows(int T) { return T <= LOW_TOKENS ? 2 * T : T < 2 * LOW_TOKENS ? 2 * LOW_TOKENS : T; }
HeadLayout head_layout(int T, int d, int V, int K, bool backward) {
  HeadLayout l{};
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t p = at; at += (bytes + 255) & ~static_cast<size_t>(255); return p; };
  const size_t n = T;
  l.strips64 = (V + 63) / 64;
  l.blocks = (T + 15) / 16;
  l.slots = K + 1;
  l.low = backward ? LOW_TOKENS : 0;
  l.control = take(CONTROL_INTS * 4);
  l.mask = take((n + 63) / 64 * 8);
  l.row_token = take(4 * n);
  l.token_row = take(4 * n);
  l.target_row = take(4 * n);
  l.target_slot = take(4 * n);
  l.xc = take(2 * static_cast<size_t>(backward ? head_dz_rows(T) : T) * d);
  const size_t items = static_cast<size_t>(l.blocks) * 16 * l.slots;
  if (K > 0) {
    l.list_start = take(static_cast<size_t>(l.blocks) * (l.strips64 + 1) * 4);
    l.items = take(items * sizeof(HeadItem));
  }
  l.item = take(n * l.slots * 4);
  if (backward) {
    l.terms = take(items * sizeof(f32x4_t));
    l.row = take(16 * n);
  }
  l.big = at;
  return l;
}
size_t head_part_bytes(int T, int V) { return static_cast<size_t>(3) * ((V + 63) / 64) * ((T + 15) & ~15) * sizeof(float); }
size_t head_dz_bytes(int T, int piece) { return (static_cast<size_t>(head_dz_rows(T)) * ((piece + 63) & ~63) * 2 + 255) & ~static_cast<size_t>(255); }

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

int run_prep(const HeadCall& c, const HeadLayout& l, const BwdRule& dx, long long dx_room) {
  uint64_t* mask = nullptr;
  const bool all = c.t.K > 0 && c.T <= ALL_TAUGHT;
  if (!all && (c.t.K > 0 || c.T > SELF_MASK_TOKENS)) {
    mask = reinterpret_cast<uint64_t*>(c.ws + l.mask);
    MOE_LAUNCH("head_mask", head_mask_kernel, dim3((c.T + 63) / 64 * 4), dim3(256), 0, c.s, c.target, c.t, c.T, c.V,
               reinterpret_cast<uint16_t*>(mask));
  }
  HeadPrepArgs p{};
  p.x = c.x; p.target = c.target; p.t = c.t; p.mask = mask; p.T = c.T; p.d = c.d; p.V = c.V; p.strips = l.strips64;
  p.low = l.low;
  p.all = all;
  p.dx = dx; p.dx_room = dx_room;
  p.target_row = reinterpret_cast<int32_t*>(c.ws + l.target_row);
  p.control = reinterpret_cast<int32_t*>(c.ws + l.control);
  p.row_token = reinterpret_cast<int32_t*>(c.ws + l.row_token);
  p.token_row = reinterpret_cast<int32_t*>(c.ws + l.token_row);
  p.target_slot = reinterpret_cast<int32_t*>(c.ws + l.target_slot);
  p.xc = reinterpret_cast<moe_bf16*>(c.ws + l.xc);
  p.list_start = reinterpret_cast<int32_t*>(c.ws + l.list_start);
  p.items = reinterpret_cast<HeadItem*>(c.ws + l.items);
  p.loss = c.loss; p.lse = c.lse; p.kd = c.kd; p.lse_t = c.lse_t;
  p.in_loss = c.in_loss; p.in_lse = c.in_lse; p.in_lse_t = c.in_lse_t; p.dloss = c.dloss; p.dkd = c.dkd;
  if (c.dx != nullptr) {
    p.terms = reinterpret_cast<f32x4_t*>(c.ws + l.terms);
    p.row = reinterpret_cast<f32x4_t*>(c.ws + l.row);
  }
  const int lds = (l.strips64 + 1) * 4;
  static bool configured[MAX_DEVICES] = {};
  if (configure_lds(&head_prep_kernel, (HEAD_MAX_V / 64 + 1) * 4, configured) != MOE_OK) return MOE_ERR_LAUNCH;
  MOE_LAUNCH("head_prep", head_prep_kernel, dim3(l.blocks + 1, (c.d + 1023) / 1024), dim3(256), lds, c.s, p);
  return moe_check_launch();
}

void fill_head(const HeadCall& c, const HeadLayout& l, GemmArgs& a, HeadArgs& h) {
  const int32_t* control = reinterpret_cast<const int32_t*>(c.ws + l.control);
  a.offsets = control + ROWS;
  a.row_token = control + DIRECT;
  a.E = 1;
  h.target = reinterpret_cast<const int32_t*>(c.ws + l.target_row);
  h.list_start = c.t.K > 0 ? reinterpret_cast<const int32_t*>(c.ws + l.list_start) : nullptr;
  h.items = reinterpret_cast<const HeadItem*>(c.ws + l.items);
  h.item = reinterpret_cast<float*>(c.ws + l.item);
  h.terms = reinterpret_cast<const f32x4_t*>(c.ws + l.terms);
  h.row = reinterpret_cast<const f32x4_t*>(c.ws + l.row);
  h.c1 = LOG2E;
  h.c2 = LOG2E / c.t.temperature;
  h.over_tau = 1.f / c.t.temperature;
  h.two = c.t.K > 0 && c.t.temperature != 1.f;
  h.list_ld = l.strips64 + 1;
  h.slots = l.slots;
}
bool too_many(long long tiles) { return tiles > 0x7FFFFFFFll / 2; }
template <int MODE> int launch_logits(GemmArgs& a, const HeadArgs& h, int edge, int rows, const char* name, hipStream_t s) {
  a.n_tiles = ceil_div(a.N, edge);
  const long long tiles = static_cast<long long>(a.n_tiles) * ceil_div(rows, edge);
  if (too_many(tiles)) return MOE_ERR_INVALID;
  return edge == 128 ? launch_gemm_head<MODE, 128>(a, h, tiles, s, name) : launch_gemm_head<MODE, 256>(a, h, tiles, s, name);
}
// For tests: the edge of a launch's tiles on entry (0: the rule decides), the one that it ran with on return.
int settle_edge(int* edge, int rule) {
  if (edge == nullptr) return rule;
  return *edge = *edge == 0 ? rule : *edge;
}

int run_head_fwd(const HeadCall& c, int* edges) {
  const HeadLayout l = head_layout(c.T, c.d, c.V, c.t.K, false);
  GemmArgs a{};
  HeadArgs h{};
  fill_head(c, l, a, h);
  a.A0 = reinterpret_cast<const uint16_t*>(c.ws + l.xc); a.A1 = c.x; a.B0 = c.W; a.K = c.d; a.N = c.V;
  const bool all = c.t.K == 0 && c.T <= ALL_TOKENS;
  int rc = MOE_OK;
  if (all) {
    a.offsets = nullptr; a.row_token = nullptr; a.A0 = c.x; a.M = c.T;
    h.target = c.target;
  } else if ((rc = run_prep(c, l, BwdRule{}, 0)) != MOE_OK) {
    return rc;
  }
  const int edge = settle_edge(edges, logits_edge(c.T, c.V, c.d, 9.5));
  h.strips = ceil_div(c.V, edge / 2);
  h.part = reinterpret_cast<float*>(c.ws + l.big);
  if ((rc = launch_logits<HEAD_STATS>(a, h, edge, c.T, "gemm_head_stats", c.s)) != MOE_OK) return rc;
  const HeadJoinArgs j{h.part, all ? nullptr : reinterpret_cast<const int32_t*>(c.ws + l.control), reinterpret_cast<const int32_t*>(c.ws + l.row_token),
                       reinterpret_cast<const int32_t*>(c.ws + l.target_slot), c.target, c.T, h.item, c.t, c.x, c.W, c.d, h.strips, c.V, c.loss, c.lse, c.kd, c.lse_t,
                       h.c1, h.c2};
  const dim3 grid(l.blocks, 16 / JOIN_ROWS), block(JOIN_THREADS);
  if (c.t.K <= MOE_WAVE) MOE_LAUNCH("head_join", head_join_kernel<1>, grid, block, 0, c.s, j);
  else if (c.t.K <= 2 * MOE_WAVE) MOE_LAUNCH("head_join", head_join_kernel<2>, grid, block, 0, c.s, j);
  else MOE_LAUNCH("head_join", head_join_kernel<HEAD_MAX_K / MOE_WAVE>, grid, block, 0, c.s, j);
  return moe_check_launch();
}

int run_head_bwd(const HeadCall& c, int v_piece, int* edges) {
  const HeadLayout l = head_layout(c.T, c.d, c.V, c.t.K, true);
  const int piece = head_piece(c.T, c.V, v_piece), wanted = edges != nullptr ? edges[1] : 0;
  uint16_t* dz = reinterpret_cast<uint16_t*>(c.ws + l.big);
  float* part = reinterpret_cast<float*>(c.ws + l.big + head_dz_bytes(c.T, piece));
  BwdShape shape = head_bwd_shape(c.T, c.d, piece, piece >= c.V);
  float* dw_part = part + static_cast<size_t>(shape.dx_parts) * c.T * c.d;
  if (wanted != 0) shape.edge = wanted;
  if (edges != nullptr) edges[1] = shape.edge;
  const int places = HEAD_CUS * 256 / shape.edge, wide = ceil_div(c.d, shape.edge);
  // (the parts are those of all pieces: no more than the smallest, the last, has steps for)
  const int last = c.V - (c.V - 1) / piece * piece;
  const BwdRule rule{shape.edge, places, c.d, ceil_div(last, BK), 0, ceil_div(last, shape.edge) * wide * shape.dw_parts, shape.dw_parts, 0,
                     static_cast<float>(shape.edge == 256 ? TileCost<256>::FIXED : TileCost<128>::FIXED),
                     static_cast<float>(shape.edge == 256 ? TileCost<256>::WGRAD : TileCost<128>::WGRAD),
                     static_cast<float>(shape.edge == 256 ? TileCost<256>::STEP : TileCost<128>::STEP)};
  int rc = run_prep(c, l, rule, static_cast<long long>(shape.dx_parts) * c.T);
  if (rc != MOE_OK) return rc;
  const int32_t* control = reinterpret_cast<const int32_t*>(c.ws + l.control);
  for (int v0 = 0; v0 < c.V; v0 += piece) {
    const int cols = c.V - v0 < piece ? c.V - v0 : piece, ld = (cols + 63) & ~63;
    GemmArgs a{};
    HeadArgs h{};
    fill_head(c, l, a, h);
    h.col0 = v0;
    h.lo = l.low;
    const uint16_t* W = c.W + static_cast<size_t>(v0) * c.d;
    a.A0 = reinterpret_cast<const uint16_t*>(c.ws + l.xc); a.A1 = c.x; a.B0 = W; a.O0 = dz; a.K = c.d; a.N = cols; a.M = ld;
    rc = launch_logits<HEAD_DZ>(a, h, settle_edge(edges, logits_edge(c.T, cols, c.d, 10.8)), c.T, "gemm_head_dz", c.s);
    if (rc != MOE_OK) return rc;
    GemmArgs b{};
    b.offsets = a.offsets; b.row_token = control + DX_PARTS; b.stream_rows = v0 > 0;
    b.A0 = dz; b.B0 = W; b.O0 = reinterpret_cast<uint16_t*>(part); b.K = ld; b.M = cols; b.N = c.d;
    GemmArgs w{};
    w.offsets = control + DW_ROWS - 1; w.E = shape.dw_parts; w.row_token = a.row_token; w.O1 = reinterpret_cast<uint16_t*>(dw_part);
    w.A0 = dz; w.B0 = a.A0; w.B1 = a.A1; w.O0 = c.dW + static_cast<size_t>(v0) * c.d; w.M = ld; w.K = cols; w.N = c.d;
    b.n_tiles = w.n_tiles = wide;
    w.m_tiles_cap = ceil_div(cols, shape.edge);
    const long long dw_tiles = static_cast<long long>(wide) * w.m_tiles_cap * w.E, tiles = dw_tiles + 64ll * ceil_div(c.T, shape.edge) * wide;
    if (too_many(tiles)) return MOE_ERR_INVALID;
    rc = shape.edge == 128 ? launch_gemm_head_bwd<128>(b, w, tiles, c.s, "gemm_head_dx+dw") : launch_gemm_head_bwd<256>(b, w, tiles, c.s, "gemm_head_dx+dw");
    if (rc != MOE_OK) return rc;
  }
  const bool few = c.t.K > 0 && c.T <= LOW_TOKENS;
  const size_t dx_groups = few ? static_cast<size_t>(c.T) * ceil_div(c.d / 8, FEW_PIECES) : (static_cast<size_t>(c.T) * (c.d / 8) + 255) / 256;
  const HeadDxArgs x{part, control, reinterpret_cast<const int32_t*>(c.ws + l.token_row), reinterpret_cast<const int32_t*>(c.ws + l.target_slot), c.target,
                     reinterpret_cast<const float*>(c.ws + l.item), c.t, c.W, c.T, c.d, c.V, c.dx, dw_part, shape.dw_parts, static_cast<int>(dx_groups), c.dW};
  const dim3 groups(static_cast<unsigned>(dx_groups + (shape.dw_parts > 1 ? (static_cast<size_t>(c.V) * (c.d / 8) + 255) / 256 : 0)));
  if (few) MOE_LAUNCH("head_dx", head_dx_few_kernel, groups, dim3(256), 0, c.s, x);
  else MOE_LAUNCH("head_dx", head_dx_kernel, groups, dim3(256), 0, c.s, x);
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
  return head_layout(T, d, V, K, false).big + head_part_bytes(T, V);
}

extern "C" size_t moe_head_bwd_workspace_bytes(int T, int d, int V, int K, int v_piece) {
  if (bad_head_dims(T, d, V, K) || v_piece < 0 || v_piece % 256 != 0) return 0;
  const int piece = head_piece(T, V, v_piece);
  const BwdShape shape = head_bwd_shape(T, d, piece, piece >= V);
  return head_layout(T, d, V, K, true).big + head_dz_bytes(T, piece) +
         (static_cast<size_t>(shape.dx_parts) * T + (shape.dw_parts > 1 ? static_cast<size_t>(shape.dw_parts) * V : 0)) * d * sizeof(float);
}

// Both losses, or (ids null, K 0) the cross entropy alone: what the calls of moe_hotpath.h come to.  edges, for tests: as in gemm.h, of the
// logits' launch, then (backward) of dx and dW together.
namespace {
bool bad_edge_list(const int* edges, int n) {
  for (int i = 0; edges != nullptr && i < n; ++i) if (edges[i] != 0 && edges[i] != 128 && edges[i] != 256) return true;
  return false;
}
}  // namespace
extern "C" int moe_head_fwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const int32_t* ids, const float* teacher, float temperature,
                            int T, int d, int V, int K, float* loss, float* lse, float* kd, float* lse_t, void* ws, size_t ws_bytes, void* stream,
                            int* edges) {
  if (bad_head_dims(T, d, V, K) || bad_temperature(temperature) || bad_edge_list(edges, 1)) return MOE_ERR_INVALID;
  if (bad_ptrs({x, W, target, loss, lse, ws}) || (K > 0 && bad_ptrs({ids, teacher, kd, lse_t}))) return MOE_ERR_INVALID;
  if (ws_bytes < moe_head_fwd_workspace_bytes(T, d, V, K)) return MOE_ERR_WORKSPACE;
  HeadCall c{};
  c.x = x; c.W = W; c.target = target; c.t = {ids, teacher, temperature, K}; c.T = T; c.d = d; c.V = V;
  c.loss = loss; c.lse = lse; c.kd = kd; c.lse_t = lse_t;
  c.ws = static_cast<char*>(ws); c.s = static_cast<hipStream_t>(stream);
  return run_head_fwd(c, edges);
}
extern "C" int moe_head_bwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const int32_t* ids, const float* teacher, float temperature,
                            const float* loss, const float* lse, const float* lse_t, const float* dloss, const float* dkd, int T, int d, int V, int K,
                            int v_piece, moe_bf16* dx, moe_bf16* dW, void* ws, size_t ws_bytes, void* stream, int* edges) {
  if (bad_head_dims(T, d, V, K) || bad_temperature(temperature) || v_piece < 0 || v_piece % 256 != 0 || bad_edge_list(edges, 2)) return MOE_ERR_INVALID;
  if (bad_ptrs({x, W, target, loss, lse, dloss, dx, dW, ws}) || (K > 0 && bad_ptrs({ids, teacher, lse_t, dkd}))) return MOE_ERR_INVALID;
  if (ws_bytes < moe_head_bwd_workspace_bytes(T, d, V, K, v_piece)) return MOE_ERR_WORKSPACE;
  HeadCall c{};
  c.x = x; c.W = W; c.target = target; c.t = {ids, teacher, temperature, K}; c.T = T; c.d = d; c.V = V;
  c.in_loss = loss; c.in_lse = lse; c.in_lse_t = lse_t; c.dloss = dloss; c.dkd = dkd; c.dx = dx; c.dW = dW;
  c.ws = static_cast<char*>(ws); c.s = static_cast<hipStream_t>(stream);
  return run_head_bwd(c, v_piece, edges);
}

extern "C" int moe_head_ce_fwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, int T, int d, int V, float* loss, float* lse,
                               void* ws, size_t ws_bytes, void* stream) {
  return moe_head_fwd(x, W, target, nullptr, nullptr, 1.f, T, d, V, 0, loss, lse, nullptr, nullptr, ws, ws_bytes, stream, nullptr);
}

extern "C" int moe_head_ce_bwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const float* loss, const float* lse,
                               const float* dloss, int T, int d, int V, int v_piece, moe_bf16* dx, moe_bf16* dW, void* ws, size_t ws_bytes,
                               void* stream) {
  return moe_head_bwd(x, W, target, nullptr, nullptr, 1.f, loss, lse, nullptr, dloss, nullptr, T, d, V, 0, v_piece, dx, dW, ws, ws_bytes, stream, nullptr);
}

extern "C" int moe_head_distill_fwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const int32_t* ids, const float* teacher,
                                    float temperature, int T, int d, int V, int K, float* loss, float* lse, float* kd, float* lse_t, void* ws,
                                    size_t ws_bytes, void* stream) {
  if (K <= 0) return MOE_ERR_INVALID;
  return moe_head_fwd(x, W, target, ids, teacher, temperature, T, d, V, K, loss, lse, kd, lse_t, ws, ws_bytes, stream, nullptr);
}

extern "C" int moe_head_distill_bwd(const moe_bf16* x, const moe_bf16* W, const int32_t* target, const int32_t* ids, const float* teacher,
                                    float temperature, const float* loss, const float* lse, const float* lse_t, const float* dloss,
                                    const float* dkd, int T, int d, int V, int K, int v_piece, moe_bf16* dx, moe_bf16* dW, void* ws,
                                    size_t ws_bytes, void* stream) {
  if (K <= 0) return MOE_ERR_INVALID;
  return moe_head_bwd(x, W, target, ids, teacher, temperature, loss, lse, lse_t, dloss, dkd, T, d, V, K, v_piece, dx, dW, ws, ws_bytes, stream, nullptr);
}
