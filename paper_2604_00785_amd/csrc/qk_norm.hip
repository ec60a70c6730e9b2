// Norm of every head's queries and keys, and the rotation by position, in one pass, and its derivative.  For a head's row x of D columns, r = 1 / sqrt(mean(x^2) + eps):
//   v = x r w;   (a, b) -> (a cos t - b sin t, a sin t + b cos t) on R columns of v, t = pos freq[i];   the other columns of v stay
//   dv = the gradient turned back;   g = dv w;   dx = r (g - x r^2 mean(g x));   dw = sum over tokens and heads of dv x r
// Bound by memory: every element is read once and written once (8192 tokens of 32 + 8 heads of 128 columns: forward 33 us, 5.1 TB/s, backward 46, 5.4; a large copy runs
// at 4.9 TB/s).  A thread has 16 columns of a head, both of every pair among them, so that nothing passes between
// threads but a row's sums; a few threads share a head, and a workgroup's threads take the heads of one or a few tokens, whose angles are formed once, in 64 bits
// (a position of 10^6 times a frequency in 32 bits is off by 0.06), and kept in LDS.
#include <initializer_list>
#include <type_traits>
#include "common.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int QK_MAX_D = 512, QK_THREADS = 256;

struct QkSide {
  const moe_bf16 *x, *dy;              // dy: of the backward pass
  const float* w;
  moe_bf16* out;                       // y, or dx
  long long x_ld, dy_ld, out_ld;       // elements from a token to the next
  int H;
};
struct QkArgs {
  QkSide q, k;
  const int32_t* pos;
  const float* freq;
  float* part;                         // backward: [gridDim.x][2][D], a workgroup's share of dw
  int T, D, R, pairs;
  float eps;
};

__device__ __forceinline__ void unpack16(const u32x4& a, const u32x4& b, float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16lo(a[i]); v[2 * i + 1] = bf16hi(a[i]);
    v[8 + 2 * i] = bf16lo(b[i]); v[8 + 2 * i + 1] = bf16hi(b[i]);
  }
}
__device__ __forceinline__ u32x4 pack_half(const float (&v)[16], int at) {
  return u32x4{pack_bf16(v[at], v[at + 1]), pack_bf16(v[at + 2], v[at + 3]), pack_bf16(v[at + 4], v[at + 5]), pack_bf16(v[at + 6], v[at + 7])};
}
// (Ordinary loads: queries and keys come straight from their projection, gradients from the attention, and the caches have most of them.)
__device__ __forceinline__ u32x4 load8(const moe_bf16* p) { return *reinterpret_cast<const u32x4*>(p); }
// Where a thread's two pieces of 8 columns begin.  Rotated pieces first: as halves i and i + R / 16, as neighbours 2 i and 2 i + 1; then the others, two and two.
struct Place { int a, b; bool turned, has_a, has_b; };
__device__ __forceinline__ Place place_of(int i, int D, int R, bool pairs) {
  const bool turned = i < R / 16;
  const int a = turned && !pairs ? i : 2 * i, b = turned && !pairs ? i + R / 16 : 2 * i + 1;
  return {8 * a, 8 * b, turned, 8 * a < D, 8 * b < D};
}
// The thread's pairs turned by its angles (sign -1: back).  Neighbours: pair j is (2 j, 2 j + 1) of the 16; halves: (j, j + 8).
template <bool PAIRS> __device__ __forceinline__ void turn(float (&v)[16], const float (&c)[8], const float (&s)[8], float sign) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    constexpr int NEXT = PAIRS ? 1 : 8;
    const int at = PAIRS ? 2 * j : j;
    const float a = v[at], b = v[at + NEXT], sn = sign * s[j];
    v[at] = __builtin_fmaf(a, c[j], -(b * sn));
    v[at + NEXT] = __builtin_fmaf(a, sn, b * c[j]);
  }
}

// TPR threads to a head, N tokens to a workgroup at a time.
template <int TPR, int N, bool PAIRS, bool BWD>
__global__ __launch_bounds__(QK_THREADS) void qk_norm_kernel(QkArgs a) {
  constexpr int GROUPS = QK_THREADS / TPR, EACH = GROUPS / N;           // groups of threads, those of a token
  constexpr int AHEAD = 2;                                              // heads requested together
  static_assert(EACH >= 1, "a group for each token");
  __shared__ float angle[2][N][QK_MAX_D / 2];
  __shared__ float share[BWD ? GROUPS * TPR * 17 : 1];
  const int tid = threadIdx.x, i = tid % TPR, group = tid / TPR, slot = group / EACH, mine = group % EACH;
  const Place at = place_of(i, a.D, a.R, PAIRS);
  const float over_D = 1.f / static_cast<float>(a.D);
  float dw[2][16];
  if constexpr (BWD) {
#pragma unroll
    for (int j = 0; j < 16; ++j) dw[0][j] = dw[1][j] = 0.f;
  }
  const int blocks = (a.T + N - 1) / N;
  for (int block = blockIdx.x; block < blocks; block += gridDim.x) {
    const int half = a.R / 2, t = block * N + slot;
    if (block != static_cast<int>(blockIdx.x)) __syncthreads();          // the angles of the tokens before have been read
    for (int j = tid; j < N * half; j += QK_THREADS) {
      const int n = j / half, f = j - n * half, token = block * N + n;
      float s = 0.f, c = 1.f;
      if (token < a.T) {
        const double turns = static_cast<double>(a.pos[token]) * static_cast<double>(a.freq[f]) * 0.15915494309189533577;
        sincospif(static_cast<float>(2.0 * (turns - floor(turns))), &s, &c);
      }
      angle[0][n][f] = c;
      angle[1][n][f] = s;
    }
    __syncthreads();
    float c[8], s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      c[j] = at.turned ? angle[0][slot][8 * i + j] : 1.f;
      s[j] = at.turned ? angle[1][slot][8 * i + j] : 0.f;
    }
    // (Addresses are a base of the workgroup's tokens and 32 bits of a thread's own: qk_tokens() sees to it that these suffice.)
    auto side = [&](const QkSide& x, auto which) __attribute__((always_inline)) {
      constexpr int W = decltype(which)::value;
      float w[16];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int col = h == 0 ? at.a : at.b;
        const bool has = h == 0 ? at.has_a : at.has_b;
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          f32x4_t v = {0.f, 0.f, 0.f, 0.f};
          if (has) v = *reinterpret_cast<const f32x4_t*>(x.w + col + j);
#pragma unroll
          for (int l = 0; l < 4; ++l) w[8 * h + j + l] = v[l];
        }
      }
      const moe_bf16* const xs = x.x + static_cast<long long>(block) * N * x.x_ld;
      const moe_bf16* const gs = BWD ? x.dy + static_cast<long long>(block) * N * x.dy_ld : nullptr;
      moe_bf16* const ys = x.out + static_cast<long long>(block) * N * x.out_ld;
      const uint32_t x0 = slot * static_cast<uint32_t>(x.x_ld), g0 = slot * static_cast<uint32_t>(x.dy_ld), y0 = slot * static_cast<uint32_t>(x.out_ld);
      for (int h0 = mine; h0 < x.H; h0 += AHEAD * EACH) {
        u32x4 xa[AHEAD], xb[AHEAD], ga[AHEAD], gb[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int h = h0 + u * EACH;
          xa[u] = xb[u] = ga[u] = gb[u] = u32x4{0, 0, 0, 0};
          if (h >= x.H) continue;
          const uint32_t head = static_cast<uint32_t>(h * a.D);
          if (at.has_a) xa[u] = load8(xs + (x0 + head + at.a));
          if (at.has_b) xb[u] = load8(xs + (x0 + head + at.b));
          if constexpr (BWD) {
            if (at.has_a) ga[u] = load8(gs + (g0 + head + at.a));
            if (at.has_b) gb[u] = load8(gs + (g0 + head + at.b));
          }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          __builtin_amdgcn_sched_barrier(0);                             // (one head's numbers in registers at a time)
          const int h = h0 + u * EACH;
          if (h >= x.H) continue;                                        // (the same for all threads of a head)
          const uint32_t head = static_cast<uint32_t>(h * a.D);
          float v[16], sum = 0.f;
          unpack16(xa[u], xb[u], v);
#pragma unroll
          for (int j = 0; j < 16; ++j) sum = __builtin_fmaf(v[j], v[j], sum);
          const float r = rsqrtf(__builtin_fmaf(group_sum<TPR>(sum), over_D, a.eps));
          if constexpr (!BWD) {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = v[j] * r * w[j];
            turn<PAIRS>(v, c, s, 1.f);
          } else {
            float g[16], dot = 0.f;
            unpack16(ga[u], gb[u], g);
            turn<PAIRS>(g, c, s, -1.f);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              dw[W][j] = __builtin_fmaf(g[j], v[j] * r, dw[W][j]);
              g[j] *= w[j];
              dot = __builtin_fmaf(g[j], v[j], dot);
            }
            const float k = group_sum<TPR>(dot) * over_D * r * r;
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = r * __builtin_fmaf(-v[j], k, g[j]);
          }
          if (at.has_a) *reinterpret_cast<u32x4*>(ys + (y0 + head + at.a)) = pack_half(v, 0);
          if (at.has_b) *reinterpret_cast<u32x4*>(ys + (y0 + head + at.b)) = pack_half(v, 8);
        }
      }
    };
    if (t < a.T) {
      side(a.q, std::integral_constant<int, 0>{});
      side(a.k, std::integral_constant<int, 1>{});
    }
  }
  if constexpr (BWD) {
    // the groups' shares meet in LDS, in their order (rows of 17 words: no two threads of a wave meet in a bank)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 16; ++j) share[tid * 17 + j] = dw[which][j];
      __syncthreads();
      for (int c = tid; c < TPR * 16; c += QK_THREADS) {
        const int owner = c / 16, j = c % 16;
        const Place o = place_of(owner, a.D, a.R, PAIRS);
        const int col = j < 8 ? o.a + j : o.b + j - 8;
        if (!(j < 8 ? o.has_a : o.has_b)) continue;
        float v = 0.f;
        for (int g = 0; g < GROUPS; ++g) v += share[(g * TPR + owner) * 17 + j];
        a.part[(static_cast<size_t>(blockIdx.x) * 2 + which) * a.D + col] = v;
      }
    }
  }
}

// dwq and dwk: the workgroups' shares, in a fixed order.  32 threads take every 32nd share of eight columns, then meet in LDS.
__global__ __launch_bounds__(256) void qk_dw_kernel(const float* __restrict__ part, int n, int D, float* __restrict__ dwq, float* __restrict__ dwk) {
  __shared__ float s[32][8];
  const int c = threadIdx.x % 8, k = threadIdx.x / 8, col = blockIdx.x * 8 + c;      // of 2 D
  float v = 0.f;
#pragma unroll 8
  for (int i = k; i < n; i += 32) v += part[static_cast<size_t>(i) * 2 * D + col];
  s[k][c] = v;
  __syncthreads();
  if (k != 0) return;
  for (int i = 1; i < 32; ++i) v += s[i][c];
  if (col < D) dwq[col] = v;
  else dwk[col - D] = v;
}

// ---- host ---------------------------------------------------------------------------------------------------------------------

bool bad_qk_dims(int T, int Hq, int Hk, int D) {
  return T <= 0 || T > (1 << 30) || Hq <= 0 || Hk <= 0 || Hq > 4096 || Hk > 4096 || D <= 0 || D % 8 != 0 || D > QK_MAX_D;
}
bool bad_side(const QkSide& s, int T, int D, bool bwd) {
  const long long least = static_cast<long long>(s.H) * D, most = 1ll << 32;
  const auto bad_ld = [&](long long ld) { return ld < least || ld % 8 != 0 || ld > most; };
  if (s.x == nullptr || s.out == nullptr || s.w == nullptr || (bwd && s.dy == nullptr)) return true;
  if (!moe_aligned16(s.x) || !moe_aligned16(s.out) || !moe_aligned16(s.w) || !moe_aligned16(s.dy)) return true;
  if (bad_ld(s.x_ld) || bad_ld(s.out_ld) || (bwd && bad_ld(s.dy_ld))) return true;
  // in place only with the rows where they are
  return (s.out == s.x && s.out_ld != s.x_ld && T > 1) || (bwd && s.out == s.dy && s.out_ld != s.dy_ld && T > 1);
}
bool bad_qk(const QkArgs& a, bool bwd) {
  if (bad_qk_dims(a.T, a.q.H, a.k.H, a.D) || a.R < 0 || a.R > a.D || a.R % 16 != 0 || !(a.eps >= 0.f)) return true;
  if (a.pos == nullptr || !moe_aligned16(a.pos) || (a.R > 0 && a.freq == nullptr) || !moe_aligned16(a.freq)) return true;
  return bad_side(a.q, a.T, a.D, bwd) || bad_side(a.k, a.T, a.D, bwd);
}
template <typename F> void with_threads(int D, F&& f) {
  if (D <= 64) f(std::integral_constant<int, 4>{});
  else if (D <= 128) f(std::integral_constant<int, 8>{});
  else if (D <= 256) f(std::integral_constant<int, 16>{});
  else f(std::integral_constant<int, 32>{});
}
// Tokens to a workgroup, where there are as many: the more, the more heads a thread has for its angles and weights, and the fewer workgroups.  The shape above, us, 1 / 2 / 4 / 8 tokens:
// forward 40 / 36 / 34 / 38, backward 69 / 55 / 50 / 52; 4001 tokens of 24 + 8 heads of 96 columns 20 / 15 / 14 / 14.
constexpr int QK_TOKENS = 4, QK_MANY = 2048;
constexpr int QK_MOST = 1 << 20;                  // workgroups of a launch (it may have 2^32 threads)
constexpr long long QK_NEAR = 1ll << 28;          // elements from a token to the next at most, where a workgroup has several
int qk_tokens(const QkArgs& a) {
  for (const QkSide* s : {&a.q, &a.k})
    for (long long ld : {s->x_ld, s->out_ld, s->dy_ld}) if (ld > QK_NEAR) return 1;
  return a.T >= QK_MANY ? QK_TOKENS : 1;
}
// Workgroups of the backward pass, each with a share of dw.
constexpr int QK_SHARES = 512;
int qk_bwd_groups(int T, int tokens) {
  const int groups = (T + tokens - 1) / tokens;
  return groups < QK_SHARES ? groups : QK_SHARES;
}
template <bool BWD> int launch_qk(const QkArgs& a, const char* name, hipStream_t s) {
  const int tokens = qk_tokens(a);
  const int blocks = (a.T + tokens - 1) / tokens;
  const dim3 grid(BWD ? qk_bwd_groups(a.T, tokens) : blocks < QK_MOST ? blocks : QK_MOST);
  with_threads(a.D, [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value;
    if (tokens == QK_TOKENS) {
      if (a.pairs) MOE_LAUNCH(name, (qk_norm_kernel<TPR, QK_TOKENS, true, BWD>), grid, dim3(QK_THREADS), 0, s, a);
      else MOE_LAUNCH(name, (qk_norm_kernel<TPR, QK_TOKENS, false, BWD>), grid, dim3(QK_THREADS), 0, s, a);
    } else {
      if (a.pairs) MOE_LAUNCH(name, (qk_norm_kernel<TPR, 1, true, BWD>), grid, dim3(QK_THREADS), 0, s, a);
      else MOE_LAUNCH(name, (qk_norm_kernel<TPR, 1, false, BWD>), grid, dim3(QK_THREADS), 0, s, a);
    }
  });
  return moe_check_launch();
}

}  // namespace

extern "C" int moe_qk_norm_rope(const moe_bf16* q, long long q_ld, const moe_bf16* k, long long k_ld, const float* wq, const float* wk, const int32_t* pos,
                                const float* freq, int pairs, float eps, int T, int Hq, int Hk, int D, int R, moe_bf16* qo, long long qo_ld, moe_bf16* ko,
                                long long ko_ld, void* stream) {
  const QkArgs a{{q, nullptr, wq, qo, q_ld, 0, qo_ld, Hq}, {k, nullptr, wk, ko, k_ld, 0, ko_ld, Hk}, pos, freq, nullptr, T, D, R, pairs, eps};
  if (bad_qk(a, false)) return MOE_ERR_INVALID;
  return launch_qk<false>(a, "qk_norm_rope", static_cast<hipStream_t>(stream));
}

extern "C" size_t moe_qk_norm_rope_bwd_workspace_bytes(int T, int Hq, int Hk, int D) {
  if (bad_qk_dims(T, Hq, Hk, D)) return 0;
  return static_cast<size_t>(T < QK_SHARES ? T : QK_SHARES) * 2 * D * sizeof(float);
}

extern "C" int moe_qk_norm_rope_bwd(const moe_bf16* dqo, long long dqo_ld, const moe_bf16* dko, long long dko_ld, const moe_bf16* q, long long q_ld,
                                    const moe_bf16* k, long long k_ld, const float* wq, const float* wk, const int32_t* pos, const float* freq, int pairs,
                                    float eps, int T, int Hq, int Hk, int D, int R, moe_bf16* dq, long long dq_ld, moe_bf16* dk, long long dk_ld, float* dwq,
                                    float* dwk, void* ws, size_t ws_bytes, void* stream) {
  const QkArgs a{{q, dqo, wq, dq, q_ld, dqo_ld, dq_ld, Hq}, {k, dko, wk, dk, k_ld, dko_ld, dk_ld, Hk}, pos, freq, static_cast<float*>(ws), T, D, R, pairs, eps};
  if (bad_qk(a, true) || dwq == nullptr || dwk == nullptr || ws == nullptr || !moe_aligned16(dwq) || !moe_aligned16(dwk) || !moe_aligned16(ws)) return MOE_ERR_INVALID;
  if (ws_bytes < moe_qk_norm_rope_bwd_workspace_bytes(T, Hq, Hk, D)) return MOE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (launch_qk<true>(a, "qk_norm_rope_bwd", s) != MOE_OK) return MOE_ERR_LAUNCH;
  MOE_LAUNCH("qk_dw", qk_dw_kernel, dim3(2 * D / 8), dim3(256), 0, s, static_cast<const float*>(ws), qk_bwd_groups(T, qk_tokens(a)), D, dwq, dwk);
  return moe_check_launch();
}
