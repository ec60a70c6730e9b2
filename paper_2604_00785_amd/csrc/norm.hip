// Residual addition and root-mean-square norm in front of a layer, its result in bfloat16 or in 8 bits with scales, and its
// derivative.  With s = x + r (rounded to bf16: what the residual stream holds is what is normalised), q = 1 / sqrt(mean(s^2) + eps):
//   y = s q w;      8 bits: scale = max |y| / 448 over each group of columns, codes = y / scale = 448 s w / max |s w| in e4m3
//   c = mean(dy w s) q^2;   dx = dr = dsum + q (dy w - s c);   dw = sum over rows of dy s q
// All of it is bound by memory: a row is read once, kept in registers between the sum and its use, and written once.
#include <climits>
#include <type_traits>
#include "common.h"

namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr int NORM_MAX_D = 32768;
constexpr float E4M3_MAX = 448.f;

struct NormArgs {
  const moe_bf16 *x, *r;       // r may be null: s = x
  const float* w;
  moe_bf16 *sum, *y;           // sum may be null where r is
  uint8_t* codes;
  float *scale, *rstd;         // rstd may be null
  int T, d, lanes;             // lanes: threads that share a scale (d / 8 or more: the whole row)
  float eps;
};

__device__ __forceinline__ void unpack8(const u32x4& p, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = bf16lo(p[i]); v[2 * i + 1] = bf16hi(p[i]); }
}
__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  return u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}
// Rows are read once and long after they were written, or by nobody else soon: non-temporal loads leave the caches to what is
// written.  One pass over other rows each time, us, ordinary -> non-temporal: 8192 x 2048 forward 30.7 -> 28.2 (4.8 TB/s), 8 bits 31.9 -> 27.4;
// 4001 x 4096 28.3 -> 24.8 (5.3 TB/s), 26.3 -> 24.3; the backward's rows take 2 to 3 us of some 30 less too.
__device__ __forceinline__ u32x4 load8(const moe_bf16* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }

// Reduction over the TPR threads of a row: inside the waves by lane permutations, across them through LDS.
template <int TPR, typename Op> __device__ __forceinline__ uint32_t row_reduce(uint32_t v, Op op, uint32_t* part) {
  v = group_reduce<TPR < MOE_WAVE ? TPR : MOE_WAVE>(v, op);
  if constexpr (TPR > MOE_WAVE) {
    __syncthreads();                              // what was there before has been read
    if (threadIdx.x % MOE_WAVE == 0) part[threadIdx.x / MOE_WAVE] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < TPR / MOE_WAVE; ++i) v = op(v, part[i]);
  }
  return v;
}
template <int TPR> __device__ __forceinline__ float row_sum(float v, uint32_t* part) {
  return __uint_as_float(row_reduce<TPR>(__float_as_uint(v), [](uint32_t a, uint32_t b) __attribute__((always_inline)) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }, part));
}
// Maximum of absolute values by their bits, which order as the values do and put NaN above everything, so that it is passed on.
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// A row by TPR threads, P pieces of 8 columns each: thread i of the row takes pieces i, i + TPR, ..
template <int TPR, int P, bool CODES>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void add_rms_norm_kernel(NormArgs a) {
  constexpr int ROWS = TPR > 256 ? 1 : 256 / TPR;
  __shared__ uint32_t part[TPR > MOE_WAVE ? TPR / MOE_WAVE : 1];
  const int row = blockIdx.x * ROWS + threadIdx.x / TPR, i0 = threadIdx.x % TPR;
  if (row >= a.T) return;                         // all of a row's threads, and only where no barrier follows
  const int pieces = a.d / 8;
  const size_t at = static_cast<size_t>(row) * a.d;
  float s[P][8];
  u32x4 xp[P], rp[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = i0 + p * TPR;
    xp[p] = rp[p] = u32x4{0, 0, 0, 0};
    if (i < pieces) {
      xp[p] = load8(a.x + at + 8 * i);
      if (a.r != nullptr) rp[p] = load8(a.r + at + 8 * i);
    }
  }
  float q = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = i0 + p * TPR;
    u32x4 total = xp[p];
    if (a.r != nullptr) {
      float xv[8], rv[8];
      unpack8(xp[p], xv);
      unpack8(rp[p], rv);
#pragma unroll
      for (int c = 0; c < 8; ++c) xv[c] += rv[c];
      total = pack8(xv);
    }
    unpack8(total, s[p]);
    if (i < pieces && a.sum != nullptr) *reinterpret_cast<u32x4*>(a.sum + at + 8 * i) = total;
#pragma unroll
    for (int c = 0; c < 8; ++c) q = __builtin_fmaf(s[p][c], s[p][c], q);
  }
  q = rsqrtf(row_sum<TPR>(q, part) / static_cast<float>(a.d) + a.eps);
  if (a.rstd != nullptr && i0 == 0) a.rstd[row] = q;
  if constexpr (!CODES) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int i = i0 + p * TPR;
      if (i >= pieces) continue;
      const f32x4_t w0 = *reinterpret_cast<const f32x4_t*>(a.w + 8 * i), w1 = *reinterpret_cast<const f32x4_t*>(a.w + 8 * i + 4);
#pragma unroll
      for (int c = 0; c < 8; ++c) s[p][c] = s[p][c] * q * (c < 4 ? w0[c] : w1[c - 4]);
      *reinterpret_cast<u32x4*>(a.y + at + 8 * i) = pack8(s[p]);
    }
  } else {
    // A code is a step of 2^-4: a quotient next to a border goes to the wrong side when its own roundings add up.  So it is formed from the exact
    // product s w (v and low), the exact largest one (m and off) and 448 over that in two parts (factor and rest), rounded once.  It does not depend
    // on q, which only says whether there is a number at all.  (None of 16 million codes of 4001 x 4096 differ from 64 bits', 5 to 16 do if y itself is divided by
    // its scale.)
    float w[P][8];
    uint32_t top = 0;
    const bool whole = a.lanes >= pieces;         // one scale for the row
    const auto amax_of = [&](int p, uint32_t most) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < 8; ++c) most = umax(most, __float_as_uint(s[p][c] * w[p][c]) & 0x7FFFFFFFu);
      return most;
    };
    // how far the largest product is above its rounding m: no other one is
    const auto above = [&](int p, float m, float most) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < 8; ++c) most = fmaxf(most, __builtin_fmaf(fabsf(s[p][c]), fabsf(w[p][c]), -m));
      return most;
    };
    const auto larger = [](uint32_t u, uint32_t v) __attribute__((always_inline)) {
      return __float_as_uint(fmaxf(__uint_as_float(u), __uint_as_float(v)));
    };
    // over the threads that share a scale
    const auto shared = [&](uint32_t v, auto op) __attribute__((always_inline)) {
      if (a.lanes >= 2) v = op(v, dpp_u32<0xB1>(v));
      if (a.lanes >= 4) v = op(v, dpp_u32<0x4E>(v));
      if (a.lanes >= 8) v = op(v, dpp_u32<0x141>(v));
      if (a.lanes >= 16) v = op(v, dpp_u32<0x140>(v));
      if (a.lanes >= 32) { const auto e = __builtin_amdgcn_permlane16_swap(v, v, false, false); v = op(e[0], e[1]); }
      if (a.lanes >= 64) { const auto e = __builtin_amdgcn_permlane32_swap(v, v, false, false); v = op(e[0], e[1]); }
      return v;
    };
    constexpr float LEAST = -3.4028235e38f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int i = i0 + p * TPR;
      f32x4_t w0{}, w1{};
      if (i < pieces) { w0 = *reinterpret_cast<const f32x4_t*>(a.w + 8 * i); w1 = *reinterpret_cast<const f32x4_t*>(a.w + 8 * i + 4); }
#pragma unroll
      for (int c = 0; c < 8; ++c) w[p][c] = c < 4 ? w0[c] : w1[c - 4];
    }
    float row_above = LEAST;
    if (whole) {
#pragma unroll
      for (int p = 0; p < P; ++p) top = amax_of(p, top);
      top = row_reduce<TPR>(top, umax, part);
#pragma unroll
      for (int p = 0; p < P; ++p) row_above = above(p, __uint_as_float(top), row_above);
      row_above = __uint_as_float(row_reduce<TPR>(__float_as_uint(row_above), larger, part));
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int i = i0 + p * TPR;
      uint32_t amax = top;
      float off = row_above;
      if (!whole) {
        amax = shared(amax_of(p, 0), umax);
        off = __uint_as_float(shared(__float_as_uint(above(p, __uint_as_float(amax), LEAST)), larger));
      }
      if (i >= pieces) continue;
      const float m = __uint_as_float(amax);
      // (far from the ends of the range only; where 448 / m is not finite the largest number instead, which leaves zeros zeros)
      const bool fine = m > 0x1p-100f && m < 0x1p100f;
      const float factor = m != 0.f ? fminf(E4M3_MAX / m, 3.4028235e38f) : 0.f, nothing = 0.f * q;
      const float rest = fine ? (__builtin_fmaf(-factor, m, E4M3_MAX) - factor * off) * (factor * (1.f / E4M3_MAX)) : 0.f, low_factor = fine ? factor : 0.f;
      float z[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const float v = __builtin_fmaf(s[p][c], w[p][c], nothing), low = __builtin_fmaf(s[p][c], w[p][c], -v);
        z[c] = __builtin_fmaf(v, factor, __builtin_fmaf(v, rest, low * low_factor));      // at most 448 and a bit, which rounds to 448
      }
      u32x2 o;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int b = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * h], z[4 * h + 1], 0, false);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * h + 2], z[4 * h + 3], b, true);
        o[h] = static_cast<uint32_t>(b);
      }
      *reinterpret_cast<u32x2*>(a.codes + at + 8 * i) = o;
      const int groups = whole ? 1 : pieces / a.lanes;
      if (whole ? i == 0 : i % a.lanes == 0) a.scale[static_cast<size_t>(row) * groups + (whole ? 0 : i / a.lanes)] = m * q * (1.f / E4M3_MAX);
    }
  }
}

struct NormBwdArgs {
  const moe_bf16 *dy, *dsum, *sum;   // dsum may be null
  const float *w, *rstd;
  moe_bf16* dx;
  float* part;                       // [gridDim.x][d]: a workgroup's share of dw
  int T, d;
};
// The workgroup's rows are blockIdx.x * ROWS + .., in steps of the whole grid; a thread keeps its columns' sums of dw over them.
template <int TPR, int P>
__global__ __launch_bounds__(TPR > 256 ? TPR : 256) void add_rms_norm_bwd_kernel(NormBwdArgs a) {
  constexpr int ROWS = TPR > 256 ? 1 : 256 / TPR;
  __shared__ uint32_t part[TPR > MOE_WAVE ? TPR / MOE_WAVE : 1];
  __shared__ float share[ROWS > 1 ? (ROWS - 1) * P * 8 * TPR : 1];
  const int first = ROWS == 1 ? blockIdx.x : blockIdx.x * ROWS + threadIdx.x / TPR, i0 = ROWS == 1 ? threadIdx.x : threadIdx.x % TPR;
  const int pieces = a.d / 8;
  // The next row's pieces are requested before this row's are used, but for rows of 1024 threads, which have 128 registers each: those are for this row, and each
  // thread keeps its weights in LDS (and forms dw with dx, when the row's sum has come).  All in registers, with the next row, went to memory and back, us:
  // 1000 x 16384 47.6 -> 34.2, 500 x 32768 120 -> 38.5, 4000 x 32768 861 -> 211 (5.0 TB/s).
  constexpr bool AHEAD = TPR < 1024;
  __shared__ f32x4_t own_w[AHEAD ? 1 : P * 2 * TPR];
  float dw[P][8];
  f32x4_t kept[P][2];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = i0 + p * TPR;
#pragma unroll
    for (int c = 0; c < 8; ++c) dw[p][c] = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      kept[p][h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (i < pieces) kept[p][h] = *reinterpret_cast<const f32x4_t*>(a.w + 8 * i + 4 * h);
      if constexpr (!AHEAD) own_w[(2 * p + h) * TPR + i0] = kept[p][h];
    }
  }
  auto weights = [&](int p, float (&v)[8]) __attribute__((always_inline)) {
    if constexpr (!AHEAD) {
      asm volatile("" ::: "memory");                      // (read here, not in front of the rows or of the pieces before)
      kept[p][0] = own_w[2 * p * TPR + i0];
      kept[p][1] = own_w[(2 * p + 1) * TPR + i0];
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = kept[p][c / 4][c % 4];
  };
  struct Row { u32x4 g[P], s[P], a[P]; float q; };
  auto load = [&](int row, Row& x) __attribute__((always_inline)) {
    const size_t at = static_cast<size_t>(row < a.T ? row : a.T - 1) * a.d;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int i = i0 + p * TPR;
      x.g[p] = x.s[p] = x.a[p] = u32x4{0, 0, 0, 0};
      if (i < pieces) {
        x.g[p] = load8(a.dy + at + 8 * i);
        x.s[p] = load8(a.sum + at + 8 * i);
        if (a.dsum != nullptr) x.a[p] = load8(a.dsum + at + 8 * i);
      }
    }
    x.q = a.rstd[row < a.T ? row : a.T - 1];
  };
  const int step = gridDim.x * ROWS;
  Row now, next;
  if constexpr (AHEAD) load(first, now);
  for (int row = first; row < a.T; row += step) {                 // (the same for all threads of a row)
    if constexpr (!AHEAD) load(row, now);
    else if (row + step < a.T) load(row + step, next);
    const size_t at = static_cast<size_t>(row) * a.d;
    const u32x4 (&gp)[P] = now.g, (&sp)[P] = now.s, (&ap)[P] = now.a;
    auto unpacked_here = [&](int p) __attribute__((always_inline)) {
      if constexpr (!AHEAD) asm volatile("" : "+v"(now.g[p]), "+v"(now.s[p]), "+v"(now.a[p]));
    };
    const float q = now.q;
    float dot = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      float g[8], s[8], w[8];
      unpacked_here(p);
      unpack8(gp[p], g);
      unpack8(sp[p], s);
      weights(p, w);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        dot = __builtin_fmaf(g[c] * w[c], s[c], dot);
        if constexpr (AHEAD) dw[p][c] = __builtin_fmaf(g[c], s[c] * q, dw[p][c]);
      }
    }
    const float k = row_sum<TPR>(dot, part) / static_cast<float>(a.d) * q * q;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int i = i0 + p * TPR;
      float g[8], s[8], w[8], v[8];
      unpacked_here(p);                                   // (again, not kept over the row's sum)
      unpack8(gp[p], g);
      unpack8(sp[p], s);
      unpack8(ap[p], v);
      weights(p, w);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        v[c] = __builtin_fmaf(q, __builtin_fmaf(-s[c], k, g[c] * w[c]), v[c]);
        if constexpr (!AHEAD) dw[p][c] = __builtin_fmaf(g[c], s[c] * q, dw[p][c]);
      }
      if (i < pieces) *reinterpret_cast<u32x4*>(a.dx + at + 8 * i) = pack8(v);
    }
    if constexpr (AHEAD) now = next;
  }
  // the shares of the workgroup's rows meet in LDS, in the order of the rows
  if constexpr (ROWS > 1) {
    const int mine = threadIdx.x / TPR;
    if (mine > 0) {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int c = 0; c < 8; ++c) share[((mine - 1) * P * 8 + p * 8 + c) * TPR + i0] = dw[p][c];
    }
    __syncthreads();
    if (mine > 0) return;
#pragma unroll
    for (int m = 0; m < ROWS - 1; ++m)
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int c = 0; c < 8; ++c) dw[p][c] += share[(m * P * 8 + p * 8 + c) * TPR + i0];
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = i0 + p * TPR;
    if (i >= pieces) continue;
    float* o = a.part + static_cast<size_t>(blockIdx.x) * a.d + 8 * i;
    *reinterpret_cast<f32x4_t*>(o) = f32x4_t{dw[p][0], dw[p][1], dw[p][2], dw[p][3]};
    *reinterpret_cast<f32x4_t*>(o + 4) = f32x4_t{dw[p][4], dw[p][5], dw[p][6], dw[p][7]};
  }
}

// dw[c] = sum of the n shares, in a fixed order: 32 threads take every 32nd share of four columns, then meet in LDS.
__global__ __launch_bounds__(256) void norm_dw_kernel(const float* __restrict__ part, int n, int d, float* __restrict__ dw) {
  __shared__ f32x4_t s[32][8];
  const int c = threadIdx.x % 8, k = threadIdx.x / 8, col = (blockIdx.x * 8 + c) * 4;
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  if (col < d) {
#pragma unroll 16
    for (int i = k; i < n; i += 32) v += *reinterpret_cast<const f32x4_t*>(part + static_cast<size_t>(i) * d + col);
  }
  s[k][c] = v;
  __syncthreads();
  if (k == 0 && col < d) {
#pragma unroll
    for (int i = 1; i < 32; ++i) v += s[i][c];
    *reinterpret_cast<f32x4_t*>(dw + col) = v;
  }
}

bool bad_norm_dims(int T, int d) { return T <= 0 || d <= 0 || d % 8 != 0 || d > NORM_MAX_D; }
int rows_of_group(int d) { return d <= 256 ? 16 : d <= 2048 ? 4 : 1; }
// Threads of a row: 16 up to 256 columns, one wave up to 2048 (no barrier in the row's sums), 256 up to 8192, else 1024.
template <typename F> void with_shape(int d, F&& f) {
  const int pieces = d / 8;
#define MOE_NORM(TPR) \
  switch ((pieces + TPR - 1) / TPR) { \
    case 1: f(std::integral_constant<int, TPR>{}, std::integral_constant<int, 1>{}); break; \
    case 2: f(std::integral_constant<int, TPR>{}, std::integral_constant<int, 2>{}); break; \
    case 3: f(std::integral_constant<int, TPR>{}, std::integral_constant<int, 3>{}); break; \
    default: f(std::integral_constant<int, TPR>{}, std::integral_constant<int, 4>{}); break; \
  }
  if (pieces <= 32) { MOE_NORM(16) } else if (pieces <= 256) { MOE_NORM(64) } else if (pieces <= 1024) { MOE_NORM(256) } else { MOE_NORM(1024) }
#undef MOE_NORM
}
// Workgroups of the backward pass, each with a share of dw: two per compute unit of a whole chip, one where a share is long, or as many as there are
// rows for.  us with 256 / 512 / 1024: 8192 x 2048 32.8 / 29.8 / 34.3, 4001 x 4096 34.5 / 29.4 / 32.0, 2000 x 8192 34.6 / 33.3 / 41.0, 1500 x 12288 37.9 / 42.2 / 51.3,
// 500 x 32768 38.8 / 52.1 / 52.3, 16384 x 136 13.1 / 11.2 / 14.1.
int norm_bwd_groups(int T, int d) {
  const int rows = rows_of_group(d), groups = (T - 1) / rows + 1, most = d <= 4096 ? 512 : 256;
  if (groups <= 4) return 1;                      // its share is dw: a few more rows in turn take less than another launch
  return groups < most ? groups : most;
}

template <bool CODES> int launch_norm(const NormArgs& a, const char* name, hipStream_t s) {
  const dim3 grid((a.T - 1) / rows_of_group(a.d) + 1);
  with_shape(a.d, [&](auto tpr, auto p) {
    constexpr int TPR = decltype(tpr)::value, P = decltype(p)::value;
    MOE_LAUNCH(name, (add_rms_norm_kernel<TPR, P, CODES>), grid, dim3(TPR > 256 ? TPR : 256), 0, s, a);
  });
  return moe_check_launch();
}

}  // namespace

extern "C" int moe_add_rms_norm(const moe_bf16* x, const moe_bf16* r, const float* w, int T, int d, float eps, moe_bf16* sum,
                                moe_bf16* y, float* rstd, void* stream) {
  if (!x || !w || !y || (r && !sum) || bad_norm_dims(T, d) || !(eps >= 0.f)) return MOE_ERR_INVALID;
  const void* ptrs[] = {x, r, w, sum, y, rstd};
  for (const void* p : ptrs) if (!moe_aligned16(p)) return MOE_ERR_INVALID;
  const NormArgs a{x, r, w, sum, y, nullptr, nullptr, rstd, T, d, 0, eps};
  return launch_norm<false>(a, "add_rms_norm", static_cast<hipStream_t>(stream));
}

extern "C" int moe_add_rms_norm_8bit(const moe_bf16* x, const moe_bf16* r, const float* w, int T, int d, float eps, int group,
                                     moe_bf16* sum, uint8_t* codes, float* scale, float* rstd, void* stream) {
  if (!x || !w || !codes || !scale || (r && !sum) || bad_norm_dims(T, d) || !(eps >= 0.f)) return MOE_ERR_INVALID;
  // a scale's columns are whole pieces of 8, a power of two of them up to a wave, or the row
  if (group != 0 && (group < 8 || group > 512 || (group & (group - 1)) != 0 || d % group != 0)) return MOE_ERR_INVALID;
  const void* ptrs[] = {x, r, w, sum, codes, scale, rstd};
  for (const void* p : ptrs) if (!moe_aligned16(p)) return MOE_ERR_INVALID;
  const NormArgs a{x, r, w, sum, nullptr, codes, scale, rstd, T, d, group == 0 ? INT_MAX : group / 8, eps};
  return launch_norm<true>(a, "add_rms_norm_8bit", static_cast<hipStream_t>(stream));
}

extern "C" size_t moe_add_rms_norm_bwd_workspace_bytes(int T, int d) {
  if (bad_norm_dims(T, d)) return 0;
  return static_cast<size_t>(norm_bwd_groups(T, d)) * d * sizeof(float);
}

extern "C" int moe_add_rms_norm_bwd(const moe_bf16* dy, const moe_bf16* dsum, const moe_bf16* sum, const float* w, const float* rstd,
                                    int T, int d, moe_bf16* dx, float* dw, void* ws, size_t ws_bytes, void* stream) {
  if (!dy || !sum || !w || !rstd || !dx || !dw || !ws || bad_norm_dims(T, d)) return MOE_ERR_INVALID;
  const void* ptrs[] = {dy, dsum, sum, w, rstd, dx, dw, ws};
  for (const void* p : ptrs) if (!moe_aligned16(p)) return MOE_ERR_INVALID;
  if (ws_bytes < moe_add_rms_norm_bwd_workspace_bytes(T, d)) return MOE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int groups = norm_bwd_groups(T, d);
  const NormBwdArgs a{dy, dsum, sum, w, rstd, dx, groups == 1 ? dw : static_cast<float*>(ws), T, d};
  with_shape(d, [&](auto tpr, auto p) {
    constexpr int TPR = decltype(tpr)::value, P = decltype(p)::value;
    MOE_LAUNCH("add_rms_norm_bwd", (add_rms_norm_bwd_kernel<TPR, P>), dim3(groups), dim3(TPR > 256 ? TPR : 256), 0, s, a);
  });
  if (moe_check_launch() != MOE_OK) return MOE_ERR_LAUNCH;
  if (groups == 1) return MOE_OK;
  MOE_LAUNCH("norm_dw", norm_dw_kernel, dim3((d / 4 + 7) / 8), dim3(256), 0, s, static_cast<const float*>(ws), groups, d, dw);
  return moe_check_launch();
}
