// What the products of the vocabulary head leave for its scores, and the kernel that joins it.
#pragma once
#include "common.h"

// HEAD_TOP: what a row has in a wave's HALF columns.  A lane's HALF / 4 of them (16 j + 4 l + c for lane l of four) have their largest logit apart; the others' sums, of all
// four lanes together, are relative to 2^E, E the row's largest logit here in units of log2 rounded up, as in HEAD_STATS: sum = sum 2^t, moment = sum t 2^t, t <= 0.
// next: the second largest of the lane's columns rounded up, as an integer in the order of the numbers, whose low bits are the largest one's place (4 j + c).
struct HeadTop { float top; uint32_t next; };
struct HeadStrip { HeadTop lane[4]; float sum, moment; };
// The same where no alternatives are wanted: the strip's largest logit, its column in the strip, and the sums of all others.
struct HeadBest { float top; uint32_t column; float sum, moment; };
__host__ __device__ __forceinline__ uint32_t ordered_u32(uint32_t bits) { return bits ^ ((bits >> 31) != 0 ? 0xFFFFFFFFu : 0x80000000u); }

constexpr int SCORE_MAX_K = 64, SCORE_SPARE = 4;
constexpr int score_wanted(int K) { return K > 0 ? K + SCORE_SPARE : 1; }       // logits that are formed anew

struct ScoreJoinArgs {
  const void* part;                                // HeadStrip, or (K 0) HeadBest [row][strips], or (whole) the logits' `parts` summands [part][T][score_ld(V)]
  const int32_t *control, *token_row, *target;     // control null: rows are tokens
  const moe_bf16 *x, *W;
  int T, d, V, K, strips, whole, parts;
  float c1;                                        // log2(e) over the temperature
  double over_tau;
  float *logp, *entropy, *lse;
  int32_t* ids;
  float* top;
  // of the backward pass (K 0, strips; else null): the first sure_rows[0] rows alone, of which it leaves log2 p of the likeliest column, of_row[row][3]
  const int32_t *sure_rows, *row_token;
  f32x4_t* of_row;
};

// Whether a logit's gradient is formed apart, with the terms of its row: if that is a SURE one (the last term is 0 or less) and the column has more than half of p.  The
// products leave NaN there.
__device__ __forceinline__ bool score_apart(float z, float c1, const f32x4_t& row) { return row[3] <= 0.f && __builtin_fmaf(z, c1, -row[0]) > -1.f; }

constexpr int SCORE_WHOLE_V = 16384;
constexpr int score_ld(int V) { return (V + 3) & ~3; }
// edge: of the tiles that the strips are from (HALF = edge / 2)
int moe_head_score_join(const ScoreJoinArgs& a, int edge, hipStream_t s);

// The logits' gradient from their summands, as HEAD_SCORE_DZ has it: dz [rows][ld], and behind it (up to `low` rows) what rounding it loses; item [row]: that of the target's.
struct ScoreDzArgs {
  const float* part;                               // [part][T][score_ld(V)]
  const int32_t *control, *target;                 // control[1]: rows
  const f32x4_t *row, *terms;
  float* item;
  uint16_t* dz;
  int T, V, ld, parts, low;
  float c1;
};
int moe_head_score_dz(const ScoreDzArgs& a, hipStream_t s);
