// Tiles of grouped bf16 MFMA GEMMs: the kernels behind the products of the expert MLP (grouped_gemm.hip) and of the vocabulary
// head (head.hip), and the rule that chooses their tiles.  Included by either, which instantiates what it launches.
//
// One workgroup of FOUR waves (one per SIMD, 512 registers each) computes one 256x256 output tile
// with a 64-deep K step; the waves form a 2 x 2 grid and each owns a 128x128 piece = 8x8
// v_mfma_f32_16x16x32_bf16 accumulators, which live in the 256 accumulation registers.  Against
// eight waves with 128x64 pieces this reads a third less operand data out of LDS per FLOP, and the
// 16x16x32 form draws less power per FLOP than the 32x32x16 form (the chip is power-limited on
// real data), but with one wave per SIMD nothing covers a wave's own stalls, so the main loop is
// written instruction by instruction:
//   * MFMAs, LDS fragment reads and direct-to-LDS loads are inline assembly in program order; the
//     accumulators are pinned to accumulation registers, so the compiler has nothing to move;
//   * between two MFMAs there is at most one other instruction (a fragment read, or a load);
//   * no vector-ALU instruction and no branch inside a K step: loads use a scalar base that is
//     advanced by scalar adds plus a 32-bit lane offset computed once per tile; the eight loads a
//     wave issues per operand tile share one M0 value (the instruction's immediate offset moves
//     the LDS address; the lane offset takes the same amount out of the global address again);
//   * the last three K steps of a tile (the last one that loads, which is the one that may load a
//     partial step of a weight gradient; the one that only awaits; the last one) are separate copies
//     of the step, and a tile enters the ring of LDS slots at the phase that puts those three on
//     phases 0, 1 and 2.
//
// The whole of it exists a second time with tiles of 128x128: four waves of 64x64 pieces = 4x4 accumulators, 80 KB of LDS and
// less than 256 registers, so that two workgroups share a compute unit.  The sums run in the same order and give the same
// bits; which size a launch takes is a rule on its expected tiles (TileCost).  What is said here in numbers is about the large tiles.
//
// The two operand tiles of a step (32 KB each) live in a ring of five LDS slots (160 KB, all
// there is): A(t) in slot 2t mod 5, B(t) in slot (2t+1) mod 5, so two and a half steps are
// resident (a small tile that holds all of an expert's few rows has a ring of its own, see few_rows_loop).
// Step t loads A(t+2) during its first 32-deep sub-step, into the slot B(t-1) left;
// its barrier follows that sub-step: behind it the tiles of step t+1 are complete (the wave's own
// loads of A(t+2) may still be in flight) and every wave is done with A(t), whose slot B(t+2) is
// loaded into during the second sub-step.  Fragments are double-buffered in registers: the reads
// of the next sub-step are issued between the MFMAs of the current one.
//
// Tile layouts.  An operand that is contiguous along K in memory (activations [rows, K],
// forward weights [N, K]) is kept as [256 rows][64 k] with 128-byte rows whose eight 16-byte
// pieces are rotated by the row (fragment = one ds_read_b128 per lane); the swizzle is
// applied on the global side of the fill, since a direct-to-LDS load writes LDS linearly.  An
// operand that is contiguous along its other dimension (weights in dgrad, both operands in
// wgrad) is kept as it lies in memory, [64 k][256 n] with 512-byte rows, and read with the
// transposing LDS load ds_read_b64_tr_b16, two per fragment (it moves half the bytes per cycle
// of ds_read_b128, which makes the weight gradients LDS-bound).
//
// The MFMAs are issued as (weight fragment) x (activation fragment), so a lane ends up with
// four consecutive output COLUMNS of one row.  The epilogue reads the accumulators by hand, rounds
// to bf16, stages 16 or 32 rows of the wave's 128x128 piece at a time in the wave's own 8 KB of LDS
// and writes them out in full 256-byte row segments; the SwiGLU forward and backward formulas are
// applied on the way, on the fp32 accumulators.
//
// Tiles of the row-grouped products are found on the device from expert_offsets: every wave
// turns the tile number into (expert, first row, column tile); inside an expert the row tiles are
// innermost; experts without rows own no tile; rows past an expert's end are clamped on load and
// dropped on store by the range check of buffer resources, and 32-row groups without a valid row issue no MFMA.
#pragma once
#include <climits>
#include <type_traits>
#include <utility>
#include "common.h"
#include "dma.h"
#include "gemm.h"

namespace {

constexpr int BK = 64;
constexpr int GEMM_THREADS = 256;
constexpr int NSLOT = 5;                              // ring of operand tile slots
// What follows from the edge S of the output tile, 256 or 128 (see TileCost).  Four waves as 2 x 2 in either case.
template <int S> struct Tile {
  static_assert(S == 256 || S == 128);
  static constexpr int BYTES = S * BK * 2;            // one operand tile: 32 or 16 KB
  static constexpr int LDS = NSLOT * BYTES;           // 160 KB, everything a compute unit has; or 80 KB, two workgroups on it
  static constexpr int PER_CU = 256 / S;              // workgroups per compute unit
  static constexpr int HALF = S / 2;                  // rows and columns of a wave's piece
  static constexpr int NB = S / 32;                   // 16 x 16 blocks along each side of it
  static constexpr int NL = S / 32;                   // direct-to-LDS loads (1 KB each) per wave and operand tile
  static constexpr int SHARE = BYTES / 4;             // a wave's share of a slot: what it fills, and stages in
  static constexpr int KN_ROW = S * 2;                // bytes of a row of a [64 k][S n] tile
  static constexpr int KN_PIECES = S / 8;             // 16-byte pieces of it
  static constexpr int KN_RPL = 64 / KN_PIECES;       // rows of it that one load fills
  static constexpr int SLOTS_PER_SET = 65536 / BYTES; // slots that an LDS read's immediate offset reaches
  static constexpr int SETS = (NSLOT + SLOTS_PER_SET - 1) / SLOTS_PER_SET;
};
// few_rows_loop: up to 64 rows, RING steps of one 16 KB slot for B and 8 KB for A behind the B slots
constexpr int FEW_ROWS = 64, FEW_RING = 3, FEW_A_BYTES = FEW_ROWS * BK * 2;
static_assert(FEW_RING * (Tile<128>::BYTES + FEW_A_BYTES) <= Tile<128>::LDS);
constexpr int LOAD_BIAS = 4096;                       // see dma16_imm
constexpr int slot_of_a(int p) { return (2 * p) % NSLOT; }       // p = ring phase of the step
constexpr int slot_of_b(int p) { return (2 * p + 1) % NSLOT; }

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int N> using IC = std::integral_constant<int, N>;
template <typename F, int... I> __device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
  (f(IC<I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void static_for(F&& f) {
  static_for_impl(static_cast<F&&>(f), std::make_integer_sequence<int, N>{});
}

enum GemmMode { GATE_UP = 0, DOWN = 1, DGRAD_H = 2, DGRAD_X = 3, WGRAD = 4, WGRAD_GATHER = 5, DGRAD_H_GATE = 6,
                WGRAD_GATHER_A = 7, HEAD_STATS = 8, HEAD_DZ = 9, HEAD_DX = 10, HEAD_DW = 11 };
// WGRAD_GATHER / WGRAD_GATHER_A: a weight gradient whose B / A operand rows are token rows found through
// row_token.  DGRAD_H_GATE: DGRAD_H for a forward pass that folded the gate weight into h: its A rows are
// rows of dout found through row_token, its epilogue scales by the row's gate weight and also emits the
// row's partial dot product with h = silu(g) u (the gradient of the gate weight).
// The vocabulary head (head.hip), rows offsets[0] = 0 to offsets[1], one group.  HEAD_STATS, HEAD_DZ: logits A0 . B0^T of which the
// epilogue makes a row's maximum and sums over the wave's columns, or the logits' gradient (row length M).  HEAD_DX: A0 (row length K) times
// B0 in row_token[0] parts of the reduction over its M rows, each part's sums in 32 bits.  HEAD_DW: WGRAD with rows of M elements, K of them
// wanted, in E parts of the reduction; with more than one O1 takes each part's sums in 32 bits.
constexpr bool is_logits(int mode) { return mode == HEAD_STATS || mode == HEAD_DZ; }
constexpr bool is_wgrad(int mode) { return mode == WGRAD || mode == WGRAD_GATHER || mode == WGRAD_GATHER_A || mode == HEAD_DW; }
constexpr bool is_dgrad_h(int mode) { return mode == DGRAD_H || mode == DGRAD_H_GATE; }

struct GemmArgs {
  // row-grouped products (modes 0-3, 6)
  const uint16_t* A0;   // [R_cap, K]   activations (phase 0)
  const uint16_t* A1;   // second K phase of DGRAD_X (du), else unused
  const uint16_t* B0;   // weights, stacked over experts
  const uint16_t* B1;   // Wu (GATE_UP: the up half of the column tile; DGRAD_X: second K phase)
  const uint16_t* G;    // DGRAD_H epilogue inputs
  const uint16_t* U;
  uint16_t* O0;         // g | yp | dg | dxp | dW
  uint16_t* O1;         // u | du
  uint16_t* O2;         // h
  const int32_t* offsets;
  const int32_t* row_token;   // not null: rows of the activation operand are gathered, row r lies at A0[row_token[r]]
                              // (GATE_UP, DGRAD_H_GATE, WGRAD_GATHER_A: the A operand; WGRAD_GATHER: the B operand)
  const float* row_weight;    // GATE_UP: not null = h is scaled by the row's gate weight; DGRAD_H_GATE: required
  float* dgate_part;          // DGRAD_H_GATE: [R_cap][N / 64] partial dot products, one per row and 64-column strip
  int E;
  int K;                // reduction length of one phase (row-grouped products)
  int N;                // output columns (per half for GATE_UP)
  int n_tiles;          // column tiles
  int m_tiles_cap;      // upper bound on row tiles (row-grouped products); row tiles of one dW (WGRAD)
  int stream_rows;      // HEAD_DX: not zero = onto the sums that are there.  GATE_UP, DOWN: nothing is done where there are at most this many rows (0: always): a launch of
                        // the streaming kernel in front has done it
  // WGRAD: out[e][M][N] = sum over the expert's rows of A[r][M] * B[r][N]
  int M;
};

// What the epilogues of the head's products take beside GemmArgs.  Items are the logits that count by themselves: of the target and of the
// teacher's entries.  Without a teacher every row has one item, its target; with one they are listed by blocks of 16 rows and, inside a block,
// by strips of 64 columns.
struct HeadItem { uint32_t at, slot; };   // at: row in the block | column << 4
struct HeadArgs {
  float* part;                // HEAD_STATS: [row block][strips of HALF columns][2 or (two) 3][16 rows]: maximum, sum and sum at the temperature, without the items
  const f32x4_t* row;         // HEAD_DZ: per row log2(e) lse, factor, and the same at the temperature
  const int32_t* target;      // [row]
  const int32_t* list_start;  // [row block][list_ld]: first item of each strip; null: no teacher
  const HeadItem* items;      // [row block][16 slots]
  const f32x4_t* terms;       // HEAD_DZ: as items, or [row]; the gradient there is t0 + t1 (exp(z / temperature - t2) - 1) + t3 exp(z - lse); with `two` and
                              // t1 = 0 it is t0 + the row's term at the temperature + t3 exp(z - lse)
  float* item;                // [row][slots]: HEAD_STATS: the logit; HEAD_DZ: what the gradient loses when it is rounded
  float c1, c2, over_tau;     // log2(e), the same over the temperature, 1 / temperature
  int two;                    // both sums, both terms
  int strips, list_ld, slots;
  int col0;                   // vocabulary column of the product's first
  int lo;                     // HEAD_DZ: up to so many rows what rounding loses is stored too, in as many rows behind the others
};

// 512 bytes of zeros: what the reduction rows past an expert's end read in the weight-gradient products.
__device__ __attribute__((aligned(512))) uint32_t g_zero_block[128];

// [256 rows][64 k] tile, 128-byte rows: the 16-byte piece `logical` (0..7) of `row` lies at physical piece
// (logical + row) mod 8.  A fragment read (16 rows x 4 neighbouring pieces per instruction) then costs 8.5
// cycles per CU, as a linear read does; XOR-ing the piece with (row ^ row >> 3) & 7 costs 8.9, no swizzle 16.
// This is the inverse: which logical piece a fill has to fetch for physical piece `phys`.
__device__ __forceinline__ int kc_logical_piece(int row, int phys) { return (phys - row) & 7; }
// [64 k][S n] tile: 16-byte pieces of a k row are XOR-swizzled with 4*(k & 3), which spreads the
// four k rows that 16 lanes of a transposing read touch over four different 64-byte bank groups.
__device__ __forceinline__ int kn_piece(int krow, int piece) { return piece ^ ((krow & 3) << 2); }

// Everything the main loop issues is inline assembly in program order (asm volatile statements keep
// their order), with immediate offsets, and is awaited by hand: fragments are read one sub-step
// ahead and loads several steps ahead, which the compiler's own wait insertion cannot express.
template <int OFF> __device__ __forceinline__ bf16x8_t lds_read_b128(uint32_t addr) {
  bf16x8_t v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
}
template <int OFF> __device__ __forceinline__ s16x4 lds_read_tr_b64(uint32_t addr) {
  s16x4 v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF) : "memory");
  return v;
}
// Direct-to-LDS loads, 16 bytes per lane: lane l lands at M0 + OFF + 16 l, and reads global address
// (scalar base) + (32-bit lane offset) + OFF.  The immediate moves both addresses: a wave's eight loads
// of a tile use OFF = (i - 4) * 1024 with one M0 value, their lane offsets carry -OFF, and LOAD_BIAS
// (subtracted from the scalar base, added to every lane offset) keeps the lane offsets non-negative.
// Nothing else in this file uses M0.
template <int OFF> __device__ __forceinline__ void set_m0(uint32_t lds_base) {
  asm volatile("s_add_i32 m0, %0, %1" :: "s"(lds_base), "n"(OFF) : "memory", "scc");
}
// the same with a 64-bit address per lane (used once per tile at most, for rows past an expert's end)
template <int OFF> __device__ __forceinline__ void dma16_lane_imm(const char* p) {
  asm volatile("global_load_lds_dwordx4 %0, off offset:%1" :: "v"(p), "n"(OFF) : "memory");
}
// A 4-byte load as (scalar base) + (32-bit lane offset) + immediate, awaited by hand like the loads above.
template <int OFF> __device__ __forceinline__ int load_i32(uint32_t voff, const int32_t* sbase) {
  int v;
  asm volatile("global_load_dword %0, %1, %2 offset:%3" : "=v"(v) : "v"(voff), "s"(sbase), "n"(OFF) : "memory");
  return v;
}
__device__ __forceinline__ void wg_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

// A fragment of a [64 k][256 n] tile: two transposing reads (k rows +0..3 and +4..7 of the lane's column).
union KnFrag {
  s16x4 h[2];
  bf16x8_t v;
};

// Reduction over the four lanes that hold the same row of an accumulator (lane, lane ^ 16, lane ^ 32, lane ^ 48).
template <typename Op> __device__ __forceinline__ float quads_reduce(float v, Op op) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// sigmoid through the hardware exp2 and reciprocal (each about 1 ulp): far inside bf16 rounding.
// exp2 overflows to +inf for very negative g and the reciprocal then returns 0, as it should.
__device__ __forceinline__ float sigmoid_f(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g));
}
__device__ __forceinline__ float silu_f(float g) { return g * sigmoid_f(g); }

// Row tiles of the grouped products: expert e owns ceil(rows_e / S) consecutive tile numbers (S: the tile's edge).
// Both functions are evaluated by a whole wave (64 experts per pass) and return wave-uniform values.
template <int S> __device__ __forceinline__ int count_row_tiles(const int32_t* offsets, int E, int lane) {
  int total = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int ee = e0 + lane;
    const int rows = ee < E ? offsets[ee + 1] - offsets[ee] : 0;
    total += wave_lane(wave_incl_scan((rows + S - 1) / S), 63);
  }
  return total;
}
// Tile number `tile` of a row-grouped product -> expert, first row, column tile.  An expert's tiles are
// numbered column tile by column tile, its row tiles innermost: the workgroups of an XCD, which take a
// run of consecutive tiles, then share each weight panel among all row tiles of the expert at the same
// time, so that it is fetched from memory once (weights are the larger operand and are used by only
// rows_e / 256 tiles each; activations of a row tile recur every rows_e / 256 tiles).
//
// With at most 128 experts (two per lane) the experts are not listed in index order: those whose tile count
// is a whole number of XCD runs come first, then those that fill half a run, then the rest.  The first
// two groups then start on run boundaries, so such an expert's tiles are worked on by one XCD at one
// time and its activation rows are fetched into one L2 once; an expert that straddles two runs has its
// rows fetched by both.  The lane keeps its expert's row range and first list position for the whole
// kernel, so the lookup needs no memory access (which would otherwise sit in front of every tile's
// first loads) and no scan.
// (kept as six plain registers: a struct of arrays behind a reference ends up in scratch memory)
__device__ __forceinline__ void sorted_first_tiles(int tiles0, int tiles1, int run, int& first0, int& first1) {
  const int r0 = tiles0 % run, r1 = tiles1 % run;
  const int cls0 = r0 == 0 ? 0 : (2 * r0 == run ? 1 : 2);
  const int cls1 = r1 == 0 ? 0 : (2 * r1 == run ? 1 : 2);
  int base = 0;
  first0 = 0;
  first1 = 0;
#pragma unroll
  for (int c = 0; c < 3; ++c) {
    const int mine0 = cls0 == c ? tiles0 : 0;
    const int inc0 = wave_incl_scan(mine0);
    if (cls0 == c) first0 = base + inc0 - mine0;
    base += wave_lane(inc0, 63);
    const int mine1 = cls1 == c ? tiles1 : 0;
    const int inc1 = wave_incl_scan(mine1);
    if (cls1 == c) first1 = base + inc1 - mine1;
    base += wave_lane(inc1, 63);
  }
}
constexpr int LANE_EXPERTS_MAX = 128;
// One half (experts 64 h .. 64 h + 63, one per lane) of the register-resident lookup.
template <int S>
__device__ __forceinline__ bool find_tile_half(int h, int lo, int hi, int first, int n_tiles, int tile, int& e, int& m0,
                                               int& m_end, int& nt, int& rt) {
  const int row_tiles = (hi - lo + S - 1) / S;
  const int tiles = row_tiles * n_tiles;
  const unsigned long long hit = __ballot(tiles > 0 && first <= tile && tile < first + tiles);
  if (!hit) return false;
  const int l = __ffsll(hit) - 1;
  e = h * 64 + l;
  const int q = tile - wave_lane(first, l);
  rt = wave_lane(row_tiles, l);
  nt = q / rt;
  m0 = wave_lane(lo, l) + (q - nt * rt) * S;
  m_end = wave_lane(hi, l);
  return true;
}
template <int S>
__device__ __forceinline__ void find_tile(const int32_t* offsets, int E, int lo0, int hi0, int first0, int lo1, int hi1,
                                          int first1, int n_tiles, int tile, int lane, int& e, int& m0, int& m_end, int& nt,
                                          int& rt) {
  e = 0; m0 = 0; m_end = 0; nt = 0; rt = 0;
  if (E <= LANE_EXPERTS_MAX) {
    if (find_tile_half<S>(0, lo0, hi0, first0, n_tiles, tile, e, m0, m_end, nt, rt)) return;
    find_tile_half<S>(1, lo1, hi1, first1, n_tiles, tile, e, m0, m_end, nt, rt);
    return;
  }
  int base = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int ee = e0 + lane;
    const int lo = ee < E ? offsets[ee] : 0, hi = ee < E ? offsets[ee + 1] : 0;
    const int row_tiles = (hi - lo + S - 1) / S;
    const int tiles = row_tiles * n_tiles;
    const int inc = wave_incl_scan(tiles);
    const int excl = base + inc - tiles;
    const unsigned long long hit = __ballot(tiles > 0 && excl <= tile && tile < excl + tiles);
    if (hit) {
      const int l = __ffsll(hit) - 1;
      e = e0 + l;
      const int q = tile - wave_lane(excl, l);
      rt = wave_lane(row_tiles, l);
      nt = q / rt;
      m0 = wave_lane(lo, l) + (q - nt * rt) * S;
      m_end = wave_lane(hi, l);
      return;
    }
    base += wave_lane(inc, 63);
  }
}

// The kernel arguments again, through a pointer the compiler cannot see through: what is read from
// it is loaded afresh (scalar loads from the argument segment) instead of being kept in scalar
// registers across the main loop.
typedef const __attribute__((address_space(4))) GemmArgs* ArgPtr;
typedef const __attribute__((address_space(4))) HeadArgs* HeadPtr;
__device__ __forceinline__ HeadPtr head_args() {       // the second argument of grouped_gemm_head_kernel
  const __attribute__((address_space(4))) char* p = (const __attribute__((address_space(4))) char*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return (HeadPtr)(p + sizeof(GemmArgs));
}
template <int ARG> __device__ __forceinline__ ArgPtr reload_args() {   // ARG: which of the kernel's GemmArgs
  ArgPtr p = (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr() + ARG;
  asm volatile("" : "+s"(p));
  return p;
}

// A wave-uniform pointer as two scalar registers.  readfirstlane returns a signed int: it is widened
// through uint32_t, or a set bit 31 of the low half would smear into the high half.
__device__ __forceinline__ const char* scalarize(const char* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u)));
  const uint32_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32)));
  return reinterpret_cast<const char*>((static_cast<uint64_t>(hi) << 32) | static_cast<uint64_t>(lo));
}

// What a workgroup knows about one tile: where it lies, where its operand loads come from, how many
// K steps it has.
template <int S>
struct TileState {
  int e, m0, m_end, nt, n0;     // expert, first output row, end of the valid rows, column tile, first output column
  int r0;                       // first of this wave's rows inside the tile
  int m_wave;                   // end of the valid rows that are this wave's
  int nv;                       // 32-row groups that every wave works on, 1 .. HALF / 32 (the others issue no load and no MFMA)
  bool few;                     // tiles of 128: takes few_rows_loop, whose ring lies across the slots of the other tiles and the shares of
                                // the waves: only in a list with no more tiles than workgroups, the first of its launch
  bool second;                  // tile of the second weight gradient of a pair
  int nk, nk_phase;             // K steps in total / in the first K phase
  int nmain, p0;                // steps in front of the last three; ring phase of step 0
  int k_lo, k_hi;               // weight gradients: the expert's row range is the reduction
  bool last_partial;            // weight gradients: the last step holds fewer than 64 rows
  uint32_t voa[Tile<S>::NL], vob[Tile<S>::NL];   // lane offsets of a wave's loads per operand tile, in bytes
  uint32_t vcb[Tile<S>::NL];    // gathered operand: lane offset of a load without its token row
  int tokn[Tile<S>::NL];        // gathered operand: tokens of the lane's reduction rows of a coming step
  const char* sa_next;          // scalar bases of the next A / B tile to load (LOAD_BIAS low)
  const char* sb_next;
  const char* sa_phase1;        // DGRAD_X, and logits of few rows: bases of the second K phase
  const char* sb_phase1;
  size_t a_step, b_step;        // bytes per step
  const int32_t* row_tok;       // gathered operand: token of the expert's first reduction row onwards
};

// How dW's tiles are dealt behind dx's (see head_deal): `extra` tiles of this workgroup's own, from `first` on in steps of `by`, then
// those behind the first `skipped`, in turn with all workgroups.
struct Deal { int extra, first, by, skipped; };

// One product's tile list, walked by this workgroup from list position first_tile in steps of
// gridDim.x.  Returns the position at which the workgroup left the list, counted from its end:
// where it enters a list that follows in the same launch.
template <int MODE, int S, int ARG>
__device__ __forceinline__ int gemm_tile_list(const GemmArgs& a, int first_tile, Deal deal = {}) {
  using TL = Tile<S>;
  using TileState = TileState<S>;
  constexpr int NL = TL::NL, NB = TL::NB, HALF = TL::HALF, TILE_BYTES = TL::BYTES;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid0 = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid0 >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  constexpr bool A_KN = is_wgrad(MODE);                                           // stored [k][m]
  constexpr bool B_KN = (is_wgrad(MODE) || is_dgrad_h(MODE) || MODE == DGRAD_X || MODE == HEAD_DX);  // stored [k][n]
  constexpr bool GATHER_B = (MODE == WGRAD_GATHER);
  constexpr bool GATHER_A = (MODE == WGRAD_GATHER_A);
  constexpr bool IS_HEAD = is_logits(MODE) || MODE == HEAD_DX || MODE == HEAD_DW;

  // What the head's products read on the device is read once: their rows (HEAD_STATS without offsets: all M tokens), whether x itself holds them, the
  // parts of dx.  (For every tile: a latency between the tiles, which counts where they have one or two steps.)
  int head_rows = 0, head_flag = 0;
  if constexpr (IS_HEAD) {
    head_rows = __builtin_amdgcn_readfirstlane(MODE == HEAD_STATS && a.offsets == nullptr ? a.M : a.offsets[1]);
    head_flag = __builtin_amdgcn_readfirstlane(a.row_token == nullptr ? 0 : a.row_token[0]);
  }

  // ---------------- tile list ---------------------------------------------------
  int total;
  // experts `lane` and `lane + 64`: row range and list position of the first tile, kept for the whole kernel
  // when E <= LANE_EXPERTS_MAX
  int lo0 = 0, hi0 = 0, first0 = 0, lo1 = 0, hi1 = 0, first1 = 0;
  // WGRAD / WGRAD_GATHER with a second A operand (A1 -> O1): two weight gradients that share their B
  // operand in one launch; an expert's tiles of the first come before its tiles of the second
  int wpair = 1;
  if constexpr (MODE == WGRAD_GATHER || MODE == WGRAD) wpair = a.A1 != nullptr ? 2 : 1;
  if constexpr (is_wgrad(MODE)) {
    total = a.E * a.m_tiles_cap * a.n_tiles * wpair;
  } else if constexpr (is_logits(MODE) || MODE == HEAD_DX) {
    total = (head_rows + S - 1) / S * a.n_tiles * (MODE == HEAD_DX ? head_flag : 1);
  } else {
    total = count_row_tiles<S>(a.offsets, a.E, tid0 & 63) * a.n_tiles;
    if constexpr (MODE == GATE_UP || MODE == DOWN) {
      if (a.stream_rows > 0 && a.offsets[a.E] <= a.stream_rows) total = 0;
    }
    if (a.E <= LANE_EXPERTS_MAX) {
      const int e0 = tid0 & 63, e1 = 64 + (tid0 & 63);
      if (e0 < a.E) { lo0 = a.offsets[e0]; hi0 = a.offsets[e0 + 1]; }
      if (e1 < a.E) { lo1 = a.offsets[e1]; hi1 = a.offsets[e1 + 1]; }
      sorted_first_tiles((hi0 - lo0 + S - 1) / S * a.n_tiles, (hi1 - lo1 + S - 1) / S * a.n_tiles, gridDim.x >> 3, first0, first1);
    }
  }
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<size_t>(LDS_PTR(lds)));
  // M0 base of this wave's loads: the middle of its share of tile slot 0 (immediates reach -4096 .. +3072)
  const uint32_t lds_fill = __builtin_amdgcn_readfirstlane(lds0 + wave * TL::SHARE + NL / 2 * 1024);

  // few_rows_loop: the same for its A tiles, 2 KB of a wave each
  const uint32_t few_a = __builtin_amdgcn_readfirstlane(lds0 + FEW_RING * TILE_BYTES + wave * 2048 + NL / 2 * 1024);

  const int lane = tid0 & 63;
  // k row (of a [64 k][S n] tile) that load i of this wave fills from this lane
  auto kn_load_row = [&](int i, int lane) __attribute__((always_inline)) { return (wave * NL + i) * TL::KN_RPL + lane / TL::KN_PIECES; };
  // Everything about tile number `tile` of the list that does not depend on the K step.
  auto setup_tile = [&](int tile, TileState& t) __attribute__((always_inline)) {
  // the thread id is laundered per tile so that the lane-dependent pieces of the load offsets are recomputed for
  // every tile instead of staying live (and spilling) across the main loop
  int tid = tid0;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63;
  int e, m0, m_end, nt, rt = 0;
  bool second = false;
  if constexpr (is_wgrad(MODE)) {
    nt = tile % a.n_tiles;
    const int rest = tile / a.n_tiles;
    const int per_expert = a.m_tiles_cap * wpair;
    e = rest / per_expert;
    int mi = rest % per_expert;
    if (mi >= a.m_tiles_cap) { mi -= a.m_tiles_cap; second = true; }
    m0 = mi * S;                        // output row of dW
    m_end = MODE == HEAD_DW ? a.K : a.M;
  } else if constexpr (is_logits(MODE)) {
    // Bands of eight row tiles, column tile by column tile: the 32 (or 64) tiles that an XCD works on at a time then share 8 panels of
    // rows and 4 (or 8) of columns; all rows of a column tile in a run would have every XCD fetch all rows in every round.
    m_end = head_rows;
    rt = (m_end + S - 1) / S;
    const int band = tile / (8 * a.n_tiles), in = tile - band * 8 * a.n_tiles;
    const int high = rt - band * 8 < 8 ? rt - band * 8 : 8;
    nt = in / high;
    m0 = (band * 8 + in - nt * high) * S;
    e = 0;
    nt = __builtin_amdgcn_readfirstlane(nt);
  } else if constexpr (MODE == HEAD_DX) {
    m_end = head_rows;
    rt = (m_end + S - 1) / S;
    e = tile / (rt * a.n_tiles);        // part of the reduction
    const int in = tile - e * rt * a.n_tiles;
    m0 = in / a.n_tiles * S;
    nt = __builtin_amdgcn_readfirstlane(in % a.n_tiles);
  } else {
    find_tile<S>(a.offsets, a.E, lo0, hi0, first0, lo1, hi1, first1, a.n_tiles, tile, lane, e, m0, m_end, nt, rt);
    nt = __builtin_amdgcn_readfirstlane(nt);
  }
  // tile coordinates are wave-uniform: keep them in scalar registers, so that everything derived
  // from them (operand base addresses in particular) is scalar too
  e = __builtin_amdgcn_readfirstlane(e);
  m0 = __builtin_amdgcn_readfirstlane(m0);
  m_end = __builtin_amdgcn_readfirstlane(m_end);
  const int n0 = nt * (MODE == GATE_UP ? HALF : S);
  t.e = e; t.m0 = m0; t.m_end = m_end; t.nt = nt; t.n0 = n0; t.second = second;
  // The tile's 32-row groups that hold a valid row are shared out evenly between the two pairs of waves, the last of an odd
  // number together with a dead one: a ragged tile keeps both pairs busy for half the time instead of one for all of it, and
  // rows of dead groups are not loaded (but for that one).
  int nv = HALF / 32, r0 = wm * HALF, m_wave = m_end;
  if constexpr (!is_wgrad(MODE)) {
    int groups = (m_end - m0 + 31) >> 5;
    groups = groups > S / 32 ? S / 32 : groups;
    nv = __builtin_amdgcn_readfirstlane((groups + 1) >> 1);
    r0 = wm * 32 * nv;
    m_wave = m_end < m0 + r0 + 32 * nv ? m_end : m0 + r0 + 32 * nv;
    r0 = __builtin_amdgcn_readfirstlane(r0);
    m_wave = __builtin_amdgcn_readfirstlane(m_wave);
  }
  t.nv = nv; t.r0 = r0; t.m_wave = m_wave;
  t.few = S == 128 && !is_wgrad(MODE) && MODE != HEAD_DX && nv == 1 && rt == 1 && total <= static_cast<int>(gridDim.x);

  // ---------------- operand sources -------------------------------------------
  // Per K step and operand tile a wave issues NL direct-to-LDS loads of 1 KB each:
  //  K-contiguous source ([row][k]): load i of wave w fills LDS rows 8 (NL w + i) .. + 8;
  //    lane l -> row + l/8, physical piece l%8, i.e. logical piece kc_logical_piece(row, l%8).
  //    The base advances by 64 elements per step.  B: these are the tile's rows.  A: they hold its rows 32 i + 8 w .. + 8, so that
  //    the first 2 nv loads of every wave bring the rows of the 2 nv live groups, and the others are left out.
  //  n-contiguous source ([k][n]): load i of wave w fills the KN_RPL (2 or 4) k rows from KN_RPL (NL w + i) on;
  //    with P = KN_PIECES (32 or 16) lane l -> k row + l/P, physical piece l%P = logical piece kn_piece(k row, l%P).
  //    The base advances by 64 rows per step.
  // Lane offsets carry LOAD_BIAS - (i - NL / 2) * 1024 (see dma16_imm); the scalar bases lie LOAD_BIAS low.
  uint32_t (&voa)[NL] = t.voa;          // lane offsets in bytes
  uint32_t (&vob)[NL] = t.vob;
  const char* abase;                    // step 0 of phase 0, without the bias
  const char* bbase;
  ptrdiff_t a_phase = 0, b_phase = 0;   // byte offset of the second K phase (DGRAD_X)
  size_t a_step, b_step;                // bytes per step
  int k_lo = 0, k_hi = 0;               // WGRAD: the expert's row range is the reduction
  const int32_t* row_tok = nullptr;     // GATHER_A/B: token of the expert's first reduction row onwards
  uint32_t (&vcb)[NL] = t.vcb;          // GATHER_A/B: lane offset of a load without its token row
#pragma unroll
  for (int i = 0; i < NL; ++i) { t.vcb[i] = 0; t.tokn[i] = 0; }
  int nk, nk_phase;                     // steps in total / in the first K phase

  if constexpr (is_wgrad(MODE)) {
    if constexpr (MODE == HEAD_DW) {
      const int all = head_rows, steps = (all + BK - 1) / BK;
      k_lo = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<long long>(steps) * e / a.E)) * BK;
      k_hi = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<long long>(steps) * (e + 1) / a.E)) * BK;
      k_hi = k_hi > all ? all : k_hi;
    } else {
      k_lo = __builtin_amdgcn_readfirstlane(a.offsets[e]);
      k_hi = __builtin_amdgcn_readfirstlane(a.offsets[e + 1]);
    }
    nk = (k_hi - k_lo + BK - 1) / BK;
    nk_phase = nk;
    if constexpr (GATHER_A) {
      abase = reinterpret_cast<const char*>(a.A0 + m0);
      a_step = 0;
      row_tok = a.row_token + k_lo;
    } else {
      abase = reinterpret_cast<const char*>((second ? a.A1 : a.A0) + static_cast<size_t>(k_lo) * a.M + m0);
      a_step = static_cast<size_t>(BK) * a.M * 2;
    }
    if constexpr (GATHER_B) {
      // the base stays at the first token row; a load's lane offset carries its token (set per step)
      bbase = reinterpret_cast<const char*>(a.B0 + n0);
      b_step = 0;
      row_tok = a.row_token + k_lo;
    } else {
      const uint16_t* B = MODE == HEAD_DW && head_flag != 0 ? a.B1 : a.B0;
      bbase = reinterpret_cast<const char*>(B + static_cast<size_t>(k_lo) * a.N + n0);
      b_step = static_cast<size_t>(BK) * a.N * 2;
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int krow = kn_load_row(i, lane);
      const int piece = kn_piece(krow, lane % TL::KN_PIECES);
      int ca = piece * 8;  if (m0 + ca > a.M - 8) ca = a.M - 8 - m0;
      int cb = piece * 8;  if (n0 + cb > a.N - 8) cb = a.N - 8 - n0;
      const uint32_t fix = static_cast<uint32_t>(LOAD_BIAS - (i - NL / 2) * 1024);
      voa[i] = static_cast<uint32_t>((krow * a.M + ca) * 2) + fix;
      vob[i] = static_cast<uint32_t>((krow * a.N + cb) * 2) + fix;
      if constexpr (GATHER_B) vcb[i] = static_cast<uint32_t>(cb * 2) + fix;
      if constexpr (GATHER_A) vcb[i] = static_cast<uint32_t>(ca * 2) + fix;
    }
  } else {
    nk = a.K / BK;
    nk_phase = nk;
    // (logits: the tokens' rows side by side, or as they are where all have a loss)
    const uint16_t* A = a.A0;
    if constexpr (is_logits(MODE)) { if (head_flag != 0) A = a.A1; }
    abase = reinterpret_cast<const char*>(A + static_cast<size_t>(m0) * a.K);
    a_step = BK * 2;
    bool gathered = false;
    if constexpr (MODE == GATE_UP) gathered = a.row_token != nullptr;
    if constexpr (MODE == DGRAD_H_GATE) gathered = true;
    if (gathered) abase = reinterpret_cast<const char*>(a.A0);   // lane offsets carry the token row
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int row = i * 32 + wave * 8 + (lane >> 3);
      const int chunk = kc_logical_piece(row, lane & 7);
      int r = row;
      if (m0 + r > m_end - 1) r = m_end - 1 - m0;
      const uint32_t fix = static_cast<uint32_t>(LOAD_BIAS - (i - NL / 2) * 1024);
      if (gathered) voa[i] = (static_cast<uint32_t>(a.row_token[m0 + r]) * a.K + chunk * 8) * 2u + fix;
      else voa[i] = static_cast<uint32_t>((r * a.K + chunk * 8) * 2) + fix;
    }
    if constexpr (MODE == DGRAD_X) { a_phase = (a.A1 - a.A0) * 2; nk *= 2; }
    if constexpr (MODE == HEAD_DX) {
      const int steps = (a.M + BK - 1) / BK;
      const int parts = head_flag;
      k_lo = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<long long>(steps) * e / parts)) * BK;
      k_hi = __builtin_amdgcn_readfirstlane(static_cast<int>(static_cast<long long>(steps) * (e + 1) / parts)) * BK;
      nk = nk_phase = (k_hi - k_lo) / BK;
      k_hi = k_hi > a.M ? a.M : k_hi;
      abase += static_cast<size_t>(k_lo) * 2;
    }
    const size_t wsz = static_cast<size_t>(a.N) * a.K;
    if constexpr (!B_KN) {
      // GATE_UP: with Q = S / 4 a wave's 2 Q tile rows are Q rows of Wg and the same Q rows of Wu: tile rows
      // [0,Q) Wg n0.., [Q,2Q) Wu n0.., [2Q,3Q) Wg n0+Q.., [3Q,4Q) Wu n0+Q.. (wave w fills rows Q w .. of them)
      const uint16_t* w = a.B0;
      int first_col = wave * (S / 4);
      if constexpr (MODE == GATE_UP) {
        if (wave & 1) w = a.B1;
        first_col = (wave >> 1) * (S / 4);
      }
      bbase = reinterpret_cast<const char*>(w + static_cast<size_t>(e) * wsz + static_cast<size_t>(n0) * a.K);
      b_step = BK * 2;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int row = (wave * NL + i) * 8 + (lane >> 3);   // LDS row of the B tile
        const int chunk = kc_logical_piece(row, lane & 7);
        int col = first_col + i * 8 + (lane >> 3);
        if (n0 + col > a.N - 1) col = a.N - 1 - n0;
        vob[i] = static_cast<uint32_t>((col * a.K + chunk * 8) * 2) + static_cast<uint32_t>(LOAD_BIAS - (i - NL / 2) * 1024);
      }
    } else {  // DGRAD_H / DGRAD_X: weights stored [K][N]
      if constexpr (MODE == HEAD_DX) bbase = reinterpret_cast<const char*>(a.B0 + static_cast<size_t>(k_lo) * a.N + n0);
      else bbase = reinterpret_cast<const char*>(a.B0 + static_cast<size_t>(e) * wsz + n0);
      b_step = static_cast<size_t>(BK) * a.N * 2;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int krow = kn_load_row(i, lane);
        int cb = kn_piece(krow, lane % TL::KN_PIECES) * 8;
        if (n0 + cb > a.N - 8) cb = a.N - 8 - n0;
        vob[i] = static_cast<uint32_t>((krow * a.N + cb) * 2) + static_cast<uint32_t>(LOAD_BIAS - (i - NL / 2) * 1024);
      }
      if constexpr (MODE == DGRAD_X) b_phase = (a.B1 - a.B0) * 2;
    }
  }

  // Both bases live in scalar registers and are advanced by scalar adds: steps are loaded in order.
  t.sa_next = scalarize(abase - LOAD_BIAS);
  t.sb_next = scalarize(bbase - LOAD_BIAS);
  t.sa_phase1 = nullptr;
  t.sb_phase1 = nullptr;
  if constexpr (MODE == DGRAD_X) { t.sa_phase1 = scalarize(abase + a_phase - LOAD_BIAS); t.sb_phase1 = scalarize(bbase + b_phase - LOAD_BIAS); }
  t.a_step = a_step; t.b_step = b_step; t.k_lo = k_lo; t.k_hi = k_hi; t.row_tok = row_tok; t.nk = nk; t.nk_phase = nk_phase;
  if constexpr (is_logits(MODE)) {
    // With one or two row tiles the product waits for memory.  Where weight rows are multiples of 4096 bytes, tiles that run in step read the same
    // few bytes of each, which lie in a fraction of the channels: they begin their reductions at different steps (57 tokens of d 4096, V 32003: 63 -> 48.5 us;
    // 200 of d 2048, V 50304: 59.6 -> 55; other rows as before; with many row tiles it costs 1 %).
    if (rt <= 2) {
      const int rot = __builtin_amdgcn_readfirstlane(nt * 3 % nk);
      t.sa_phase1 = t.sa_next; t.sb_phase1 = t.sb_next;
      t.sa_next += rot * BK * 2; t.sb_next += rot * BK * 2;
      t.nk_phase = nk - rot;
    }
  }
  t.last_partial = (is_wgrad(MODE) || MODE == HEAD_DX) && ((k_hi - k_lo) % BK) != 0;
  // The last three steps of a tile are copies of their own: the last step that loads (it loads the tile's last
  // step, the one that may be partial in a weight gradient), the step that only awaits, and the last one.
  // The tile enters the ring at the phase p0 that puts these three on phases 0, 1 and 2, so that the steps
  // before them end on a round of the five phases.
  t.nmain = nk >= 3 ? nk - 3 : 0;
  t.p0 = nk >= 3 ? (NSLOT - t.nmain % NSLOT) % NSLOT : (nk == 2 ? 1 : 2);
  };


  // Load i of the A / B tile of step kt (M0 must point at the tile's slot already).  In the weight gradients the
  // last step of an expert may be partial (its row count is no multiple of 64): reduction rows at or past the
  // expert's end then read zeros in one operand (per-lane 64-bit addresses) and a valid row in the other.
  // SP 0: the step is known to be whole; 1: known to be the partial one; 2: look (first loads of a tile).
  auto a_part = [&](TileState& t, int kt, auto i_tag, auto sp_tag) __attribute__((always_inline)) {
    constexpr int i = decltype(i_tag)::value, SP = decltype(sp_tag)::value;
    constexpr int OFF = (i - NL / 2) * 1024;
    if constexpr (is_wgrad(MODE) && !GATHER_A && SP != 0) {
      if (SP == 1 || (t.last_partial && kt == t.nk - 1)) {
        const int krow = t.k_lo + kt * BK + kn_load_row(i, lane);
        dma16_lane_imm<OFF>(krow < t.k_hi ? t.sa_next + t.voa[i]
                                        : reinterpret_cast<const char*>(g_zero_block) + lane % TL::KN_PIECES * 16 - OFF);
        return;
      }
    }
    dma16_imm<OFF>(t.voa[i], t.sa_next);   // GATHER_A: rows past the expert's end were clamped when their tokens were fetched
  };
  auto b_part = [&](TileState& t, int kt, auto i_tag, auto sp_tag) __attribute__((always_inline)) {
    constexpr int i = decltype(i_tag)::value, SP = decltype(sp_tag)::value;
    constexpr int OFF = (i - NL / 2) * 1024;
    if constexpr ((GATHER_A || MODE == WGRAD || MODE == HEAD_DW || MODE == HEAD_DX) && SP != 0) {
      if (SP == 1 || (t.last_partial && kt == t.nk - 1)) {
        const int krow = t.k_lo + kt * BK + kn_load_row(i, lane);
        if constexpr (GATHER_A) {
          // the gathered operand repeats the expert's last row past its end: this one reads zeros there
          dma16_lane_imm<OFF>(krow < t.k_hi ? t.sb_next + t.vob[i]
                                          : reinterpret_cast<const char*>(g_zero_block) + lane % TL::KN_PIECES * 16 - OFF);
        } else {
          // ... and the other operand reads its last valid row there, so that zero times it is zero (HEAD_DX: rows of A
          // are zero from there to a multiple of 64)
          dma16_lane_imm<OFF>(t.sb_next + t.vob[i] - (krow < t.k_hi ? 0 : static_cast<size_t>(krow - (t.k_hi - 1)) * a.N * 2));
        }
        return;
      }
    }
    dma16_imm<OFF>(t.vob[i], t.sb_next);   // GATHER_B: rows past the expert's end were clamped when their tokens were fetched
  };
  auto a_end = [&](TileState& t, int kt) __attribute__((always_inline)) {
    t.sa_next += t.a_step;
    if constexpr (MODE == DGRAD_X || is_logits(MODE)) {
      if (kt + 1 == t.nk_phase) t.sa_next = t.sa_phase1;
    }
  };
  auto b_end = [&](TileState& t, int kt) __attribute__((always_inline)) {
    t.sb_next += t.b_step;
    if constexpr (MODE == DGRAD_X || is_logits(MODE)) {
      if (kt + 1 == t.nk_phase) t.sb_next = t.sb_phase1;
    }
  };
  // GATHER_A/B: the tokens of the lane's NL reduction rows of step kt (kn_load_row), loaded
  // without any vector-ALU work except in an expert's last, partial step (rows past its end repeat its last
  // row: the other operand is zero there), and their turn into lane offsets of the gathered operand's loads.
  // The loads are asynchronous: apply_tok may only run after a wait that covers them.
  const uint32_t tok_voff = static_cast<uint32_t>(kn_load_row(0, lane) * 4);   // row of load 0; load i: + KN_RPL i rows
  auto fetch_tok = [&](TileState& t, int kt, int (&tk)[NL]) __attribute__((always_inline)) {
    if constexpr (GATHER_B || GATHER_A) {
      if (t.k_lo + (kt + 1) * BK > t.k_hi) {
        settle(t.row_tok);
        const int last = t.k_hi - t.k_lo - 1;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          int r = kt * BK + kn_load_row(i, lane);
          if (r > last) r = last;
          tk[i] = load_i32<0>(static_cast<uint32_t>(r) * 4u, t.row_tok);
        }
      } else {
        const int32_t* base = t.row_tok + static_cast<size_t>(kt) * BK;
        settle(base);
        static_for<NL>([&](auto i_tag) {
          constexpr int i = decltype(i_tag)::value;
          tk[i] = load_i32<i * TL::KN_RPL * 4>(tok_voff, base);
        });
      }
    }
  };
  auto apply_tok = [&](TileState& t, int (&tk)[NL]) __attribute__((always_inline)) {
    if constexpr (GATHER_B || GATHER_A) {
      const uint32_t row_bytes = static_cast<uint32_t>(GATHER_B ? a.N : a.M) * 2u;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        asm volatile("" : "+v"(tk[i]));   // not before the wait that precedes this call
        const uint32_t off = static_cast<uint32_t>(tk[i]) * row_bytes + t.vcb[i];
        if constexpr (GATHER_B) t.vob[i] = off; else t.voa[i] = off;
      }
    }
  };

  // ---------------- fragment addresses ------------------------------------------
  // Slot, block and sub-step are immediate offsets of the LDS reads, which reach 64 KB: one set of per-lane addresses
  // serves slots 0-1, one slots 2-3, one slot 4 (S = 128: slots 0-3, slot 4); up to four addresses per set and operand.
  //  [row][k] tile: block b = rows 16 b + (lane & 15), sub-step s (32 k) = logical piece 4 s + lane / 16.
  //    The row's share of the swizzle is lane & 7 whatever the block, so the address of (b, s) is
  //    base[s] + 2048 b.
  //  [k][n] tile: block b = columns 16 b + (lane & 15); within 16 lanes, lane i supplies the address of four
  //    consecutive n of k row i / 4, n group i % 4, and lane l receives k rows 0..3 of column l; lanes
  //    16 g .. 16 g + 15 take k rows 8 g .. of the sub-step.  The k-row swizzle XORs bits 1-2 of the block
  //    number (counted over the whole row), so the address of block b is base[b / 2] + 32 (b & 1); the second half of a
  //    fragment lies 4 k rows further, sub-step 1 32 k rows.
  //  The row-grouped A operand is kept as eight rows per wave of every 32-row group (see the loads): row 32 i + 8 w + s lies
  //    at LDS row 8 (NL w + i) + s, so block b begins at LDS rows 16 NL (b & 1) + 8 (b / 2) and its second half 8 NL rows further.
  //    Its addresses carry the wave's first row r0, which depends on the tile (a multiple of 32, that is 8 LDS rows).
  uint32_t fa_base[TL::SETS][4], fb_base[TL::SETS][4];
#pragma unroll
  for (int st = 0; st < TL::SETS; ++st) {
    const uint32_t org = lds0 + st * TL::SLOTS_PER_SET * TILE_BYTES;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int i16 = lane & 15;
      // [row][k]
      const int pc = ((x & 1) * 4 + (lane >> 4) + (lane & 7)) & 7;   // sub-step x & 1; the block is an immediate offset
      const uint32_t kc_a = org + (i16 >> 3) * (NL * 1024) + (lane & 7) * 128 + pc * 16;   // + 32 r0 of the tile, see main_loop
      const uint32_t kc_b = org + (wn * HALF + i16) * 128 + pc * 16;
      // [k][n]
      const int krow = (lane >> 4) * 8 + (i16 >> 2);
      const int sw = krow & 3;
      const uint32_t kn_lane = org + krow * TL::KN_ROW + ((i16 >> 1) & 1) * 16 + (i16 & 1) * 8;
      const uint32_t kn_a = kn_lane + (((wm * (NB / 2) + x) ^ sw) << 6);   // 64-byte group of block 2 x in the row
      const uint32_t kn_b = kn_lane + (((wn * (NB / 2) + x) ^ sw) << 6);
      fa_base[st][x] = A_KN ? kn_a : kc_a;
      fb_base[st][x] = B_KN ? kn_b : kc_b;
    }
  }
  int fa_r0 = 0;                 // the r0 that the A addresses carry

  // ---------------- main loop ----------------------------------------------------
  f32x4_t acc[NB][NB];

  // two fragment sets: one feeds the MFMAs while the other is being read
  KnFrag fa[2][NB], fb[2][NB];
  constexpr int A_OPS_PER_BLK = A_KN ? 2 : 1, B_OPS_PER_BLK = B_KN ? 2 : 1, SPS = TL::SLOTS_PER_SET;
  // Read instruction number `op` of a sub-step: the A blocks first (only the live ones), then the B blocks.
  auto read_op = [&](auto slot_a_tag, auto slot_b_tag, auto s_tag, auto set_tag, auto nv_tag, auto op_tag) __attribute__((always_inline)) {
    constexpr int SA = decltype(slot_a_tag)::value, SB = decltype(slot_b_tag)::value, SUB = decltype(s_tag)::value;
    constexpr int SET = decltype(set_tag)::value, NV = decltype(nv_tag)::value, OP = decltype(op_tag)::value;
    constexpr int A_OPS = 2 * NV * A_OPS_PER_BLK;
    if constexpr (OP < A_OPS) {
      constexpr int blk = OP / A_OPS_PER_BLK;
      if constexpr (A_KN) {
        constexpr int half = OP % 2;
        fa[SET][blk].h[half] = lds_read_tr_b64<SA % SPS * TILE_BYTES + SUB * 32 * TL::KN_ROW + half * 4 * TL::KN_ROW + (blk & 1) * 32>(fa_base[SA / SPS][blk >> 1]);
      } else {
        fa[SET][blk].v = lds_read_b128<SA % SPS * TILE_BYTES + (blk & 1) * 2 * NL * 1024 + (blk >> 1) * 1024>(fa_base[SA / SPS][SUB]);
      }
    } else {
      constexpr int OB = OP - A_OPS;
      constexpr int blk = OB / B_OPS_PER_BLK;
      if constexpr (B_KN) {
        constexpr int half = OB % 2;
        fb[SET][blk].h[half] = lds_read_tr_b64<SB % SPS * TILE_BYTES + SUB * 32 * TL::KN_ROW + half * 4 * TL::KN_ROW + (blk & 1) * 32>(fb_base[SB / SPS][blk >> 1]);
      } else {
        fb[SET][blk].v = lds_read_b128<SB % SPS * TILE_BYTES + blk * 2048>(fb_base[SB / SPS][SUB]);
      }
    }
  };
  // weight fragment first: the lane then holds 4 consecutive output columns of one row
  auto mma = [&](auto set_tag, auto i_tag, auto j_tag) __attribute__((always_inline)) {
    constexpr int SET = decltype(set_tag)::value, i = decltype(i_tag)::value, j = decltype(j_tag)::value;
    f32x4_t& c = acc[i][j];
    const bf16x8_t& wfrag = fb[SET][j].v;
    const bf16x8_t& afrag = fa[SET][i].v;
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(wfrag), "v"(afrag));
  };

  // One 32-deep sub-step: the live MFMAs of fragment set SET, in 2 x 2 blocks of accumulators so that within a block every product shares an operand
  // with the one before it, now the weights and now the rows; from one block to the next of the same pair of rows neither is shared (12 of the 63 steps of a
  // whole wave's piece).  The chip runs at its power limit here, and operands that were read a
  // moment ago cost less than new ones: with nothing but these MFMAs 1.007 us per K step in this order, 1.041 row by row (one operand held for
  // eight), 1.081 in scattered order; with the loop's reads, loads and barriers 1.225 / 1.256 us, the clock 1.82 / 1.78 GHz.
  // Products of 65536 rows, d 2048, f 1024, 64 experts, row by row -> 2 x 2: gate_up 440 -> 434 us, down of 2048 steps 422 -> 419, dgrad_x 419 -> 412,
  // the weight gradients 806 -> 799 and 423 -> 417.  Between the MFMAs (one per gap) stand the read
  // instructions of the next sub-step and, in a step that loads, the wave's LOADS loads of one
  // tile.  Gap g is the place after MFMA g: reads take the even gaps 0, 2, .. (every gap when they would not fit
  // otherwise), M0 is set in gap 1, loads take gaps 3, 7, .., 4 LOADS - 1; what does not fit behind
  // the last live MFMA follows it.
  constexpr auto a_loads = [](int nv) { return is_wgrad(MODE) ? NL : 2 * nv; };   // A loads per wave and step
  auto sub_step = [&](auto set_tag, auto nv_tag, auto nreads_tag, auto reader, auto loads_tag, auto set_m0_fn, auto loader)
      __attribute__((always_inline)) {
    constexpr int SET = decltype(set_tag)::value, NV = decltype(nv_tag)::value;
    constexpr int NREADS = decltype(nreads_tag)::value;
    constexpr int LOADS = decltype(loads_tag)::value;   // how many, 0: none
    constexpr int ML = 2 * NB * NV;                     // live MFMAs: blocks i < 2 NV, all j
    constexpr int RSTRIDE = 2 * NREADS > NB * NB ? 1 : 2;
    constexpr int LAST_LOAD = 4 * LOADS - 1;
    constexpr int LAST_GAP = (NREADS - 1) * RSTRIDE > LAST_LOAD ? (NREADS - 1) * RSTRIDE : LAST_LOAD;
    constexpr int SLOTS = ML > LAST_GAP + 1 ? ML : LAST_GAP + 1;
    static_for<SLOTS>([&](auto g_tag) {
      constexpr int g = decltype(g_tag)::value;
      if constexpr (g < ML) {
        constexpr int pair = g / (2 * NB), q = g % 4, at = g % (2 * NB) / 4, jj = pair & 1 ? NB / 2 - 1 - at : at;
        mma(IC<SET>{}, IC<2 * pair + q / 2>{}, IC<2 * jj + ((q & 1) ^ (q >> 1))>{});
      }
      if constexpr (g % RSTRIDE == 0 && g / RSTRIDE < NREADS) reader(IC<g / RSTRIDE>{});
      if constexpr (LOADS > 0) {
        if constexpr (g == 1) set_m0_fn();
        if constexpr (g >= 3 && g <= LAST_LOAD && (g - 3) % 4 == 0) loader(IC<(g - 3) / 4>{});
      }
    });
  };

  // Step kt at ring phase P.  KIND 2: a step that loads A(kt+2) (before its barrier, into B(kt-1)'s old slot) and
  // B(kt+2) (behind it, into A(kt)'s slot); KIND 1: the second to last step (nothing left to load); KIND 0: the
  // last step (no barrier, no next fragments).
  auto step = [&](TileState& t, int kt, auto phase_tag, auto kind_tag, auto nv_tag, auto sp_tag) __attribute__((always_inline)) {
    constexpr int P = decltype(phase_tag)::value, KIND = decltype(kind_tag)::value, NV = decltype(nv_tag)::value;
    using SA = IC<slot_of_a(P)>;
    using SB = IC<slot_of_b(P)>;
    using NextA = IC<slot_of_a((P + 1) % NSLOT)>;
    using NextB = IC<slot_of_b((P + 1) % NSLOT)>;
    constexpr int LA = slot_of_a((P + 2) % NSLOT);
    constexpr int ALOADS = a_loads(NV);
    constexpr int NREADS = 2 * NV * A_OPS_PER_BLK + NB * B_OPS_PER_BLK;
    if constexpr (KIND == 2 && GATHER_A) {
      // the tokens of A(kt+2) were fetched a step ago and are covered by that step's wait; those of A(kt+3)
      // are requested before the loads of A(kt+2), the only ones this step's wait leaves in flight
      apply_tok(t, t.tokn);
      if (kt + 3 < t.nk) fetch_tok(t, kt + 3, t.tokn);
    }
    sub_step(IC<0>{}, nv_tag, IC<NREADS>{},
             [&](auto op) __attribute__((always_inline)) { read_op(SA{}, SB{}, IC<1>{}, IC<1>{}, nv_tag, op); },
             IC<KIND == 2 ? ALOADS : 0>{},
             [&]() __attribute__((always_inline)) { set_m0<LA * TILE_BYTES>(lds_fill); settle(t.sa_next); },
             [&](auto i) __attribute__((always_inline)) { a_part(t, kt + 2, i, sp_tag); });
    if constexpr (KIND == 2) a_end(t, kt + 2);
    lds_wait<0>();
    if constexpr (KIND >= 1) {
      if constexpr (KIND == 2) wait_vm<ALOADS>(); else wait_vm<0>();   // this wave's loads of A(kt+2) may stay in flight
      wg_barrier();
    }
    if constexpr (KIND == 2 && GATHER_B) apply_tok(t, t.tokn);   // fetched a step ago, older than the loads of A(kt+2)
    sub_step(IC<1>{}, nv_tag, IC<KIND >= 1 ? NREADS : 0>{},
             [&](auto op) __attribute__((always_inline)) { read_op(NextA{}, NextB{}, IC<0>{}, IC<0>{}, nv_tag, op); },
             IC<KIND == 2 ? NL : 0>{},
             [&]() __attribute__((always_inline)) { set_m0<SA::value * TILE_BYTES>(lds_fill); settle(t.sb_next); },
             [&](auto i) __attribute__((always_inline)) { b_part(t, kt + 2, i, sp_tag); });
    if constexpr (KIND == 2) {
      b_end(t, kt + 2);
      if constexpr (GATHER_B) {
        // a whole step ahead of their use; the next step's wait covers them (they are older than its A loads)
        if (kt + 3 < t.nk) fetch_tok(t, kt + 3, t.tokn);
      }
    }
    lds_wait<0>();
  };

  // The first loads of a tile: steps 0 and 1 into the slots of phases p0 and p0 + 1.  They are requested BEFORE the epilogue
  // of the tile before, which is staged in the slot that they leave free (spare_slot; the SwiGLU derivative needs two, so
  // that B(1) waits until it is done), and awaited when the tile's main loop starts.
  // What a tile waits for between main loops counts where tiles are short: a training step of 2048 tokens (d 2048, f 1024, 64
  // experts, 4 steps per weight gradient) 885 -> 868 us, the forward of 4001 tokens over 128 experts of f 512 328 -> 322 us;
  // at 1024 rows per expert and more the chip is power-limited and the step takes as long as before (0-1.5 % less).
  // A tile with few rows is the only one of its workgroup's list (see TileState::few): there is no epilogue before it.
  auto spare_slot = [&](const TileState& t) __attribute__((always_inline)) { return (2 * t.p0 + 4) % NSLOT; };
  auto spare_slot2 = [&](const TileState& t) __attribute__((always_inline)) { return (2 * t.p0 + 3) % NSLOT; };
  auto a_unit = [&](TileState& t, int kt) __attribute__((always_inline)) {   // kt: 0 or 1
    int at = lds_fill + (2 * t.p0 + 2 * kt) % NSLOT * TILE_BYTES;
    if (t.few) at = few_a + kt * FEW_A_BYTES;
    set_m0_rt(__builtin_amdgcn_readfirstlane(at));
    settle(t.sa_next);
    if constexpr (is_wgrad(MODE)) {
      static_for<NL>([&](auto i) { a_part(t, kt, i, IC<2>{}); });
    } else {
      static_for<HALF / 32>([&](auto g) {
        constexpr int i = 2 * decltype(g)::value;
        if (i == 0 || i < 2 * t.nv) { a_part(t, kt, IC<i>{}, IC<2>{}); a_part(t, kt, IC<i + 1>{}, IC<2>{}); }
      });
    }
    a_end(t, kt);
  };
  auto b_unit = [&](TileState& t, int kt) __attribute__((always_inline)) {
    const int slot = t.few ? kt : (2 * t.p0 + 2 * kt + 1) % NSLOT;
    set_m0_rt(__builtin_amdgcn_readfirstlane(lds_fill + slot * TILE_BYTES));
    settle(t.sb_next);
    static_for<NL>([&](auto i) { b_part(t, kt, i, IC<2>{}); });
    b_end(t, kt);
  };
  auto first_loads = [&](TileState& t) __attribute__((always_inline)) {
    if (t.nk <= 0) return;
    if constexpr (GATHER_A || GATHER_B) {
      // The tokens of steps 0, 1 and 2 are requested first, older than the loads of the other operand, and are here before
      // the epilogue starts: no register that a load has yet to write lives across it.  Rows past the expert's end, and
      // steps that do not exist, repeat its last row.
      int tk[3][NL];
      const int last = t.k_hi - t.k_lo - 1;
      settle(t.row_tok);
      static_for<3>([&](auto s_tag) {
        constexpr int s = decltype(s_tag)::value;
        static_for<NL>([&](auto i_tag) {
          constexpr int i = decltype(i_tag)::value;
          int r = s * BK + kn_load_row(i, lane);
          if (r > last) r = last;
          tk[s][i] = load_i32<0>(static_cast<uint32_t>(r) * 4u, t.row_tok);
        });
      });
      if constexpr (GATHER_B) a_unit(t, 0); else b_unit(t, 0);
      wait_vm<NL>();                            // on every path, behind no branch: the compiler does not know of these loads
#pragma unroll
      for (int i = 0; i < 3 * NL; ++i) asm volatile("" : "+v"(tk[i / NL][i % NL]));
      if (t.nk > 1) { if constexpr (GATHER_B) a_unit(t, 1); else b_unit(t, 1); }
      apply_tok(t, tk[0]);
      if constexpr (GATHER_B) b_unit(t, 0); else a_unit(t, 0);
      apply_tok(t, tk[1]);
#pragma unroll
      for (int i = 0; i < NL; ++i) t.tokn[i] = tk[2][i];
      if (t.nk > 1) { if constexpr (GATHER_B) b_unit(t, 1); else a_unit(t, 1); }
    } else {
      b_unit(t, 0);
      a_unit(t, 0);
      if (t.nk > 1) {
        if (!is_dgrad_h(MODE) || t.few) b_unit(t, 1);
        a_unit(t, 1);
      }
    }
  };
  auto last_first_loads = [&](TileState& t) __attribute__((always_inline)) {
    if constexpr (is_dgrad_h(MODE)) { if (t.nk > 1 && !t.few) b_unit(t, 1); }
  };
  auto main_loop = [&](TileState& t, auto nv_tag) __attribute__((always_inline)) {
    if (t.nk <= 0) return;
    if constexpr (!A_KN) {
#pragma unroll
      for (int st = 0; st < TL::SETS; ++st) {
        fa_base[st][0] += (t.r0 - fa_r0) * 32;
        fa_base[st][1] += (t.r0 - fa_r0) * 32;
      }
      fa_r0 = t.r0;
    }
    const int p0 = t.p0, nmain = t.nmain;
    // The tile's first loads are awaited; those of step 1 may stay in flight (the last of a gathered operand only: both
    // steps of the other one come first).  Stores of the epilogue before are in flight too; as loads complete in order
    // among themselves, the waits here and in the steps hold wherever the stores lie between them.
    constexpr int NV = decltype(nv_tag)::value;
    if (t.nk <= 1) wait_vm<0>(); else if (GATHER_A || GATHER_B) wait_vm<NL>(); else wait_vm<a_loads(NV) + NL>();
    wg_barrier();
    // ---- first fragments: sub-step 0 of step 0, from the slots of phase p0
    constexpr int NREADS = 2 * NV * A_OPS_PER_BLK + NB * B_OPS_PER_BLK;
    auto first_reads = [&](auto phase_tag) __attribute__((always_inline)) {
      constexpr int P = decltype(phase_tag)::value;
      static_for<NREADS>([&](auto op) { read_op(IC<slot_of_a(P)>{}, IC<slot_of_b(P)>{}, IC<0>{}, IC<0>{}, nv_tag, op); });
    };
    switch (p0) {
      case 0: first_reads(IC<0>{}); break;
      case 1: first_reads(IC<1>{}); break;
      case 2: first_reads(IC<2>{}); break;
      case 3: first_reads(IC<3>{}); break;
      default: first_reads(IC<4>{}); break;
    }
    lds_wait<0>();
    asm volatile("s_nop 7" ::: "memory");   // the accumulators were cleared by vector-ALU writes: keep the first MFMA clear of them
    // ---- the steps that load, in rounds of the five phases (the first round starts at p0)
    int kt = 0;
    int skip = p0;
    while (kt < nmain) {
      if (skip <= 0) { step(t, kt, IC<0>{}, IC<2>{}, nv_tag, IC<0>{}); ++kt; }
      if (skip <= 1) { step(t, kt, IC<1>{}, IC<2>{}, nv_tag, IC<0>{}); ++kt; }
      if (skip <= 2) { step(t, kt, IC<2>{}, IC<2>{}, nv_tag, IC<0>{}); ++kt; }
      if (skip <= 3) { step(t, kt, IC<3>{}, IC<2>{}, nv_tag, IC<0>{}); ++kt; }
      step(t, kt, IC<4>{}, IC<2>{}, nv_tag, IC<0>{}); ++kt;
      skip = 0;
    }
    // ---- the last three steps
    if (t.nk >= 3) step(t, t.nk - 3, IC<0>{}, IC<2>{}, nv_tag, IC<is_wgrad(MODE) || MODE == HEAD_DX ? 1 : 0>{});
    if (t.nk >= 2) step(t, t.nk - 2, IC<1>{}, IC<1>{}, nv_tag, IC<0>{});
    step(t, t.nk - 1, IC<2>{}, IC<0>{}, nv_tag, IC<0>{});
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");   // the last MFMAs have written before the accumulators are read
  };
  // The main loop of a small tile that holds all of an expert's at most 64 rows, in a list with no more tiles than workgroups.  It
  // shares its weights with nobody, has little to multiply, and what it waits for is the latency of memory: in the ring above a
  // step's B tile is requested one step before it is awaited; the rows that are not there make room for FEW_RING steps of B and A,
  // all but one of them in flight.  The loop is kept plain (slots are computed, fragments are read in front of the products
  // that use them): there is time for it.
  // Not for what is left of an expert after whole tiles, nor in tiles of 256: those share their weights with the expert's other
  // tiles, and taking more than their part of the memory's bandwidth slows the others down (2048 tokens, d 2048, f 1024, 64
  // experts, forward and backward: 901 -> 921 us when they had such a ring too).  Nor in longer lists, which wait for bandwidth
  // rather than latency (501 tokens of the same layer, forward: 192 -> 197 us on one card, 212 -> 202 us on another).
  // Without / with, us: forward of 597 tokens, d 2240, f 192, 41 experts, 1 per token 57.8 / 50.2; of 146 tokens, d 256, f 1216, 33
  // experts, 6 per token 42.3 / 40.5; forward and backward of 453 tokens, d 3072, f 128, 3 of 38 experts 100 / 96.8.
  auto few_rows_loop = [&](TileState& t) __attribute__((always_inline)) {
    constexpr int STEP_LOADS = 2 + NL;
    constexpr int NREADS = 2 + NB * B_OPS_PER_BLK;       // per 32-deep sub-step
    const int i16 = lane & 15;
    // row 32 i + 8 w + s of the tile lies at LDS row 8 (2 w + i) + s (see the loads; i is 0 or 1)
    const uint32_t a_lane = lds0 + FEW_RING * TILE_BYTES + (i16 >> 3) * 2048 + (lane & 7) * 128 + t.r0 * 32;
    const uint32_t a_sub0 = a_lane + (((lane >> 4) + (lane & 7)) & 7) * 16, a_sub1 = a_lane + ((4 + (lane >> 4) + (lane & 7)) & 7) * 16;
    asm volatile("s_nop 7" ::: "memory");   // the accumulators were cleared by vector-ALU writes
    int cur = 0, nxt = 2;                   // slots of step kt and of step kt + 2
#pragma clang loop unroll(disable)
    for (int kt = 0; kt < t.nk; ++kt) {
      asm volatile("" : "+s"(kt));          // one copy of the body: two would keep the accumulators in different registers
      // this step's tiles are here (requests complete in order) ...
      if (kt + 1 < t.nk) wait_vm<STEP_LOADS>(); else wait_vm<0>();
      wg_barrier();                         // ... those of the other waves too, and every wave is done with step kt - 1, whose slot
      if (kt + 2 < t.nk) {                  // is requested anew
        set_m0_rt(__builtin_amdgcn_readfirstlane(lds_fill + nxt * TILE_BYTES));
        settle(t.sb_next);
        static_for<NL>([&](auto i) { b_part(t, kt + 2, i, IC<0>{}); });
        b_end(t, kt + 2);
        set_m0_rt(__builtin_amdgcn_readfirstlane(few_a + nxt * FEW_A_BYTES));
        settle(t.sa_next);
        static_for<2>([&](auto i) { a_part(t, kt + 2, i, IC<0>{}); });
        a_end(t, kt + 2);
      }
      uint32_t a_at[2] = {a_sub0 + cur * FEW_A_BYTES, a_sub1 + cur * FEW_A_BYTES}, b_at[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) b_at[x] = fb_base[0][x] + cur * TILE_BYTES;
      static_for<2>([&](auto s_tag) {
        constexpr int SUB = decltype(s_tag)::value;
        static_for<2>([&](auto b_tag) {
          constexpr int blk = decltype(b_tag)::value;
          fa[SUB][blk].v = lds_read_b128<blk * 4096>(a_at[SUB]);
        });
        static_for<NB>([&](auto b_tag) {
          constexpr int blk = decltype(b_tag)::value;
          if constexpr (B_KN) {
            static_for<2>([&](auto h_tag) {
              constexpr int half = decltype(h_tag)::value;
              fb[SUB][blk].h[half] = lds_read_tr_b64<SUB * 32 * TL::KN_ROW + half * 4 * TL::KN_ROW + (blk & 1) * 32>(b_at[blk >> 1]);
            });
          } else {
            fb[SUB][blk].v = lds_read_b128<blk * 2048>(b_at[SUB]);
          }
        });
      });
      static_for<2>([&](auto s_tag) {
        constexpr int SUB = decltype(s_tag)::value;
        lds_wait<SUB == 0 ? NREADS : 0>();      // the reads of the other sub-step may be under way
        static_for<2>([&](auto i) { static_for<NB>([&](auto j) { mma(IC<SUB>{}, i, j); }); });
      });
      cur = cur + 1 == FEW_RING ? 0 : cur + 1;
      nxt = nxt + 1 == FEW_RING ? 0 : nxt + 1;
      // the last MFMAs have written before the accumulators are read, or moved, which the compiler may do where paths join and
      // without a wait, since it does not know the statements above for what they are
      asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
    }
  };
  // one copy of the loop per number of live 32-row groups
  auto run_main = [&](TileState& t) __attribute__((always_inline)) {
    if constexpr (is_wgrad(MODE)) {
      main_loop(t, IC<HALF / 32>{});
    } else if constexpr (S == 128) {
      if (t.few) few_rows_loop(t); else if (t.nv == 2) main_loop(t, IC<2>{}); else main_loop(t, IC<1>{});
    } else {
      switch (t.nv) {
        case 4: main_loop(t, IC<4>{}); break;
        case 3: main_loop(t, IC<3>{}); break;
        case 2: main_loop(t, IC<2>{}); break;
        default: main_loop(t, IC<1>{}); break;
      }
    }
  };
  // ---------------- epilogue -----------------------------------------------------
  // acc[i][j][c] is the wave's element (row, col) with row = 16 i + (lane & 15) and col = 16 j + 4 (lane / 16) + c.
  // The wave stages its bf16 rows of S bytes in LDS of its own (its share of a ring slot; 16-byte pieces
  // swizzled by the row), a few rows at a time, and stores 16 bytes per lane in full row segments.
  // The accumulators are read out of the accumulation registers at the point of use, by hand: left to the
  // compiler they are moved (and spilled) in bulk where the copies of the main loop join.
  auto accq = [&](auto i_tag, auto j_tag) __attribute__((always_inline)) -> f32x4_t {
    constexpr int i = decltype(i_tag)::value, j = decltype(j_tag)::value;
    f32x4_t v;
    float x;
    const float c0 = acc[i][j][0], c1 = acc[i][j][1], c2 = acc[i][j][2], c3 = acc[i][j][3];
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c0));  v[0] = x;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c1));  v[1] = x;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c2));  v[2] = x;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c3));  v[3] = x;
    return v;
  };
  // GATE_UP with gate weights folded into h, DGRAD_H_GATE: the weights of the lane's NB rows, requested
  // right behind the main loop and awaited before the next tile's first loads are requested.
  float wv[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) wv[i] = 1.f;
  auto fetch_row_weights = [&](const TileState& t, const float* rw) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      int r = t.m0 + t.r0 + i * 16 + (lane & 15);  if (r > t.m_end - 1) r = t.m_end - 1;
      wv[i] = rw[r];
    }
    asm volatile("" ::: "memory");            // requested here, not where they are used
  };

  // The logits' epilogues.  A lane holds up to IT of the items in its wave's piece (place 0 to HALF - 1 of the row | column << 8, or -1), with
  // their place in HeadArgs::item and (HEAD_DZ) their terms; `many`: there are more, and the parts look them up.
  // Without a teacher these are the targets of the lane's rows.  Otherwise the bounds of the lists of the wave's blocks (in lanes 0 to NB - 1) are
  // requested with the tile's first loads, so that one latency, not two in a row, stands behind the main loop.
  // (What a lane of a tile of 128 needs of its rows comes with them; a tile of 256 has no registers for that.)
  constexpr int IT = HALF / 64;
  constexpr bool EARLY = S == 128;
  int early_target[IT] = {};
  f32x4_t early_term[IT] = {}, early_row[NB] = {};
  int item_lo = 0, item_hi = 0, list_lo = 0, list_hi = 0, item_at[IT], item_place[IT];
  bool many = false;
  f32x4_t item_term[MODE == HEAD_DZ ? IT : 1], rowp[NB];
  auto fetch_rows = [&](const TileState& t, f32x4_t (&to)[NB]) __attribute__((always_inline)) {
    const HeadPtr he = head_args();
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      int r = t.m0 + t.r0 + i * 16 + (lane & 15);
      if (r > t.m_end - 1) r = t.m_end - 1;
      to[i] = he->row[r];
    }
  };
  auto fetch_lists = [&](const TileState& t) __attribute__((always_inline)) {
    const HeadPtr he = head_args();
    const int first = t.m0 + t.r0, last = t.m_end - 1;
    if constexpr (EARLY && MODE == HEAD_DZ) fetch_rows(t, early_row);
    if (he->list_start == nullptr) {
#pragma unroll
      for (int k = 0; k < IT; ++k) {
        const int r = first + lane + 64 * k, row = r < t.m_wave ? r : last;
        early_target[k] = he->target[row];
        if constexpr (EARLY && MODE == HEAD_DZ) early_term[k] = he->terms[row];
      }
      asm volatile("" ::: "memory");
      return;
    }
    int b = (first >> 4) + (lane < NB ? lane : NB - 1);
    if (b > last >> 4) b = last >> 4;
    int strip = (he->col0 + t.n0 + wn * HALF) >> 6, end = strip + HALF / 64;
    if (strip > he->list_ld - 1) strip = he->list_ld - 1;
    if (end > he->list_ld - 1) end = he->list_ld - 1;
    const int32_t* start = he->list_start + static_cast<size_t>(b) * he->list_ld;
    list_lo = start[strip];
    list_hi = start[end];
    asm volatile("" ::: "memory");            // requested here, not where they are used
  };
  auto fetch_items = [&](const TileState& t) __attribute__((always_inline)) {
    const HeadPtr he = head_args();
    const int first = t.m0 + t.r0, last = t.m_end - 1, col = he->col0 + t.n0 + wn * HALF;
    many = false;
    if (he->list_start == nullptr) {
#pragma unroll
      for (int k = 0; k < IT; ++k) {
        const int r = lane + 64 * k, row = first + r < t.m_wave ? first + r : last;
        const int c = early_target[k] - col;
        item_at[k] = first + r < t.m_wave && c >= 0 && c < HALF ? r | c << 8 : -1;
        item_place[k] = row;
        if constexpr (MODE == HEAD_DZ) item_term[k] = EARLY ? early_term[k] : he->terms[row];
      }
    } else {
      item_lo = list_lo;
      item_hi = list_hi;
      const int n = lane < NB && first + lane * 16 < t.m_wave ? item_hi - item_lo : 0, end = wave_incl_scan(n);
      many = wave_lane(end, 63) > 64 * IT;
#pragma unroll
      for (int k = 0; k < IT; ++k) {
        const int i = lane + 64 * k;
        int part = 0;
#pragma unroll
        for (int p = 0; p < NB - 1; ++p) part += i >= wave_lane(end, p) ? 1 : 0;
        const int in = i - (__shfl(end, part) - __shfl(n, part)) + __shfl(item_lo, part);
        item_at[k] = -1;
        if (i < wave_lane(end, NB - 1)) {
          const size_t at = static_cast<size_t>((first >> 4) + part) * 16 * he->slots + in;
          const HeadItem x = he->items[at];
          const int r = part * 16 + (x.at & 15);
          item_at[k] = r | (static_cast<int>(x.at >> 4) - col) << 8;
          item_place[k] = (first + r) * he->slots + static_cast<int>(x.slot);
          if constexpr (MODE == HEAD_DZ) item_term[k] = he->terms[at];
        }
      }
    }
    if constexpr (MODE == HEAD_DZ) {
      if constexpr (EARLY) {
#pragma unroll
        for (int i = 0; i < NB; ++i) rowp[i] = early_row[i];
      } else {
        fetch_rows(t, rowp);
      }
    }
    asm volatile("" ::: "memory");            // requested here, not where they are used
  };

  // what the epilogue needs of a tile whose successor is set up already (and its first loads in flight: slot, and for the
  // SwiGLU derivative slot2, is what they leave free)
  struct Finished { int e, m0, n0, r0, m_wave, slot, slot2; bool second; };
  auto epilogue = [&](const Finished& t) __attribute__((always_inline)) {
    const ArgPtr ae = reload_args<ARG>();     // the epilogue reads its arguments afresh
    int tid = tid0;                           // laundered as in setup_tile
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, l16 = lane & 15, lq = lane >> 4;
    const int m_end = t.m_wave, n0 = t.n0;                               // end of the wave's valid rows
    const int grow0 = t.m0 + t.r0;                                       // wave's first output row
    const int gcol0 = n0 + wn * (MODE == GATE_UP ? S / 4 : HALF);        // wave's first output column
    constexpr int RB = S, RP = S / 16;          // bytes and 16-byte pieces of a staged row of all the wave's columns
    char* stage = lds + t.slot * TILE_BYTES + wave * TL::SHARE;
    // address of the 8 bytes of columns 4 lq .. + 3 of 16-column block `blk` in staged row `row`
    auto quad_addr = [&](int row, int blk) __attribute__((always_inline)) -> char* {
      return stage + row * RB + (((2 * blk + (lq >> 1)) ^ (row & (RP - 1))) << 4) + (lq & 1) * 8;
    };
    auto put_quad = [&](int row, int blk, const f32x4_t& v) __attribute__((always_inline)) {
      u32x2 o;
      o.x = pack_bf16(v[0], v[1]);
      o.y = pack_bf16(v[2], v[3]);
      *reinterpret_cast<u32x2*>(quad_addr(row, blk)) = o;
    };
    // Rows are stored (and g, u loaded) through buffer resources that end with the wave's last valid row: what lies past it
    // is dropped (reads as zero) by the hardware's range check, and a lane whose columns do not exist carries an offset
    // past every end (the row is part of the lane's offset, which is what the check looks at).  So the whole epilogue is
    // straight-line code, ragged or not.
    const int ncol = ae->N;
    int rows = m_end - grow0;
    rows = rows < 0 ? 0 : (rows > HALF ? HALF : rows);
    auto rows_of = [&](const void* base, int ld_bytes) __attribute__((always_inline)) {
      const char* first = scalarize(static_cast<const char*>(base) + static_cast<size_t>(grow0) * ld_bytes);
      return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(first), 0, __builtin_amdgcn_readfirstlane(rows * ld_bytes), 0x00020000);
    };
    typedef decltype(rows_of(nullptr, 0)) Rsrc;
    // as unsigned 2^31: not before the end of 128 rows of any width for which the loads' 32-bit lane offsets suffice, and
    // still past it with the row of a part added
    constexpr int PAST = INT_MIN;
    // PASSES staged passes of 64 / PIECES rows of RB bytes each (16-byte pieces swizzled by row & (RB / 16 - 1), region at
    // `base`), the PIECES pieces from PIECE0 on of each row: read into registers, and stored from there (first row
    // `first`, counted from the wave's first) to columns col0 + 8 piece.  NT: the output is not read again soon (g and u: not
    // before the backward pass; dWg, dWu and the head's dW: not by this layer at all), so its stores are marked non-temporal and leave
    // the caches to what the next kernels read (measured: 0.4-0.6 % of the step, most of it in the kernels that follow).
    auto read_staged = [&](u32x4* v, const char* base, auto rb_tag, auto passes_tag, auto piece0_tag, auto pieces_tag)
        __attribute__((always_inline)) {
      constexpr int RB = decltype(rb_tag)::value, PASSES = decltype(passes_tag)::value, PIECES = decltype(pieces_tag)::value;
      constexpr int RPP = 64 / PIECES, SWZ = RB / 16 - 1;
#pragma unroll
      for (int k = 0; k < PASSES; ++k) {
        const int row = k * RPP + lane / PIECES;
        v[k] = *reinterpret_cast<const u32x4*>(base + row * RB + (((decltype(piece0_tag)::value + lane % PIECES) ^ (row & SWZ)) << 4));
      }
    };
    auto store_rows = [&](auto nt_tag, const u32x4* v, Rsrc out, int first, auto passes_tag, auto pieces_tag)
        __attribute__((always_inline)) {
      constexpr int PASSES = decltype(passes_tag)::value, PIECES = decltype(pieces_tag)::value, RPP = 64 / PIECES;
      const int gc = gcol0 + lane % PIECES * 8;
      const int off = gc < ncol ? (lane / PIECES * ncol + gc) * 2 : PAST;
#pragma unroll
      for (int k = 0; k < PASSES; ++k)
        __builtin_amdgcn_raw_buffer_store_b128(v[k], out, off + (first + k * RPP) * ncol * 2, 0, decltype(nt_tag)::value ? 2 : 0);
    };

    // A wave with HALF - 32 rows or fewer takes a second copy, which tests in front of every part whether it has a row: the tests
    // end the overlap, but the parts left out are worth more.
    // Measured against masked stores issued part by part: gate_up 470 -> 459 us and the launch of dgrad_h 575 -> 560 us at
    // 65536 rows, d 2048, f 1024, 64 experts; 17 -> 13 and 25 -> 17 us where experts have 56 rows (d 128, f 512).
    // In every form a part's rows are read back from LDS as soon as they are staged and stored behind the arithmetic of the
    // part after it: with one wave per SIMD nothing else covers the round trip through LDS.
    if constexpr (MODE == GATE_UP) {
      // The first half of the blocks are g, the other half the same columns of u.  Parts of 16 rows: g in the first and u in
      // the second half of the staged rows, h = silu(g) * u (from the fp32 accumulators, times the row's gate weight if
      // the caller folds the weights into h) in rows of half their length behind them.
      const bool weighted = ae->row_weight != nullptr;
      constexpr int HP = RP / 2, GP = 16 * HP / 64;   // pieces of a row of g, u or h; passes of 64 pieces over 16 rows
      char* hstage = stage + 16 * RB;
      const Rsrc go = rows_of(ae->O0, ncol * 2), uo = rows_of(ae->O1, ncol * 2), ho = rows_of(ae->O2, ncol * 2);
      u32x4 v[3 * GP];
      auto store_part = [&](int part) __attribute__((always_inline)) {
        store_rows(IC<1>{}, v, go, part * 16, IC<GP>{}, IC<HP>{});
        store_rows(IC<1>{}, v + GP, uo, part * 16, IC<GP>{}, IC<HP>{});
        store_rows(IC<0>{}, v + 2 * GP, ho, part * 16, IC<GP>{}, IC<HP>{});
      };
      auto parts = [&](auto ragged_tag) __attribute__((always_inline)) {
      constexpr bool RAGGED = decltype(ragged_tag)::value != 0;
      static_for<NB>([&](auto i_tag) {
        constexpr int i = decltype(i_tag)::value;
        if constexpr (RAGGED) { if (i * 16 >= rows) return; }
        const int row = l16;
        const float w = weighted ? wv[i] : 1.f;
        static_for<NB / 2>([&](auto j_tag) {
          constexpr int j = decltype(j_tag)::value;
          const f32x4_t gv = accq(i_tag, IC<j>{});
          const f32x4_t uv = accq(i_tag, IC<j + NB / 2>{});
          put_quad(row, j, gv);
          put_quad(row, j + NB / 2, uv);
          u32x2 o;
          float h[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) h[c] = silu_f(gv[c]) * uv[c] * w;
          o.x = pack_bf16(h[0], h[1]);
          o.y = pack_bf16(h[2], h[3]);
          *reinterpret_cast<u32x2*>(hstage + row * (RB / 2) + (((2 * j + (lq >> 1)) ^ (row & (HP - 1))) << 4) + (lq & 1) * 8) = o;
        });
        __builtin_amdgcn_wave_barrier();
        if constexpr (!RAGGED && i > 0) store_part(i - 1);
        read_staged(v, stage, IC<RB>{}, IC<GP>{}, IC<0>{}, IC<HP>{});
        read_staged(v + GP, stage, IC<RB>{}, IC<GP>{}, IC<HP>{}, IC<HP>{});
        read_staged(v + 2 * GP, hstage, IC<RB / 2>{}, IC<GP>{}, IC<0>{}, IC<HP>{});
        __builtin_amdgcn_wave_barrier();
        if constexpr (RAGGED) store_part(i);
      });
      if constexpr (!RAGGED) store_part(NB - 1);
      };
      if (rows > HALF - 32) parts(IC<0>{}); else parts(IC<1>{});
    } else if constexpr (is_dgrad_h(MODE)) {
      // In parts of 16 rows, staged alternately in the wave's share of two ring slots: g rows in the first half, u rows in
      // the second half of the part's buffer, overwritten in place by dg and du.
      // DGRAD_H_GATE: the accumulators hold dh0 = dout[token] . Wd; the row's gate weight w turns them into
      // dh = w dh0, and the sum over a 64-column strip of dh0 * silu(g) * u is the strip's share of the
      // gradient of w (a lane holds 16 of the strip's columns of its row, lanes ^ 16, ^ 32 the others).
      constexpr bool GATE = (MODE == DGRAD_H_GATE);
      constexpr int GU_PASSES = 16 * RP / 64;   // 16 rows of RP pieces of 16 bytes, 64 per pass
      constexpr int GU_ROWS = 64 / RP;          // rows of a pass
      constexpr int UOFF = TL::SHARE / 2;
      const Rsrc gi = rows_of(ae->G, ncol * 2), ui = rows_of(ae->U, ncol * 2);
      const Rsrc dgo = rows_of(ae->O0, ncol * 2), duo = rows_of(ae->O1, ncol * 2);
      u32x4 pg[GU_PASSES], pu[GU_PASSES];
      const int gu_off = gcol0 + lane % RP * 8 < ncol ? (lane / RP * ncol + gcol0 + lane % RP * 8) * 2 : PAST;
      auto gu_load = [&](int part) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < GU_PASSES; ++p) {
          pg[p] = __builtin_amdgcn_raw_buffer_load_b128(gi, gu_off + (part * 16 + p * GU_ROWS) * ncol * 2, 0, 0);
          pu[p] = __builtin_amdgcn_raw_buffer_load_b128(ui, gu_off + (part * 16 + p * GU_ROWS) * ncol * 2, 0, 0);
        }
      };
      auto gu_stage = [&](char* buf) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < GU_PASSES; ++p) {
          const int row = p * GU_ROWS + lane / RP, piece = lane % RP;
          const int so = row * RB + ((piece ^ (row & (RP - 1))) << 4);
          *reinterpret_cast<u32x4*>(buf + so) = pg[p];
          *reinterpret_cast<u32x4*>(buf + UOFF + so) = pu[p];
        }
      };
      char* const bufs[2] = {stage, lds + t.slot2 * TILE_BYTES + wave * TL::SHARE};
      int qoff[NB];                 // offsets of the lane's quads in a part's buffer: the same for every part
#pragma unroll
      for (int j = 0; j < NB; ++j) qoff[j] = static_cast<int>(quad_addr(l16, j) - stage);
      u32x4 v[2 * GU_PASSES];
      auto store_part = [&](int part) __attribute__((always_inline)) {
        store_rows(IC<0>{}, v, dgo, part * 16, IC<GU_PASSES>{}, IC<RP>{});
        store_rows(IC<0>{}, v + GU_PASSES, duo, part * 16, IC<GU_PASSES>{}, IC<RP>{});
      };
      constexpr int STRIPS = HALF / 64;         // 64-column strips of the wave's piece
      float dpart[NB][STRIPS];
      auto parts = [&](auto ragged_tag) __attribute__((always_inline)) {
      constexpr bool RAGGED = decltype(ragged_tag)::value != 0;
      gu_load(0);
      gu_stage(bufs[0]);
      gu_load(1);
      static_for<NB>([&](auto part_tag) {
        constexpr int part = decltype(part_tag)::value;
        if constexpr (RAGGED) { if (part * 16 >= rows) return; }
        char* const buf = bufs[part & 1];
        const float wrow = GATE ? wv[part] : 1.f;
        float dsum[STRIPS] = {};
        __builtin_amdgcn_wave_barrier();
        // the lane's g and u quads of the part, read in one go: the quads are overwritten in place below, so
        // reads issued one by one would each wait behind the previous quad's write
        u32x2 gqs[NB], uqs[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          gqs[j] = *reinterpret_cast<const u32x2*>(buf + qoff[j]);
          uqs[j] = *reinterpret_cast<const u32x2*>(buf + qoff[j] + UOFF);
        }
        static_for<NB>([&](auto j_tag) {
          constexpr int j = decltype(j_tag)::value;
          const f32x4_t dhv = accq(part_tag, j_tag);
          char* ga = buf + qoff[j];
          char* ua = ga + UOFF;
          const u32x2 gq = gqs[j];
          const u32x2 uq = uqs[j];
          const float g4[4] = {bf16lo(gq.x), bf16hi(gq.x), bf16lo(gq.y), bf16hi(gq.y)};
          const float u4[4] = {bf16lo(uq.x), bf16hi(uq.x), bf16lo(uq.y), bf16hi(uq.y)};
          float dg[4], du[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float sg = sigmoid_f(g4[c]);
            if constexpr (GATE) {
              const float dh0 = dhv[c];
              const float sl = g4[c] * sg;                 // silu(g)
              const float t0 = dh0 * u4[c];
              dsum[j >> 2] = __builtin_fmaf(t0, sl, dsum[j >> 2]);   // 4 blocks to a strip
              du[c] = (dh0 * wrow) * sl;
              dg[c] = (t0 * wrow) * (sg * __builtin_fmaf(g4[c], 1.0f - sg, 1.0f));
            } else {
              const float dh = dhv[c];
              const float x = dh * sg;                     // shared by both derivatives
              du[c] = x * g4[c];
              dg[c] = (x * u4[c]) * __builtin_fmaf(g4[c], 1.0f - sg, 1.0f);
            }
          }
          u32x2 o;
          o.x = pack_bf16(dg[0], dg[1]);  o.y = pack_bf16(dg[2], dg[3]);
          *reinterpret_cast<u32x2*>(ga) = o;
          o.x = pack_bf16(du[0], du[1]);  o.y = pack_bf16(du[2], du[3]);
          *reinterpret_cast<u32x2*>(ua) = o;
        });
        if constexpr (GATE) {
#pragma unroll
          for (int s2 = 0; s2 < STRIPS; ++s2) {
            float x = dsum[s2];
            x += __shfl_xor(x, 16, 64);
            x += __shfl_xor(x, 32, 64);
            dpart[part][s2] = x;
          }
        }
        __builtin_amdgcn_wave_barrier();
        if constexpr (part + 1 < NB) gu_stage(bufs[(part + 1) & 1]);   // awaits the loads of part + 1
        __builtin_amdgcn_wave_barrier();
        if constexpr (!RAGGED && part > 0) store_part(part - 1);
        read_staged(v, buf, IC<RB>{}, IC<GU_PASSES>{}, IC<0>{}, IC<RP>{});
        read_staged(v + GU_PASSES, buf + UOFF, IC<RB>{}, IC<GU_PASSES>{}, IC<0>{}, IC<RP>{});
        __builtin_amdgcn_wave_barrier();
        if constexpr (RAGGED) store_part(part);
        if constexpr (part + 2 < NB) gu_load(part + 2);
      });
      if constexpr (!RAGGED) store_part(NB - 1);
      };
      if (rows > HALF - 32) parts(IC<0>{}); else if (rows > 0) parts(IC<1>{});
      if constexpr (GATE) {
        // the strips' shares of the gate gradient, stored behind everything else
        const int strips = ncol >> 6;
        const Rsrc dpo = rows_of(ae->dgate_part, strips * 4);
#pragma unroll
        for (int s2 = 0; s2 < STRIPS; ++s2) {
          // a strip past the last column has no share
          const int off = lq == 0 && gcol0 + s2 * 64 < ncol ? (l16 * strips + (gcol0 >> 6) + s2) * 4 : PAST;
          static_for<NB>([&](auto part_tag) {
            constexpr int part = decltype(part_tag)::value;
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(dpart[part][s2]), dpo, off + part * 16 * strips * 4, 0, 0);
          });
        }
      }
    } else if constexpr (is_logits(MODE)) {
      // In parts of 16 rows.  A part that holds items puts its logits into LDS (rows of HALF floats, 16-byte pieces swizzled by the row), where
      // the items are picked up, a lane each; HEAD_STATS takes them out of the maximum and the sums there: a loss near zero is the logarithm
      // of one plus what the other columns weigh, which the difference of two whole sums would lose.
      // A sum's exponentials are taken relative to 2^E, E the row's maximum in units of log2 rounded up: exact in the fused product below and
      // wherever sums of several strips are put on one scale.
      const HeadPtr he = head_args();
      constexpr float NONE = -__builtin_inff();
      const int left = ncol - gcol0;                       // columns that the wave has
      const float c1 = he->c1, c2 = he->c2;
      const bool two = he->two != 0;
      auto z_piece = [&](int row, int piece) __attribute__((always_inline)) {
        return reinterpret_cast<float*>(stage + row * (HALF * 4) + ((piece ^ row) << 4));
      };
      // f(there, row, place in HeadArgs::item, terms, its logit's place in LDS) for the part's items, a lane each, all lanes together
      auto over_items = [&](auto part_tag, auto&& f) __attribute__((always_inline)) {
        constexpr int part = decltype(part_tag)::value;
        if (!many) {
#pragma unroll
          for (int k = 0; k < IT; ++k) {
            const bool there = item_at[k] >= 0 && (item_at[k] >> 4 & (HALF / 16 - 1)) == part;
            const int row = there ? item_at[k] & 15 : 0, c = there ? item_at[k] >> 8 : 0;
            f(there, row, item_place[k], item_term[MODE == HEAD_DZ ? k : 0], z_piece(row, c >> 2) + (c & 3));
          }
          return;
        }
        const int hi = wave_lane(item_hi, part);
        const size_t first = static_cast<size_t>((grow0 >> 4) + part) * 16 * he->slots;
        for (int n0 = wave_lane(item_lo, part); n0 < hi; n0 += 64) {
          const int n = n0 + lane < hi ? n0 + lane : hi - 1;
          const HeadItem x = he->items[first + n];
          const int row = x.at & 15, c = static_cast<int>(x.at >> 4) - he->col0 - gcol0;
          f(n0 + lane < hi, row, (grow0 + part * 16 + row) * he->slots + static_cast<int>(x.slot), MODE == HEAD_DZ ? he->terms[first + n] : f32x4_t{},
            z_piece(row, c >> 2) + (c & 3));
        }
      };
      auto has_items = [&](auto part_tag) __attribute__((always_inline)) {
        constexpr int part = decltype(part_tag)::value;
        if (many) return wave_lane(item_hi, part) > wave_lane(item_lo, part);
        bool mine = false;
#pragma unroll
        for (int k = 0; k < IT; ++k) mine = mine || (item_at[k] >= 0 && (item_at[k] >> 4 & (HALF / 16 - 1)) == part);
        return __ballot(mine) != 0;
      };
      // (a wave's LDS operations are carried out in order; the compiler is not to change theirs)
      auto in_order = []() __attribute__((always_inline)) { __builtin_amdgcn_wave_barrier(); asm volatile("" ::: "memory"); };
      auto put_logits = [&](const auto& v) __attribute__((always_inline)) {
        static_for<NB>([&](auto j) { *reinterpret_cast<f32x4_t*>(z_piece(l16, 4 * decltype(j)::value + lq)) = v[decltype(j)::value]; });
        in_order();
      };
      auto get_logits = [&](auto& v) __attribute__((always_inline)) {
        in_order();
        static_for<NB>([&](auto j) { v[decltype(j)::value] = *reinterpret_cast<const f32x4_t*>(z_piece(l16, 4 * decltype(j)::value + lq)); });
        in_order();
      };
      auto mask = [&](auto& v, float with) __attribute__((always_inline)) {
        if (left >= HALF) return;
        static_for<NB>([&](auto j_tag) {
          constexpr int j = decltype(j_tag)::value;
#pragma unroll
          for (int c = 0; c < 4; ++c) v[j][c] = 16 * j + 4 * lq + c < left ? v[j][c] : with;
        });
      };
      if constexpr (MODE == HEAD_STATS) {
        const int planes = two ? 3 : 2;
        const size_t block = static_cast<size_t>(he->strips) * planes * 16;
        float* const out = he->part + (grow0 >> 4) * block + gcol0 / HALF * planes * 16 + lane;
        static_for<NB>([&](auto i_tag) {
          constexpr int i = decltype(i_tag)::value;
          if (i * 16 >= rows || left <= 0) return;
          f32x4_t v[NB];
          static_for<NB>([&](auto j) { v[decltype(j)::value] = accq(i_tag, j); });
          if (has_items(i_tag)) {
            put_logits(v);
            over_items(i_tag, [&](bool there, int, int at, const f32x4_t&, float* z) __attribute__((always_inline)) { if (there) he->item[at] = *z; });
            in_order();
            over_items(i_tag, [&](bool there, int, int, const f32x4_t&, float* z) __attribute__((always_inline)) { if (there) *z = NONE; });
            get_logits(v);
          }
          mask(v, NONE);
          float m = NONE;
#pragma unroll
          for (int j = 0; j < NB; ++j) m = fmaxf(fmaxf(fmaxf(m, v[j][0]), fmaxf(v[j][1], v[j][2])), v[j][3]);
          m = quads_reduce(m, [](float x, float y) __attribute__((always_inline)) { return fmaxf(x, y); });
          const float e1 = m > NONE ? ceilf(m * c1) : 0.f;
          float s1 = 0.f, s2 = 0.f;
#pragma unroll
          for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) s1 += __builtin_amdgcn_exp2f(__builtin_fmaf(v[j][c], c1, -e1));
          const auto add = [](float x, float y) __attribute__((always_inline)) { return x + y; };
          s1 = quads_reduce(s1, add);
          if (two) {
            const float e2 = m > NONE ? ceilf(m * c2) : 0.f;
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
              for (int c = 0; c < 4; ++c) s2 += __builtin_amdgcn_exp2f(__builtin_fmaf(v[j][c], c2, -e2));
            s2 = quads_reduce(s2, add);
          }
          if (lq < planes && i * 16 + l16 < rows) out[i * block] = lq == 0 ? m : lq == 1 ? s1 : s2;
        });
      } else {
        const int ld = ae->M;
        const Rsrc oo = rows_of(ae->O0, ld * 2);
        const int all_rows = ae->offsets[1];
        const bool lows = all_rows <= he->lo;
        const Rsrc ol = rows_of(ae->O0 + (lows ? static_cast<size_t>(all_rows) * ld : 0), ld * 2);
        constexpr int PASSES = 16 * RP / 64;
        u32x4 v4[PASSES];
        const int gc = gcol0 + lane % RP * 8;
        const int off = gc < ld ? (lane / RP * ld + gc) * 2 : PAST;
        auto stage_part = [&](const f32x4_t (&v)[NB]) __attribute__((always_inline)) {
          static_for<NB>([&](auto j) { put_quad(l16, decltype(j)::value, v[decltype(j)::value]); });
          in_order();
          read_staged(v4, stage, IC<RB>{}, IC<PASSES>{}, IC<0>{}, IC<RP>{});
          in_order();
        };
        auto store_part = [&](int part, Rsrc out) __attribute__((always_inline)) {
#pragma unroll
          for (int k = 0; k < PASSES; ++k)
            __builtin_amdgcn_raw_buffer_store_b128(v4[k], out, off + (part * 16 + k * (64 / RP)) * ld * 2, 0, 0);
        };
        const auto rounded = [](float x) __attribute__((always_inline)) { return bf16_to_f32(f32_to_bf16(x)); };
        static_for<NB>([&](auto i_tag) {
          constexpr int i = decltype(i_tag)::value;
          if (i * 16 >= rows) return;
          const f32x4_t p = rowp[i];
          f32x4_t v[NB];
          static_for<NB>([&](auto j) { v[decltype(j)::value] = accq(i_tag, j); });
          auto gradient = [&](float z) __attribute__((always_inline)) {
            const float g = __builtin_amdgcn_exp2f(__builtin_fmaf(z, c1, -p[0])) * p[1];
            return two ? __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(z, c2, -p[2])), p[3], g) : g;
          };
          if (has_items(i_tag)) {
            // the gradient at the items replaces their logits; a lane knows it by its bits, which are made to differ from the logit's
            put_logits(v);
            over_items(i_tag, [&](bool there, int row, int at, const f32x4_t& t, float* zp) __attribute__((always_inline)) {
              const float z = *zp, lse = __shfl(p[0], row);
              float g = t[0], lse_t = 0.f, of_p = 0.f;
              if (two) { lse_t = __shfl(p[2], row); of_p = __shfl(p[3], row); }
              if (t[1] != 0.f) g = __builtin_fmaf(t[1], expm1f(__builtin_fmaf(z, he->over_tau, -t[2])), g);
              else if (two) g = __builtin_fmaf(of_p, __builtin_amdgcn_exp2f(__builtin_fmaf(z, c2, -lse_t)), g);
              if (t[3] != 0.f) g = __builtin_fmaf(t[3], __builtin_amdgcn_exp2f(__builtin_fmaf(z, c1, -lse)), g);
              if (!there) return;
              he->item[at] = g - rounded(g);
              *zp = __uint_as_float(__float_as_uint(g) ^ (__float_as_uint(g) == __float_as_uint(z) ? 1u : 0u));
            });
            f32x4_t special[NB];
            get_logits(special);
            static_for<NB>([&](auto j_tag) {
              constexpr int j = decltype(j_tag)::value;
#pragma unroll
              for (int c = 0; c < 4; ++c)
                v[j][c] = __float_as_uint(special[j][c]) != __float_as_uint(v[j][c]) ? special[j][c] : gradient(v[j][c]);
            });
          } else {
            static_for<NB>([&](auto j_tag) {
              constexpr int j = decltype(j_tag)::value;
#pragma unroll
              for (int c = 0; c < 4; ++c) v[j][c] = gradient(v[j][c]);
            });
          }
          mask(v, 0.f);
          if constexpr (i > 0) { if (!lows) store_part(i - 1, oo); }     // behind the arithmetic of the part after it, as above
          stage_part(v);
          if (lows) {
            store_part(i, oo);
            static_for<NB>([&](auto j) {
#pragma unroll
              for (int c = 0; c < 4; ++c) v[decltype(j)::value][c] -= rounded(v[decltype(j)::value][c]);
            });
            stage_part(v);
            store_part(i, ol);
          }
        });
        if (!lows && rows > 0) store_part((rows - 1) >> 4, oo);
      }
    } else if (MODE == HEAD_DX || (MODE == HEAD_DW && ae->E > 1)) {
      // a part's sums in 32 bits, behind those of the parts before it
      float* const out = reinterpret_cast<float*>(MODE == HEAD_DX ? ae->O0 : ae->O1) + static_cast<size_t>(t.e) * (MODE == HEAD_DX ? ae->offsets[1] : ae->K) * ncol;
      const Rsrc oo = rows_of(out, ncol * 4);
      const bool add = MODE == HEAD_DX && ae->stream_rows != 0;
      static_for<NB>([&](auto i_tag) {
        constexpr int i = decltype(i_tag)::value;
        if (i * 16 >= rows) return;
        static_for<NB>([&](auto j_tag) {
          constexpr int j = decltype(j_tag)::value;
          const int gc = gcol0 + 16 * j + 4 * lq;
          const int off = gc < ncol ? (l16 * ncol + gc) * 4 : PAST;
          f32x4_t v = accq(i_tag, j_tag);
          if (add) v += __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(oo, off + i * 16 * ncol * 4, 0, 0));
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), oo, off + i * 16 * ncol * 4, 0, 0);
        });
      });
    } else {
      uint16_t* out = t.second ? ae->O1 : ae->O0;
      if constexpr (is_wgrad(MODE) && MODE != HEAD_DW) out += static_cast<size_t>(t.e) * ae->M * ncol;
      const Rsrc oo = rows_of(out, ncol * 2);
      constexpr int PASSES = 32 * RP / 64;
      u32x4 v[PASSES];
      // parts of 32 rows
      auto store_part = [&](int part) __attribute__((always_inline)) {
        store_rows(IC<(MODE == WGRAD_GATHER || MODE == HEAD_DW) ? 1 : 0>{}, v, oo, part * 32, IC<PASSES>{}, IC<RP>{});
      };
      auto parts = [&](auto ragged_tag) __attribute__((always_inline)) {
      constexpr bool RAGGED = decltype(ragged_tag)::value != 0;
      static_for<HALF / 32>([&](auto part_tag) {
        constexpr int part = decltype(part_tag)::value;
        if constexpr (RAGGED) { if (part * 32 >= rows) return; }
        static_for<2>([&](auto i2_tag) {
          constexpr int i2 = decltype(i2_tag)::value;
          static_for<NB>([&](auto j_tag) { put_quad(i2 * 16 + l16, decltype(j_tag)::value, accq(IC<part * 2 + i2>{}, j_tag)); });
        });
        __builtin_amdgcn_wave_barrier();
        if constexpr (!RAGGED && part > 0) store_part(part - 1);
        read_staged(v, stage, IC<RB>{}, IC<PASSES>{}, IC<0>{}, IC<RP>{});
        __builtin_amdgcn_wave_barrier();
        if constexpr (RAGGED) store_part(part);
      });
      if constexpr (!RAGGED) store_part(HALF / 32 - 1);
      };
      if (rows > HALF - 32) parts(IC<0>{}); else parts(IC<1>{});
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): this wave's staging reads are done
  };

  // ---------------- the tile loop ------------------------------------------------
  // A workgroup that always took the same place of an XCD's run would meet the same row tile of every expert whose
  // number of row tiles divides the run, the whole one or the ragged one; so the places move on by one each round
  // (inside a run, where runs are whole: the list stays covered once).
  int tile = first_tile;
  // Where experts have few row tiles (three or fewer on average) the launch waits for weights, and an expert with one row
  // tile needs far more of them per operation than one with many.  The runs are then taken from the two ends of the list in
  // turn, so that a round asks memory for two stretches of experts instead of one.  What they hold depends on the load: inside
  // a class the list is in index order.  Forward and backward pass, in us, list from the front / from both ends, zipf-like
  // load with the experts sorted by size, reversed, in two random orders, and an even load:
  //   64 experts, 2048 tokens, d 2048   949/909  994/980  965/956  983/961  959/942
  //   128 experts, 3000 tokens, d 1024  918/905  902/892  978/947  987/963  770/763
  //   96 experts, 4099 tokens, d 2048   1651/1607  1677/1687  1709/1702  1628/1657  1503/1501
  // (Listing the experts by their tile counts first changed this by -3 to +3 %, on average by nothing.)  Not with reductions
  // under 16 steps: there the experts that straddle two runs, fetched twice when the runs are far apart in time, weigh more
  // (down of 128 experts with 250 rows and 8 steps: 116 -> 124 us), nor with more row tiles (no difference).
  bool mix = false;
  if constexpr (!is_wgrad(MODE) && !is_logits(MODE) && MODE != HEAD_DX) mix = a.K * (MODE == DGRAD_X ? 2 : 1) >= 16 * BK && total <= 3 * a.E * a.n_tiles;
  const int run = static_cast<int>(gridDim.x >> 3);
  const int whole_runs = total / run;
  int block = first_tile / run, place = first_tile - block * run;
  if constexpr (MODE == HEAD_DW) tile = deal.extra > 0 ? deal.first : deal.skipped + first_tile;
  auto list_entry = [&]() __attribute__((always_inline)) {
    if (MODE == HEAD_DW || block >= whole_runs) return tile;
    return (mix ? ((block & 1) ? whole_runs - 1 - (block >> 1) : (block >> 1)) : block) * run + place;
  };
  if (tile < total) {
    TileState cur;
    setup_tile(list_entry(), cur);
    if constexpr (is_logits(MODE)) fetch_lists(cur);
    first_loads(cur);
    for (;;) {
      last_first_loads(cur);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] = 0.f;
      run_main(cur);
      wg_barrier();                             // every wave is done with the operand tiles
      bool weighted = (MODE == DGRAD_H_GATE);
      if constexpr (MODE == GATE_UP) weighted = a.row_weight != nullptr;
      if constexpr (MODE == GATE_UP || MODE == DGRAD_H_GATE) {
        if (weighted) fetch_row_weights(cur, a.row_weight);
      }
      if constexpr (is_logits(MODE)) fetch_items(cur);
      Finished done{cur.e, cur.m0, cur.n0, cur.r0, cur.m_wave, 0, 4, cur.second};
      if constexpr (MODE == HEAD_DW) {
        if (deal.extra > 1) tile += deal.by;
        else if (deal.extra == 1) tile = deal.skipped + first_tile;
        else tile += gridDim.x;
        deal.extra -= deal.extra > 0;
      } else {
        tile += gridDim.x;
      }
      const bool more = tile < total;
      if (more) {
        block += 8;
        place = place + 1 == run ? 0 : place + 1;
        setup_tile(list_entry(), cur);
        done.slot = __builtin_amdgcn_readfirstlane(spare_slot(cur));
        if constexpr (is_dgrad_h(MODE)) done.slot2 = __builtin_amdgcn_readfirstlane(spare_slot2(cur));
      }
      if constexpr (MODE == GATE_UP || MODE == DGRAD_H_GATE) {
        // (a use that the compiler sees: left to the epilogue, its wait would cover the first loads too)
#pragma unroll
        for (int i = 0; i < NB; ++i) asm volatile("" : "+v"(wv[i]));
      }
      if constexpr (is_logits(MODE)) {
#pragma unroll
        for (int k = 0; k < IT; ++k) asm volatile("" : "+v"(item_at[k]), "+v"(item_place[k]));
        if constexpr (MODE == HEAD_DZ) {
#pragma unroll
          for (int k = 0; k < IT; ++k) asm volatile("" : "+v"(item_term[k]));
#pragma unroll
          for (int i = 0; i < NB; ++i) asm volatile("" : "+v"(rowp[i]));
        }
        if (more) fetch_lists(cur);
      }
      if (more) first_loads(cur);
      epilogue(done);
      // a wave stages in, and loads into, its own share of a slot only: no barrier between epilogue and later loads
      if (!more) break;
    }
  }
  return tile - total;
}

// The launch is persistent: gridDim.x workgroups (one per compute unit) walk the tile list.
// Workgroups are dealt to the 8 XCDs round-robin, so workgroup b takes position
// (b % 8) * (gridDim.x / 8) + b / 8 of every round: each XCD then works on a run of
// consecutive tiles (same expert, neighbouring panels) that share its L2.
__device__ __forceinline__ int first_list_position() {
  const int per_xcd = gridDim.x >> 3;
  return (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
}

template <int MODE, int S>
__global__ __launch_bounds__(GEMM_THREADS, Tile<S>::PER_CU) void grouped_gemm_kernel(GemmArgs a) {
  gemm_tile_list<MODE, S, 0>(a, first_list_position());
}

// The constants of the model of a tile's time (see below, where tile edges are chosen).
template <int S> struct TileCost;
template <> struct TileCost<256> { static constexpr double FIXED = 5.2, WGRAD = 6.0, STEP = 1.0, SWIGLU_BWD = 16.0, RAGGED = 0.5; };
template <> struct TileCost<128> { static constexpr double FIXED = 2.7, WGRAD = 3.8, STEP = 0.75, SWIGLU_BWD = 9.0, RAGGED = 0.8; };

// dx and dW of the head in one launch.  dx has few tiles with long reductions: in the last round of them `idle` workgroups have none, and take
// as many tiles of dW as fit into that time; the rest is dealt to all in turn, to those first that have waited.
struct HeadDeal { int idle, extra; };
__host__ __device__ __forceinline__ HeadDeal head_deal(int dx_tiles, float dx_each, int dw_tiles, float dw_each, int places) {
  const int rest = dx_tiles % places;
  if (rest == 0) return {places, 0};
  const int idle = places - rest, fit = static_cast<int>(dx_each / dw_each), most = dw_tiles / idle;
  return {idle, fit < most ? fit : most};
}
template <int S> __host__ __device__ __forceinline__ float head_dx_each(int steps, int parts) {
  return static_cast<float>(TileCost<S>::FIXED) + static_cast<float>(TileCost<S>::STEP) * static_cast<float>(steps) / static_cast<float>(parts);
}
template <int S> __host__ __device__ __forceinline__ float head_dw_each(int steps, int parts) {
  return static_cast<float>(TileCost<S>::WGRAD) + 1.1f * static_cast<float>(TileCost<S>::STEP) * static_cast<float>(steps) / static_cast<float>(parts);
}
// How long the two take together, in the model's units: half the workgroup that ends last, half the mean (idle units leave the others power).
__host__ __device__ __forceinline__ float head_bwd_time(int dx_tiles, float dx_each, int dw_tiles, float dw_each, int places) {
  const HeadDeal deal = head_deal(dx_tiles, dx_each, dw_tiles, dw_each, places);
  const int rounds = dx_tiles / places, left = dw_tiles - deal.idle * deal.extra, whole = left / places, rest = left - whole * places;
  float last = rounds * dx_each + (deal.extra + whole + (rest > 0 ? 1 : 0)) * dw_each;
  if (dx_tiles > rounds * places) {
    const float busy = (rounds + 1) * dx_each + (whole + (rest > deal.idle ? 1 : 0)) * dw_each;
    last = busy > last ? busy : last;
  }
  return 0.5f * (last + (dx_tiles * dx_each + dw_tiles * dw_each) / places);
}
template <int S>
__global__ __launch_bounds__(GEMM_THREADS, Tile<S>::PER_CU) void grouped_gemm_head_bwd_kernel(GemmArgs a, GemmArgs b) {
  const int next = gemm_tile_list<HEAD_DX, S, 0>(a, first_list_position());
  const int parts = a.row_token[0], dx_tiles = (a.offsets[1] + S - 1) / S * a.n_tiles * parts, dw_tiles = b.E * b.m_tiles_cap * b.n_tiles;
  const HeadDeal d = head_deal(dx_tiles, head_dx_each<S>((a.M + BK - 1) / BK, parts), dw_tiles, head_dw_each<S>((b.offsets[1] + BK - 1) / BK, b.E), gridDim.x);
  const int extra = __builtin_amdgcn_readfirstlane(d.extra);
  gemm_tile_list<HEAD_DW, S, 1>(b, next, Deal{next < d.idle ? extra : 0, next, d.idle, d.idle * extra});
}

template <int MODE, int S>
__global__ __launch_bounds__(GEMM_THREADS, Tile<S>::PER_CU) void grouped_gemm_head_kernel(GemmArgs a, HeadArgs) {
  gemm_tile_list<MODE, S, 0>(a, first_list_position());
}

// Two products that do not depend on each other in one launch: the tile list of the second follows
// that of the first, so the workgroups that run out of tiles of the first go on with the second
// instead of idling until the next launch (one tail and one start-up instead of two).
template <int MODE_A, int MODE_B, int S>
__global__ __launch_bounds__(GEMM_THREADS, Tile<S>::PER_CU) void grouped_gemm_pair_kernel(GemmArgs a, GemmArgs b) {
  const int next = gemm_tile_list<MODE_A, S, 0>(a, first_list_position());
  gemm_tile_list<MODE_B, S, 1>(b, next);
}

// Per-device facts, looked up once per device: HIP keeps function attributes and the number of compute
// units per device, and a process may drive several.  Races between host threads are benign (both write
// the same values).
constexpr int MAX_DEVICES = 64;
int current_device() {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) { (void)hipGetLastError(); dev = 0; }
  return dev >= 0 && dev < MAX_DEVICES ? dev : 0;
}
// Workgroups of the persistent launch: as many per compute unit as the LDS allows (one or two),
// a multiple of 8 so that every XCD gets the same share, and no more than there can be tiles.
int compute_units() {
  static int cus_of[MAX_DEVICES] = {};
  const int dev = current_device();
  int cus = cus_of[dev];
  if (cus == 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 8) {
      (void)hipGetLastError();
      n = 256;
    }
    cus = cus_of[dev] = n & ~7;
  }
  return cus;
}
template <int S> int persistent_grid(long long max_tiles) {
  const int most = Tile<S>::PER_CU * compute_units();
  long long g = (max_tiles + 7) & ~7ll;
  if (g > most) g = most;
  if (g < 8) g = 8;
  return static_cast<int>(g);
}
// Raises the kernel's dynamic-LDS limit on the current device, once per device.
template <typename K>
int configure_lds(K kernel, int bytes, bool (&done)[MAX_DEVICES]) {
  const int dev = current_device();
  if (done[dev]) return MOE_OK;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) !=
      hipSuccess) {
    (void)hipGetLastError();
    return MOE_ERR_LAUNCH;
  }
  done[dev] = true;
  return MOE_OK;
}

template <int MODE, int S>
int launch_gemm(const GemmArgs& a, long long max_tiles, hipStream_t s, const char* name) {
  const dim3 grid(persistent_grid<S>(max_tiles));
  static bool configured[MAX_DEVICES] = {};
  if (configure_lds(&grouped_gemm_kernel<MODE, S>, Tile<S>::LDS, configured) != MOE_OK) return MOE_ERR_LAUNCH;
  MOE_LAUNCH(name, (grouped_gemm_kernel<MODE, S>), grid, dim3(GEMM_THREADS), Tile<S>::LDS, s, a);
  return moe_check_launch();
}

template <int MODE, int S>
int launch_gemm_head(const GemmArgs& a, const HeadArgs& h, long long max_tiles, hipStream_t s, const char* name) {
  const dim3 grid(persistent_grid<S>(max_tiles));
  static bool configured[MAX_DEVICES] = {};
  if (configure_lds(&grouped_gemm_head_kernel<MODE, S>, Tile<S>::LDS, configured) != MOE_OK) return MOE_ERR_LAUNCH;
  MOE_LAUNCH(name, (grouped_gemm_head_kernel<MODE, S>), grid, dim3(GEMM_THREADS), Tile<S>::LDS, s, a, h);
  return moe_check_launch();
}

template <int S>
int launch_gemm_head_bwd(const GemmArgs& a, const GemmArgs& b, long long max_tiles, hipStream_t s, const char* name) {
  const dim3 grid(persistent_grid<S>(max_tiles));
  static bool configured[MAX_DEVICES] = {};
  if (configure_lds(&grouped_gemm_head_bwd_kernel<S>, Tile<S>::LDS, configured) != MOE_OK) return MOE_ERR_LAUNCH;
  MOE_LAUNCH(name, (grouped_gemm_head_bwd_kernel<S>), grid, dim3(GEMM_THREADS), Tile<S>::LDS, s, a, b);
  return moe_check_launch();
}

template <int MODE_A, int MODE_B, int S>
int launch_gemm_pair(const GemmArgs& a, const GemmArgs& b, long long max_tiles, hipStream_t s, const char* name) {
  const dim3 grid(persistent_grid<S>(max_tiles));
  static bool configured[MAX_DEVICES] = {};
  if (configure_lds(&grouped_gemm_pair_kernel<MODE_A, MODE_B, S>, Tile<S>::LDS, configured) != MOE_OK) return MOE_ERR_LAUNCH;
  MOE_LAUNCH(name, (grouped_gemm_pair_kernel<MODE_A, MODE_B, S>), grid, dim3(GEMM_THREADS), Tile<S>::LDS, s, a, b);
  return moe_check_launch();
}

// The launches fill in what depends on the tile's edge: column tiles, row tiles and the bound on the tile list.
int ceil_div(int n, int by) { return (n + by - 1) / by; }
template <int MODE, int S>
long long count_tiles(GemmArgs& a, int R_cap) {
  if constexpr (is_wgrad(MODE)) {
    a.n_tiles = ceil_div(a.N, S);
    a.m_tiles_cap = ceil_div(a.M, S);         // row tiles of one expert's dW
    return static_cast<long long>(a.n_tiles) * a.m_tiles_cap * a.E * (a.A1 != nullptr ? 2 : 1);
  } else {
    a.n_tiles = ceil_div(a.N, MODE == GATE_UP ? S / 2 : S);
    a.m_tiles_cap = R_cap / S + a.E;
    return static_cast<long long>(a.n_tiles) * a.m_tiles_cap;
  }
}

// Which tile edge a launch takes: the one for which the model below expects less time.  Both give the same bits.
//
// 256: half the operand bytes per operation, and what long lists are quickest with.  128: two workgroups share a compute
// unit, so that one's waits and epilogue lie under the other's main loop; four times the tiles, so that a short list still
// reaches every compute unit; a quarter of the epilogue behind the last step of a reduction of a few; half the padding where
// experts have few rows or d, f are no multiple of 256.
//
// The model, in units of one K step of a 256-edge tile (1.4 us): a tile costs something fixed (start, epilogue) and something
// per step.  A launch takes its tiles' sum, spread over the places of the chip, plus one tile of the longest kind, since a list
// rarely ends evenly; a list alone in its launch also ends on whole rounds.  The row tiles are counted for an even load of
// the expected rows; RAGGED is what the last one of an expert counts for.  The constants are a fit to 7700 layers of 64 to 12000
// tokens, d and f 128 to 4096, 4 to 240 experts, all or a share of them local, even and zipf-like loads (four launches each, timed
// with both edges).  On 26900 others the edge chosen is on average 1.05 % slower than the better one (gate_up 0.8, down 0.7, dgrad_h with dWd 1.05, dgrad_x
// with dWg and dWu 1.6), always 256 17 % slower, always 128 4 %; constants fitted to these themselves reach 1.0 %.  In 4 % of the launches it is wrong by
// 10 % or more: under 100 rows per expert weight gradients of narrow layers, and a share of the
// experts that holds the large ones of a skewed load, whose rows are far more than expected.  (The constants before, a fit to 152 layers, are 1.23 % off
// on the same 26900, 10 % or more in 5 %; a layer's four launches together gain 2 to 7 % over them in one of twenty, lose 4 % in one of a hundred.)
// Some of them, 256 / 128 in us, gate_up, down, dgrad_h with dWd, dgrad_x with dWg and dWu:
//   256 tokens, d 128, f 256, 8 experts, 2 per token        11 / 9      10 / 8      16 / 11     13 / 10
//   248 tokens, d 320, f 320, 28 of 57 experts, 6           13 / 11     11 / 9      15 / 13     23 / 19
//   7380 tokens, d 512, f 1600, 19 of 39 experts, 2         44 / 58     42 / 34     77 / 57     97 / 89
//   2000 tokens, d 1024, f 512, 128 experts, 8              76 / 83     43 / 46     85 / 112   152 / 164
//   1500 tokens, d 2048, f 1024, 64 experts, 8             156 / 166    72 / 84    165 / 196   312 / 361
//   2048 tokens of the same layer                          163 / 204    91 / 110   222 / 245   350 / 422
//   8192 tokens of the same layer                          470 / 646   263 / 324   557 / 683   876 / 1214
struct ListCost { double tiles, each; };
// rows: routed rows to expect
template <int MODE, int S>
ListCost list_cost(const GemmArgs& a, double rows) {
  const double r = rows / a.E;
  if (is_wgrad(MODE)) {
    const double steps = r / BK + 0.5 > 1.0 ? r / BK + 0.5 : 1.0;
    return {static_cast<double>(a.E) * ceil_div(a.M, S) * ceil_div(a.N, S) * (a.A1 != nullptr ? 2 : 1),
            TileCost<S>::WGRAD + 1.1 * TileCost<S>::STEP * steps};
  }
  const double row_tiles = a.E * (r < 1.0 ? r : 1.0) * (r / S + TileCost<S>::RAGGED > 1.0 ? r / S + TileCost<S>::RAGGED : 1.0);
  return {row_tiles * ceil_div(a.N, MODE == GATE_UP ? S / 2 : S),
          TileCost<S>::FIXED + (is_dgrad_h(MODE) ? TileCost<S>::SWIGLU_BWD : 0.0) +
              TileCost<S>::STEP * (a.K / BK) * (MODE == DGRAD_X ? 2 : 1)};
}
template <int S> double places() { return static_cast<double>(Tile<S>::PER_CU) * compute_units(); }
template <int S> double launch_cost(const ListCost& l) {
  const double rounds = l.tiles / places<S>();
  const long long whole = static_cast<long long>(rounds + 0.95);      // a twentieth of a round too many does not count
  return 0.6 * (0.9 * rounds * l.each + l.each) + 0.4 * (whole < 1 ? 1 : whole) * l.each;
}
template <int S> double launch_cost(const ListCost& l, const ListCost& m) {
  return 0.65 * (l.tiles * l.each + m.tiles * m.each) / places<S>() + (l.each > m.each ? l.each : m.each);
}

// edge: null, or in: the edge to take (0: the rule's), out: the edge taken
bool take_small(int* edge, double small, double large) {
  const bool is_small = edge != nullptr && *edge != 0 ? *edge == 128 : small < large;
  if (edge != nullptr) *edge = is_small ? 128 : 256;
  return is_small;
}
template <int MODE>
int run_gemm(GemmArgs& a, int R_cap, long long rows, hipStream_t s, const char* name, int* edge) {
  const double r = static_cast<double>(rows);
  if (take_small(edge, launch_cost<128>(list_cost<MODE, 128>(a, r)), launch_cost<256>(list_cost<MODE, 256>(a, r)))) {
    const long long tiles = count_tiles<MODE, 128>(a, R_cap);
    return launch_gemm<MODE, 128>(a, tiles, s, name);
  }
  const long long tiles = count_tiles<MODE, 256>(a, R_cap);
  return launch_gemm<MODE, 256>(a, tiles, s, name);
}
template <int MODE_A, int MODE_B>
int run_gemm_pair(GemmArgs& a, GemmArgs& b, int R_cap, long long rows, hipStream_t s, const char* name, int* edge) {
  const double r = static_cast<double>(rows);
  if (take_small(edge, launch_cost<128>(list_cost<MODE_A, 128>(a, r), list_cost<MODE_B, 128>(b, r)),
                 launch_cost<256>(list_cost<MODE_A, 256>(a, r), list_cost<MODE_B, 256>(b, r)))) {
    const long long tiles = count_tiles<MODE_A, 128>(a, R_cap) + count_tiles<MODE_B, 128>(b, R_cap);
    return launch_gemm_pair<MODE_A, MODE_B, 128>(a, b, tiles, s, name);
  }
  const long long tiles = count_tiles<MODE_A, 256>(a, R_cap) + count_tiles<MODE_B, 256>(b, R_cap);
  return launch_gemm_pair<MODE_A, MODE_B, 256>(a, b, tiles, s, name);
}
bool bad_edges(const int* edges) {
  if (edges == nullptr) return false;
  for (int i = 0; i < 2; ++i) if (edges[i] != 0 && edges[i] != 128 && edges[i] != 256) return true;
  return false;
}


}  // namespace
