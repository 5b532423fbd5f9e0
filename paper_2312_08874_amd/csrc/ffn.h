// The gated feed-forward block: what its launch sequence hands to the product kernels, and the rules that choose their tiles.
// Plain C++ with no GPU dependency, so that the rules can be tested without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace aa {

// Rows of the tensors that the block makes for itself (h, the gradients of gate and up, what the forward pass keeps) are a
// multiple of this many elements long, zeros behind the hidden width: a step of a product over them never leaves a row.
constexpr int kFfnPad = 64;
inline int ffn_pitch(int hidden) { return (hidden + kFfnPad - 1) / kFfnPad * kFfnPad; }

enum class FfnEpilogue {
  kStore,        // out[m][n] = sum (+ bias[n]), rounded to the element type; rows from row_part on go to out[1]
  kGate,         // n is hidden: h = act(gate) up, and what the backward pass needs of it
  kGateGrad,     // n is hidden: sum = dh; dgate = dh p, dup = dh q, side by side in out[0]
};

// One product D[m][n] = sum over k of A(m,k) B(n,k).  An operand lies k-contiguous ([m][k], leading dimension in elements) or
// m-contiguous ([k][m]); every row starts on 16 bytes.
struct FfnProduct {
  const void* a;
  const void* b[2];      // kGate: rows of gate and of up; b_parts == 2: k < k_part from b[0], the rest from b[1]
  long long lda, ldb;
  int M, N, K;           // of a k-contiguous operand: whole pieces of 16 bytes, zeros in what that adds
  int a_m, b_m;          // columns of an m-contiguous operand, whole pieces of 16 bytes
  int k_part, b_rows;    // b_parts == 2: a multiple of kFfnPad; rows of an m-contiguous B (of each part), zeros behind them
  int b_parts;
  int terms;             // kGateGrad: of 2, the second lie behind the first in a row; b_parts == 2: A's k runs through B once for each
  int b_twice;           // 1: two neighbouring values of k share a row of an m-contiguous B (A's rows are the two terms of each)
  int grid_m, grid_n;
  // epilogues
  void* out[2];
  long long ldo;
  int row_part;                 // kStore: first row of out[1] (and of its rows' count, `rows`); 0: one part
  int rows;
  int aligned;                  // 16-byte stores may be used
  const void* bias[2];          // kStore: [0]; kGate: gate, up
  int pitch;                    // of h, p, q, and (two of them) dgate | dup
  int hidden;                   // kGate, kGateGrad
  int activation;
  void* h;
  uint16_t *p_hi, *q_hi;        // d h / d gate and d h / d up, upper 16 and next 8 bits of fp32 (fp32 elements: all in p_hi)
  uint8_t *p_lo, *q_lo;
};

// which operands are m-contiguous: A and B k-contiguous, B alone m-contiguous, both
enum class FfnForm { kKK, kKM, kMM };

// A block's tile; `full` tiles are summed by one block each, the others by `parts` blocks of `each` steps.
struct FfnTile {
  int rows, cols, full, parts, each;
};
// One or two products of one form over the same k in one launch: tiles from `first` on are the second's.
struct FfnGroup {
  FfnProduct p[2];
  int first, tiles, full, parts, each;
  float* partial;      // [part][tile - full][rows][cols]
};

#ifdef __HIPCC__
#define AA_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define AA_HOST_DEVICE inline
#endif
// Tile `at` of a grid of tiles: eight rows of tiles down before the next column, so that neighbours share operands.
AA_HOST_DEVICE void ffn_place(unsigned at, unsigned grid_m, unsigned grid_n, int& tm, int& tn) {
  const unsigned group = 8u * grid_n, gi = at / group, rest = at - gi * group, left = grid_m - 8u * gi, high = left < 8u ? left : 8u;
  tm = (int)(8u * gi + rest % high);
  tn = (int)(rest / high);
}
// Block L of `count` (of the grid's rounded up to eights): each of the eight XCDs, to which blocks go in turn, takes a run of
// neighbours, so that its L2 serves what they share.  count or more: no work.
AA_HOST_DEVICE unsigned ffn_run(unsigned L, unsigned count) { return (L & 7u) * ((count + 7u) / 8u) + (L >> 3); }

// A launch of `blocks` blocks: this many along x at most, since it has to stay below 2^32 threads there (2^30 rows of 16 channels are
// 2^24 blocks of 256); further ones lie along y, and the last layer may have blocks without work.
constexpr unsigned kFfnLaunchBlocks = 1u << 22;
inline unsigned ffn_layers(long long blocks) { return (unsigned)((blocks + kFfnLaunchBlocks - 1) / kFfnLaunchBlocks); }

// A few tokens: x -> h (w: gate and up, K = width, N = hidden) and h -> y (w[0]: down, K = hidden, N = width).  Weights [N][K], dense.
constexpr int kFfnFewRows = 64;      // most tokens of their kernels
inline bool ffn_few_rows(int T, int C, int F) {
  // up to one tile of tokens; to four while the weights are small enough that the other kernels' latency counts (bf16, T tokens,
  // these and those: 512 x 1365, 64 tokens 18.9 and 21.7 us; 1024 x 2816, 32: 17.7, 20.2, 48: 24.8, 20.5; 2048 x 5504, 24: 33.8, 29.3)
  return T <= 16 || (T <= kFfnFewRows && (long long)T * C * F <= 100000000ll);
}
// Terms of dgate and dup (16-bit elements), as operands of dx, the weights' and the biases' gradients: of few tokens and in small blocks
// two, as of h in the forward pass of few tokens, since dx has too few values for the errors of rounded operands to even out.  The first
// term alone is no rounding: beyond the type's range it is the largest number, and only both are right or infinite.  dx in two terms
// costs nothing, its product waits for memory and launches; the weights' gradients pay for the steps (bf16, backward pass: 64 tokens of
// 2048 x 5504 80.8 us, 76.7 from the first term alone; 300 of 512 x 512 29.7, 26.9; 1000 of 256 x 384 36.2, 28.9).
inline int ffn_terms(int T, int C, int F, int es) { return es == 2 && (T <= kFfnFewRows || (long long)T * C * F <= 100000000ll) ? 2 : 1; }
struct FfnRows {
  const void *w[2], *x, *bias[2];
  long long ldx, ldy;
  int M, N, K, pitch, activation;      // pitch: of h and of what is kept
  void *h, *kept_h, *y;                // h: two terms of 16 bits, [2][M][pitch], or fp32; kept_h, p and q for the backward pass, where p_hi is set
  uint16_t *p_hi, *q_hi;
  uint8_t *p_lo, *q_lo;
};
// Waves of a block, which share out the steps of 64 bytes.
inline int ffn_rows_waves(int steps) { return steps >= 16 ? 8 : 4; }

// The block as its caller describes it; rows of `ld` elements where they may be apart.
struct FfnBlock {
  int T, C, F, dtype, activation;      // tokens, width, hidden width
  const void *x, *w_gate, *b_gate, *w_up, *b_up, *w_down, *b_down;
  long long ldx, ldy, lddx;
  void* y;
  const void* dy;
  void *dx, *dw_gate, *db_gate, *dw_up, *db_up, *dw_down, *db_down;
  int es() const { return dtype == 0 ? 4 : 2; }
  int unit() const { return 16 / es(); }      // elements of 16 bytes
};

// Tile of one or two products (second: M2 x N2, or 0) over `steps` steps of 128 bytes, and how the tiles that are left after whole
// rounds of the compute units are shared out along k (`split`: whether they may be): the least estimated time.
//
// Microseconds, measured over 4 to 36 steps (16-bit elements, k-contiguous operands; m-contiguous ones within 8 %): a step of as
// many blocks as a compute unit holds, of one alone, and what a block costs beside its steps.  fp32 steps are those of its matrix
// rate.  narrow: 64 x 96 tiles may be taken (fp32, results stored as they are), which leave nothing of the widths of three times a
// power of two unused: 10664 tokens, 288 x 768, the three products 338 us without them, 297 with; training steps of 2100 tokens,
// 288 x 768, 133 and 129 us; 2100, 576 x 1536, 343 and 349; 700, 1024 x 2730, 359 and 350.
inline FfnTile ffn_tile(long long M, long long N, long long M2, long long N2, long long steps, int es, bool split, bool gated, int compute_units,
                        bool narrow = false) {
  struct Shape {
    int rows, cols, held;
    double step, alone, fixed, fixed_alone;
  };
  static const Shape half[4] = {{256, 256, 1, 1.38, 1.38, 9.0, 9.0}, {256, 128, 1, 0.78, 0.78, 5.0, 5.0}, {128, 128, 2, 0.84, 0.56, 6.0, 3.5}, {64, 64, 4, 0.74, 0.35, 3.5, 1.5}};
  static const Shape single[3] = {{128, 128, 2, 3.75, 2.05, 8.0, 5.0}, {64, 64, 4, 2.0, 0.62, 4.5, 2.0}, {64, 96, 3, 2.2, 0.85, 4.5, 2.0}};
  FfnTile best{64, 64, 1, 1, (int)steps};
  double least = 1e30;
  for (int i = 0; i < (es == 4 ? (narrow ? 3 : 2) : 4); ++i) {
    const Shape& s = es == 4 ? single[i] : half[i];
    const long long cols = gated ? s.cols / 2 : s.cols;
    const long long tiles = (M + s.rows - 1) / s.rows * ((N + cols - 1) / cols) + (M2 + s.rows - 1) / s.rows * ((N2 + cols - 1) / cols);
    const long long room = (long long)compute_units * s.held;
    // of `blocks` blocks of `each` steps, dealt out evenly
    auto time = [&](long long blocks, long long each) {
      const long long per = (blocks + compute_units - 1) / compute_units, whole = per / s.held, rest = per % s.held;
      const double share = s.held > 1 ? (double)(rest - 1) / (s.held - 1) : 0.0;
      double t = whole * (each * s.step + s.fixed);
      if (rest > 0) t += each * (s.alone + share * (s.step - s.alone)) + s.fixed_alone + share * (s.fixed - s.fixed_alone);
      return t;
    };
    auto consider = [&](long long full, int parts, long long each) {
      double t = time(full, steps);
      if (parts > 1)      // their sums are written, read and added up by one more launch
        t += time((tiles - full) * parts, each) + 4.0 + 8.0e-6 * (tiles - full) * parts * s.rows * s.cols / 4.5;
      if (t < least) least = t, best = FfnTile{s.rows, s.cols, (int)full, parts, (int)each};
    };
    consider(tiles, 1, steps);
    if (!split) continue;
    const long long full = tiles / room * room, tail = tiles - full;      // whole rounds, and what is left
    if (tail == 0) continue;
    int before = 1;
    for (int rounds = 1; rounds <= 3; ++rounds) {      // as many parts as fill one, two or three rounds
      const int most = (int)std::min<long long>(std::min(64ll, steps / 2), room * rounds / tail);
      if (most <= before) continue;
      const long long each = (steps + most - 1) / most;
      const int parts = (int)((steps + each - 1) / each);      // every part has steps of its own
      if (parts > before) consider(full, parts, each), before = parts;
    }
  }
  return best;
}

}  // namespace aa
