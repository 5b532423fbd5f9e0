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
  kPartial,      // partial[split][m][n] = sum over the split's part of k, fp32
  kGate,         // n is hidden: h = act(gate) up, and what the backward pass needs of it
  kGateGrad,     // n is hidden: sum = dh; dgate = dh p, dup = dh q
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
  int splits, split_steps;      // k is cut into `splits` of split_steps steps
  int grid_m, grid_n;
  // epilogues
  void* out[2];
  long long ldo;
  int row_part;                 // kStore: first row of out[1] (and of its rows' count, `rows`); 0: one part
  int rows;
  int aligned;                  // 16-byte stores may be used
  const void* bias[2];          // kStore: [0]; kGate: gate, up
  float* partial;
  int pitch;                    // of h, p, q, dgate | dup (two of them) and of a row of `partial`
  int hidden;                   // kGate, kGateGrad
  int activation;
  void* h;
  uint16_t *p_hi, *q_hi;        // d h / d gate and d h / d up, upper 16 and next 8 bits of fp32 (fp32 elements: all in p_hi)
  uint8_t *p_lo, *q_lo;
};

// A few tokens: x -> h (w: gate and up, K = width, N = hidden) and h -> y (w[0]: down, K = hidden, N = width).  Weights [N][K], dense.
constexpr int kFfnFewRows = 64;
struct FfnRows {
  const void *w[2], *x, *bias[2];
  long long ldx, ldy;
  int M, N, K, pitch, activation;      // pitch: of h and of what is kept
  void *h, *kept_h, *y;                // h: 16 bits (up to four tokens: two terms, [2][M][pitch]) or fp32; kept_h, p and q for the backward pass, where p_hi is set
  uint16_t *p_hi, *q_hi;
  uint8_t *p_lo, *q_lo;
};
// Waves of a block, which share out the steps of 64 bytes.
inline int ffn_rows_waves(int steps) { return steps >= 16 ? 8 : 4; }

// which operands are m-contiguous: A and B k-contiguous, B alone m-contiguous, both
enum class FfnForm { kKK, kKM, kMM };

struct FfnTile {
  int rows, cols, splits;      // of a block; parts that k is cut into
};

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

// Tile and parts of k of a product of M x N results over `steps` steps of 128 bytes: the least estimated time.  A compute unit
// holds one block of 256 x 256, two of 128 x 128, four of 64 x 64 (which alone has work for few rows).
inline FfnTile ffn_tile(long long M, long long N, int steps, int es, bool can_split, bool gated, int compute_units) {
  struct Shape {
    int size, held;
    double step, least, fixed;      // microseconds: of a step with a full compute unit, of one block alone, of a block's start and end
  };
  static const Shape shapes[3] = {{256, 1, 2.2, 2.2, 5.0}, {128, 2, 1.5, 0.9, 3.0}, {64, 4, 1.3, 0.7, 2.0}};
  FfnTile best{64, 64, 1};
  double least = 1e30;
  for (const Shape& s : shapes) {
    if (s.size == 256 && es == 4) continue;
    const long long cols = gated ? s.size / 2 : s.size, blocks = ((M + s.size - 1) / s.size) * ((N + cols - 1) / cols);
    for (int splits = 1; splits <= 64; splits *= 2) {
      if (splits > 1 && (!can_split || steps / splits < 4)) break;
      const int each = (steps + splits - 1) / splits, parts = (steps + each - 1) / each;
      const long long total = blocks * parts, room = (long long)compute_units * s.held, rounds = (total + room - 1) / room;
      const long long on_one = std::min<long long>((total + compute_units - 1) / compute_units, s.held);
      const double slow = es == 4 ? 8.0 : 1.0, step = std::max(s.least, s.step * slow * on_one / s.held);
      double t = rounds * (each * step + s.fixed);
      if (parts > 1) t += 4.0 + 8e-6 * parts * M * N / 4.0;      // written and read again, 4 TB/s
      if (t < least) least = t, best = FfnTile{s.size, s.size, parts};
    }
  }
  return best;
}

}  // namespace aa
