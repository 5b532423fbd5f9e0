// Rotary positions with several axes and the norms of queries and keys: what the C-ABI layer hands to the kernels, and the
// rules that choose a kernel's shape.  Plain C++ with no GPU dependency, so that the rules can be tested without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace aa {

constexpr int kRotaryAxes = 4, kRotaryPairs = 128;      // most axes, most pairs (256 channels)

// A token tensor [batch][heads][tokens][d] in memory: element strides, channels side by side.
struct TokenView {
  char* data;
  long long sb, sh, sn;
};

struct RotaryArgs {
  int batch, tokens, heads[2], d;      // heads of the queries and of the keys
  // pair j < pairs turns by turn[j] * (position along its axis) whole turns; axis a has the pairs from first[a] to first[a + 1]
  int pairs, axes, pairing, first[kRotaryAxes + 1];
  int grid[kRotaryAxes];       // of tokens, row-major; grid[0] == 0: `positions` [batch or 1][tokens][axes]
  const void* positions;
  int positions_float;
  long long positions_batch;      // elements from one sequence's positions to the next one's; 0: all share them
  float sign;                     // -1: the gradient's way, the transposed rotation
  TokenView in[2], grad[2], out[2];      // queries, keys; grad: gradients of the results (backward pass alone)
  const float* weight[2];      // of the norm, or null: ones
  int weight_heads;            // 1: a weight of its own for each head, 0: one [d] for all
  float eps, inv_d;
  float* partial;      // backward pass: sums of the weights' gradients, [slot][block][d]
  double turn[kRotaryPairs];
};

enum class RotaryMode { kRotate, kNorm, kNormBackward };
enum RotaryPairing { kAdjacent = 0, kHalves = 1, kAxisHalves = 2 };

// Channels a load takes at once: the most, up to 16 bytes, that divide the width, every stride and address, and the runs of
// channels that the pairing keeps together (adjacent pairs are inside a load, the others in two loads of equal width).
struct RotaryShape {
  int ve;        // channels of a load
  int lanes;     // lanes of a row, a power of two; each has `duos` pairs of loads
  int duos;
};
inline int rotary_duos(int ve) { return ve >= 4 ? 1 : ve == 2 ? 2 : 4; }
inline RotaryShape rotary_shape(int es, int d, int pairing, int axes, const int* first, unsigned long long misaligned_bytes) {
  // misaligned_bytes: all addresses and byte strides, or-ed
  for (int ve = 16 / es;; ve /= 2) {
    bool ok = d % ve == 0 && misaligned_bytes % (unsigned)(ve * es) == 0;
    if (axes > 0 && pairing == kHalves) ok = ok && first[axes] % ve == 0;
    if (axes > 0 && pairing == kAxisHalves)
      for (int a = 1; a <= axes; ++a) ok = ok && first[a] % ve == 0;
    if (!ok && ve > 1) continue;
    const int duos = rotary_duos(ve), count = (d + 2 * ve - 1) / (2 * ve);
    int lanes = 1;
    while (lanes * duos < count) lanes *= 2;
    return {ve, lanes, duos};
  }
}

// Heads a wave takes for its tokens (their angles are computed once): all, halved while the waves are fewer than four for each of
// the 1024 SIMDs.
inline int rotary_heads_per_wave(long long rows, int heads, int lanes) {
  const long long tiles = (rows * lanes + 63) / 64;
  int chunk = heads;
  while (chunk > 1 && tiles * ((heads + chunk - 1) / chunk) < 4096) chunk = (chunk + 1) / 2;
  return chunk;
}

// Backward pass: blocks that walk over the tokens (their sums of the weights' gradients are added up by a second kernel).
constexpr int kRotarySumBlocks = 1024;

}  // namespace aa
