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
  int lanes;     // lanes of a row, a power of two
  int duos;      // pairs of loads of a lane
};
constexpr int rotary_duos(int ve) { return ve >= 4 ? 1 : ve == 2 ? 2 : 4; }
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

// How a launch shares out its rows.  A block of four waves takes the tokens of 4 / across waves (64 / lanes tokens each), and
// `across` of its waves take `chunk` heads each, side by side: the angles of a token, which cost as much as two heads or three,
// are computed once a block.
struct RotaryPlan {
  int lanes, shift;      // lanes of a row, and their logarithm
  int across, chunk;
  int chunks[2];         // blocks along y: those of the queries, then those of the keys; forward: [0] has the heads of both
  int tiles, blocks;     // tiles of tokens, blocks along x
};

// Forward: blocks along x at most, since a launch has to stay below 2^32 threads there (2^26 tokens of 256 channels are 2^24 blocks of
// 256); more tiles lie along z, this many a layer.  (As launches of their own, which hand the kernel a first tile: 4096 x 2 tokens
// 8.0 us and not 7.8.)
constexpr int kRotaryLaunchBlocks = 1 << 23;
inline int rotary_layers(const RotaryPlan& p) { return (p.blocks - 1) / kRotaryLaunchBlocks + 1; }

// Backward pass: blocks walk over the tiles and leave sums of the weights' gradients, which a second kernel adds up; at most this
// many for one weight.
constexpr int kRotarySumBlocks = 1024;
// Waves that a launch is cut into where it can be, two for each of the 1024 SIMDs: with four the norm of 12544 tokens of 6 heads
// takes 10.0 us and not 8.5, with one it is the same.
constexpr long long kRotaryWaves = 2048;

// Forward: four waves along the heads (two: long clips 115 us and not 110).  Backward, whose waves hold fewer rows: two, and as
// many tiles a block as leave two blocks to a CU, up to four, since a block's sums cost as much as a tile (16384 tokens, 8
// heads each of 64 channels: 25.5 us; a tile each: 27.3, four waves along the heads: 30.4; 12544 tokens, 3 heads: 17.1, 19.3, 22.7).
inline RotaryPlan rotary_plan(const RotaryShape& s, long long rows, int heads_q, int heads_k, bool backward, bool one_head) {
  // one_head (backward): a wave takes one head, whose weights and sums are its own
  RotaryPlan p{};
  p.lanes = s.lanes;
  while (1 << p.shift < s.lanes) ++p.shift;
  const int most = backward ? std::max(heads_q, heads_k) : heads_q + heads_k;
  p.across = backward ? std::min(most, 2) : most >= 3 ? 4 : most;
  const long long per = (4 / p.across) * (64 / s.lanes);
  p.tiles = (int)((rows + per - 1) / per);
  auto count = [&](int chunk, int heads) { return (heads + p.across * chunk - 1) / (p.across * chunk); };
  auto blocks = [&](int chunk) { return backward ? count(chunk, heads_q) + count(chunk, heads_k) : count(chunk, most); };
  p.chunk = backward && one_head ? 1 : (most + p.across - 1) / p.across;
  while (p.chunk > 1 && 4 * (long long)p.tiles * blocks(p.chunk) < kRotaryWaves) p.chunk = (p.chunk + 1) / 2;
  p.chunks[0] = count(p.chunk, backward ? heads_q : most), p.chunks[1] = backward ? count(p.chunk, heads_k) : 0;
  p.blocks = p.tiles;
  if (backward) {
    const long long each = std::min(4ll, std::max(1ll, ((long long)p.tiles * blocks(p.chunk) + 256) / 512));
    const int most_blocks = std::max(1, kRotarySumBlocks / (one_head ? 1 : std::max(p.chunks[0], p.chunks[1])));
    p.blocks = (int)std::min<long long>((p.tiles + each - 1) / each, most_blocks);
  }
  return p;
}

}  // namespace aa
