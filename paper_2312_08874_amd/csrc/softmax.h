// Softmax attention: what the C-ABI layer hands to the kernels, and the rules that choose among them.  Plain C++ with no GPU
// dependency, so that the rules can be tested without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "rotary.h"      // TokenView

namespace aa {

constexpr int kSoftmaxWidth = 256;      // most channels of a head
// What rounding took from out is kept for queries that see up to so many keys: without it the error of D shows in dq and dk of 16-bit
// types, which are off by 1.4 roundings with it, and by 2.2 for 2 keys, 1.6 for 64, 1.45 for 512 without.
constexpr int kLowKeys = 512;
constexpr int kPeakBlocks = 512;      // most blocks that look for fp16's peaks

struct SoftmaxArgs {
  TokenView q, k, v, out, dout, dq, dk, dv;
  TokenView dout_whole;      // fp32, whose q, k, v and dout are taken apart into terms
  unsigned term;             // bytes from a row's one term to the next
  // what the forward pass keeps, null: nothing: lse (natural logarithm) [batch][heads_q][tokens_q] and, of 16-bit types, what
  // rounding took from out, [..][d], itself in the type
  float* lse;
  char* low;
  const int *starts_q, *starts_k;        // packed: [sequences + 1], batch 1
  const int *lengths_q, *lengths_k;      // padded: [batch], or null: every row
  int batch, heads_q, heads_k, tokens_q, tokens_k, d, sequences;      // sequences 0: not packed
  int causal;
  int waves;            // of a block: 2, 4 or 8, each of which has 32 rows
  int shared;           // softmax_shared
  int two;              // backward: softmax_two_roundings
  int wide;             // whole 16-byte pieces wherever a result is stored
  float scale, c;       // c = scale log2 e
  // columns kernel: query heads side by side in a tile, tokens of a tile, ranges of keys and where each leaves its part
  int pack, tile_tokens, splits;
  float *part, *part_stats;      // [split][batch, head, token][d]; [..][3]: reference, sum, what rounding took from it
  // backward pass: what the queries' kernel leaves for the keys' of every query, [2][batch][heads_q][tokens_q], and fp16's peaks
  float* stats;
  float* peaks;         // [2][kPeakBlocks]: of each of peak_blocks blocks, the largest squared length of a row of dout, and of v
  int peak_blocks;      // a multiple of eight
  // parts of dq, or of dk and dv: [split][batch, head, token][d]
  float *part_a, *part_b;
  int first_batch;      // of a launch that sums them
};

// Width that the kernels are compiled for: channels of the scores' products, in steps of 16; results are taken in tiles of 32.
inline int softmax_width(int d) {
  for (const int w : {32, 48, 64, 80, 96, 128})
    if (d <= w) return w;
  return 256;
}
constexpr int softmax_tiles_across(int dp) { return (dp + 31) / 32; }

// Tiles of `rows` tokens along the queries (or keys) of all sequences together; sequence s of a packed run has the tiles from
// starts[s] / rows + s on, which leaves each at least the tiles it needs, whatever the lengths on the device are.
inline long long softmax_tiles(int tokens, int batch, int sequences, int rows) {
  return sequences > 0 ? (long long)tokens / rows + sequences : (long long)batch * (((long long)tokens + rows - 1) / rows);
}

// A tile of keys (or of queries, for the keys' kernel) on its way through LDS, and the tokens that a block's waves take side by side.
// dp: width that the kernels are compiled for
constexpr int softmax_step(int es, int dp) { return es == 4 && dp > 32 ? 32 : 64; }
// Terms that an operand is taken apart into by all kernels but that of few queries, which reads keys and values once and is bound by that:
// three bf16 terms for fp32, up to where two tiles of them fit in LDS.
constexpr int softmax_terms(int es, int dp) { return es == 4 && dp <= 128 ? 3 : 1; }
// Waves of a columns block: as many as 160 KB of LDS hold two tiles of 32 keys of.
constexpr int softmax_column_waves(int es, int dp) { return es * dp <= 256 ? 4 : es * dp <= 512 ? 2 : 1; }

constexpr int kSoftmaxUnits = 256;      // compute units

// Whether blocks are of 64 rows and two waves share every 32 of them, each with half of every tile of 64 keys (or queries): where there are so
// few blocks that the length of the longest is the time, and not so long ones that ranges are worth their parts.  `blocks`: of 64 rows,
// `across`: what each goes over.  Measured, training steps, shared and not: 1500 tokens, 2 x 8 heads of 64, causal, 63 us and 88; 2 x 2000,
// 8 heads of 80 120 and 140; 4096, 8 heads of 64 187 and 214; but 8192 packed tokens, 8 heads, 1184 blocks, 108 and 100, 2 x 1900, 16 heads of
// 128, 960 blocks, 427 and 355, and 2 x 4096, 16 heads on 4 of 128, whose keys 16384 rows see, 919 and 648.
inline bool softmax_shared(int es, long long blocks, long long across) { return es == 2 && blocks < 3 * kSoftmaxUnits && across < 8192; }

// Waves of a block of rows, 32 rows each: as few rounds of blocks over the compute units as may be, two waves where four would be half
// empty, eight, which share every tile of keys, where they cost no round.  Measured: windows of 49 tokens, 2048 x 12 heads, 79 us with two
// and 96 with four; 37 packed images of 8192 tokens in all, a training step, 101 and 110; 128 x 128 tokens, 2359 with eight (forward and
// for dq), 2432 with four, 2912 with two.  Terms take three times the LDS: two waves then cost more.
constexpr int softmax_most_waves(int es, int d) { return es == 2 && d > 32 && d <= 128 ? 8 : 4; }
inline int softmax_waves(int es, int tokens, int batch, int sequences, int heads, long long across, int most, int terms) {
  auto rounds = [&](int waves) {
    const long long blocks = softmax_tiles(tokens, batch, sequences, 32 * waves) * heads;
    return (blocks + kSoftmaxUnits - 1) / kSoftmaxUnits * waves;
  };
  if (softmax_shared(es, softmax_tiles(tokens, batch, sequences, 64) * heads, across)) return 2;
  const int waves = rounds(2) * (terms > 1 ? 3 : 2) < rounds(4) * 2 ? 2 : 4;
  return most >= 8 && rounds(8) <= rounds(waves) ? 8 : waves;
}

struct SoftmaxPlan {
  int waves;
  bool columns, shared;
  int pack, tile_tokens, splits;
  long long tiles;      // of queries
};
// Ranges that make up for blocks that are too few, each of `least` keys at the least.
inline int softmax_splits(long long blocks, long long wanted, long long keys, int least) {
  const long long most = std::max(1ll, keys / least);
  return (int)std::min(std::min(most, 128ll), std::max(1ll, (wanted + blocks - 1) / std::max(1ll, blocks)));
}
// keys (or queries) of a sequence, as far as the host knows
inline long long softmax_typical(int tokens, int sequences) {
  return sequences > 1 ? std::min<long long>(tokens, 2ll * tokens / sequences + 1) : tokens;
}
inline SoftmaxPlan softmax_plan(const SoftmaxArgs& a, int es) {
  SoftmaxPlan p{};
  const int group = a.heads_q / a.heads_k, outer = a.sequences > 0 ? 1 : a.batch;
  const long long queries = softmax_typical(a.tokens_q, a.sequences), keys = softmax_typical(a.tokens_k, a.sequences);
  p.waves = softmax_waves(es, a.tokens_q, a.batch, a.sequences, a.heads_q, keys, softmax_most_waves(es, a.d), softmax_terms(es, softmax_width(a.d)));
  const long long row_blocks = softmax_tiles(a.tokens_q, a.batch, a.sequences, 128) * a.heads_q;
  p.columns = queries <= 16 || (row_blocks < kSoftmaxUnits && keys >= (es == 4 ? 512 : 1536));
  p.pack = 1, p.tile_tokens = 32 * p.waves, p.splits = 1;
  if (p.columns) {
    // heads that share keys side by side, where the tokens leave room
    if (queries * 2 <= 32)
      for (int n = 2; n <= group && n <= 32; ++n)
        if (group % n == 0 && (queries * n <= 32 || n <= 4)) p.pack = n;
    p.tile_tokens = 32 / p.pack;
  }
  p.shared = !p.columns && p.waves == 2 && softmax_shared(es, softmax_tiles(a.tokens_q, a.batch, a.sequences, 64) * a.heads_q, keys);
  p.tiles = softmax_tiles(a.tokens_q, outer, a.sequences, p.tile_tokens);
  if (a.sequences == 0) p.tiles /= outer;
  if (p.columns) {
    const long long blocks = p.tiles * outer * a.heads_q / p.pack;
    // two blocks a compute unit: 8 sequences of up to 65536 keys, 4 heads of 128 in fp16, 133 us; with one 130, with four 145, eight 166
    // and ranges of 512 keys at the least; for single tokens of 256 up to some thousand keys and in fp32, whose tiles take long: four tokens over
    // 2000 keys of 8 heads of 64, 12.7 us and 14.1 with 512, fp32 19.3 and 24.9, but one token over 20000 keys of 2 heads of 128 19.5 and 17.3,
    // 64 tokens over 2 x 4096 of 8 heads 28.8 and 21.4
    const int least = queries <= 16 && (es == 4 || keys <= 8192) ? 256 : 512;
    p.splits = softmax_splits(blocks, 2 * kSoftmaxUnits, keys, least);
  }
  return p;
}
// Whether the backward pass of 16-bit types takes P and dS as two roundings, the value's and what that left: of one, gradients are off by
// 1.41 roundings of their own, and by up to 1.56 where a head is so narrow that sums over the keys come out much smaller than their
// terms; where they are few values, by chance more.  Up to 32 channels two cost nothing (2048 tokens, 4 x 8 heads of 16: 140 us, 140 with
// one); in small calls of others some 3 us (256 tokens, 4 x 8 heads of 128: 46.3, 41.9 with one), of 8192 packed tokens of 8 heads of 64
// 114 instead of 99.
constexpr int kTwoWidth = 32;
inline bool softmax_two_roundings(const SoftmaxArgs& a, int es) {
  const double scores = (double)a.batch * a.heads_q * a.tokens_q * (double)softmax_typical(a.tokens_k, a.sequences);
  return es == 2 && (a.d <= kTwoWidth || scores * a.d <= 1e8);
}
// The backward pass: ranges of keys for the queries' kernel, of queries (all heads that share the keys) for the keys'.
struct SoftmaxBackPlan {
  int waves, splits;
  bool shared;
  long long tiles;      // of one sequence, or of the packed run
};
inline SoftmaxBackPlan softmax_back_plan(const SoftmaxArgs& a, int es, bool keys) {
  const int tokens = keys ? a.tokens_k : a.tokens_q, heads = keys ? a.heads_k : a.heads_q;
  SoftmaxBackPlan p;
  const long long across = keys ? softmax_typical(a.tokens_q, a.sequences) * (a.heads_q / a.heads_k) : softmax_typical(a.tokens_k, a.sequences);
  p.waves = softmax_waves(es, tokens, a.batch, a.sequences, heads, across, keys ? 4 : softmax_most_waves(es, a.d), softmax_terms(es, softmax_width(a.d)));
  if (a.d > kTwoWidth && softmax_two_roundings(a, es)) p.waves = 2;      // so that not every kernel is there twice
  p.tiles = softmax_tiles(tokens, 1, a.sequences, 32 * p.waves);
  // Blocks for each compute unit that ranges are to make up for.  Uneven ones (causal) are shared out better where there are more, which
  // costs their parts' way through memory: the keys' kernel of 2 x 4096 tokens, 16 heads on 4 of 128, and its sum take 383 us with two
  // ranges, 315 with three, 328 with four; of 2 x 2000 tokens, 8 heads of 80, a step takes 229 with two and 247 with three.
  const int each = keys ? (a.causal && across >= 8192 ? 3 : 2) : a.causal ? 2 : 1;
  // and each range of 512 at the least, in fp32, whose tiles take long, 128: 1000 tokens, 6 heads of 48, 159 us with 512, 113 with 256, 102 so;
  // 2048 tokens, 8 heads of 64 in bf16 104 with 512, 128 with 256 and twice the blocks
  const long long blocks = p.tiles * (a.sequences > 0 ? 1 : a.batch) * heads;
  p.shared = p.waves == 2 && softmax_shared(es, blocks, across);
  p.splits = softmax_splits(blocks, each * kSoftmaxUnits / (p.shared ? 2 : 1), across, es == 4 ? 128 : 512);
  return p;
}

// Launches of one element type (softmax_{bf16,f16,f32}.hip, and softmax_bwd_*).
enum class SoftmaxPass { kRows, kColumns, kJoin, kPeaks, kQueries, kKeys, kSumQueries, kSumKeys };

}  // namespace aa
