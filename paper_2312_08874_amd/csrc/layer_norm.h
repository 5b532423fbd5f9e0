// Layer norm: what the C-ABI layer hands to the kernels, and the rule that shares a row out among lanes.  Plain C++ but for
// float2, so that the rule can be tested without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace aa {

constexpr int kNormWidth = 32768;      // most channels of a row

struct NormRows {      // rows of a tensor: stride in elements
  char* data;
  long long stride;
};

struct NormArgs {
  NormRows x, r, y, sum;              // r: none, where what is normed is x
  NormRows dy, dsum, dx;              // backward
  const void *w, *b;                  // in fp32 or the element type
  int wide_weights;                   // 1: fp32
  float2* stats;                      // [rows]: mean, 1 / deviation
  int rows, width;
  float eps, inv;                     // inv = 1 / width
  float* partial;                     // backward: [block][2][width], sums of dy h and of dy
  int blocks;
};

// A lane takes 16 bytes at a time, `pieces` times, `lanes` of them a row (a power of two up to a wave, or a whole block of 256 or 1024).
struct NormShape {
  int lanes, pieces, threads;
  int rows_at_once() const { return lanes >= threads ? 1 : threads / lanes; }
};
// At most 32 channels a lane forward and, where rows are no longer than a block of 1024 takes so, 16 backward, whose lanes also hold the next
// row and the sums of the weights' gradients.  Backward, blocks of 1024 have 128 registers a lane, which is too few above 8192 channels: up to 16384
// 64 to 146 are spilled in 16 bits and up to 203 in fp32, above that 528 to 711 and up to 1022.  A step of 4096 rows in bf16, both ways with the
// residual, takes 166 us of 8192 channels, 384 of 16384 and 1677 of 32768, where a large copy's rate gives 98, 196 and 392; in fp32 258, 1004 and 3418
// (196, 392 and 785).
inline NormShape norm_shape(int es, int width, bool backward) {
  const int per = 16 / es, count = (width + per - 1) / per, most = (backward && width <= 16384 ? 16 : 32) / per;
  NormShape s{64, 1, 256};
  if (count > 256 * most) s.lanes = s.threads = 1024;
  else if (count > 64 * most) s.lanes = 256;
  else
    while (s.lanes > 1 && s.lanes / 2 * 2 >= count) s.lanes /= 2;      // two pieces a lane where rows are short
  while (s.lanes * s.pieces < count) s.pieces *= 2;
  return s;
}

// What norm_shape comes to, and so what the kernels are compiled for: rows shared by blocks of `threads`, or (block false) by up to a wave.
constexpr bool norm_takes(int es, int threads, bool block, int pieces, bool backward) {
  const int most = (backward ? 16 : 32) * es / 16;
  if (!block) return pieces <= most;
  return pieces >= most / 2 && pieces <= (backward && threads == 1024 ? 2 * most : most);
}

// Blocks of the backward pass, each of which leaves a part of the weights' gradients, two for each compute unit: training steps with the residual
// of 65536 x 2048 in fp16 take 478 us (256 blocks: 573, 768: 493), in fp32 930 (946, 967), of 16384 x 512 in bf16 37 (any of these).
constexpr int kNormBlocks = 512;
inline int norm_blocks(const NormShape& s, int rows, bool backward) {
  const long long needed = ((long long)rows + s.rows_at_once() - 1) / s.rows_at_once();
  return (int)std::min<long long>(needed, backward ? kNormBlocks : 2048);
}

}  // namespace aa
