// Launches of the rotary kernels, and the sum of the norm weights' gradients over their blocks.
#include "kernels.h"

namespace aa {

namespace {

// dst[c] = sum over the blocks of partial[block][c], in a fixed order: a block takes 16 channels, 64 threads each.
__global__ __launch_bounds__(1024) void rotary_sum_kernel(const float* partial, int blocks, int d, int slots_q, float* dw_q, float* dw_k) {
  __shared__ float sums[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4, slot = blockIdx.y;
  float* dst = slot < slots_q ? dw_q : dw_k;
  if (dst == nullptr) return;
  float v = 0.0f;
  if (c < d)
    for (int i = part; i < blocks; i += 64) v += partial[((size_t)slot * blocks + i) * d + c];
  sums[part][threadIdx.x & 15] = v;
  __syncthreads();
  if (threadIdx.x >= 16 || c >= d) return;
  v = 0.0f;
  for (int i = 0; i < 64; ++i) v += sums[i][threadIdx.x];
  dst[(size_t)(slot < slots_q ? slot : slot - slots_q) * d + c] = v;
}

int chunk_of(const RotaryArgs& a, const RotaryShape& s, RotaryMode mode) {
  if (mode == RotaryMode::kNormBackward && a.weight_heads) return 1;
  return rotary_heads_per_wave((long long)a.batch * a.tokens, a.heads[0] + a.heads[1], s.lanes);
}
int blocks_of(const RotaryArgs& a, const RotaryShape& s, RotaryMode mode, int chunk) {
  const long long per = 4 * (64 / s.lanes), tiles = ((long long)a.batch * a.tokens + per - 1) / per;
  if (mode != RotaryMode::kNormBackward) return (int)tiles;
  const int chunks = (a.heads[0] + a.heads[1] + chunk - 1) / chunk;
  return (int)std::min<long long>(tiles, std::max(1, kRotarySumBlocks / chunks));
}

}  // namespace

size_t rotary_partial_floats(const RotaryArgs& a) {
  // the most blocks that any shape of these tensors gives: those of chunks y side by side, or one slot per head
  return a.weight_heads ? (size_t)(a.heads[0] + a.heads[1]) * kRotarySumBlocks * a.d
                        : (size_t)2 * std::max(kRotarySumBlocks, a.heads[0] + a.heads[1]) * a.d;
}

hipError_t launch_rotary(int dtype, RotaryArgs& a, const RotaryShape& s, RotaryMode mode, float* dw_q, float* dw_k, hipStream_t st) {
  a.inv_d = 1.0f / (float)a.d;
  const int chunk = chunk_of(a, s, mode), blocks = blocks_of(a, s, mode, chunk);
  const bool sums = mode == RotaryMode::kNormBackward && (dw_q != nullptr || dw_k != nullptr);
  if (!sums) a.partial = nullptr;
  const hipError_t err = dtype == 0 ? launch_rotary_f32(a, s, mode, chunk, blocks, st)
                                    : dtype == 1 ? launch_rotary_f16(a, s, mode, chunk, blocks, st) : launch_rotary_bf16(a, s, mode, chunk, blocks, st);
  if (err != hipSuccess || !sums) return err;
  const int heads = a.heads[0] + a.heads[1], slots = a.weight_heads ? heads : 2;
  const int each = a.weight_heads ? blocks : blocks * ((heads + chunk - 1) / chunk);
  rotary_sum_kernel<<<dim3((unsigned)((a.d + 15) / 16), (unsigned)slots), dim3(1024), 0, st>>>(
      a.partial, each, a.d, a.weight_heads ? a.heads[0] : 1, dw_q, dw_k);
  return hipGetLastError();
}

}  // namespace aa
