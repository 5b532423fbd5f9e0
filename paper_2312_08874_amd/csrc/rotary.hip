// Launches of the rotary kernels, and the sum of the norm weights' gradients over their blocks.
#include "kernels.h"

namespace aa {

namespace {

// dst[c] = sum over the blocks of partial[block][c], in a fixed order: a block takes 16 channels, 64 threads each, which ask for
// eight values at a time.
__global__ __launch_bounds__(1024) void rotary_sum_kernel(const float* partial, size_t slot_floats, int blocks_q, int blocks_k, int d,
                                                          int slots_q, float* dw_q, float* dw_k) {
  __shared__ float sums[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4, slot = blockIdx.y;
  const bool query = slot < slots_q;
  float* dst = query ? dw_q : dw_k;
  if (dst == nullptr) return;
  const int blocks = query ? blocks_q : blocks_k;
  const float* from = partial + slot * slot_floats + min(c, d - 1);
  float v[8] = {};
  for (int i = part; i < blocks; i += 64 * 8)
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float x = from[(size_t)min(i + 64 * u, blocks - 1) * d];
      v[u] += i + 64 * u < blocks ? x : 0.0f;
    }
  sums[part][threadIdx.x & 15] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  __syncthreads();
  if (threadIdx.x >= 16 || c >= d) return;
#pragma unroll
  for (int u = 0; u < 4; ++u) v[u] = 0.0f;
#pragma unroll
  for (int i = 0; i < 64; ++i) v[i & 3] += sums[i][threadIdx.x];
  dst[(size_t)(query ? slot : slot - slots_q) * d + c] = (v[0] + v[1]) + (v[2] + v[3]);
}

}  // namespace

size_t rotary_partial_floats(const RotaryArgs& a) {
  // the most blocks that any shape of these tensors gives: those of chunks y side by side, or one slot per head
  return a.weight_heads ? (size_t)(a.heads[0] + a.heads[1]) * kRotarySumBlocks * a.d
                        : (size_t)2 * std::max(kRotarySumBlocks, a.heads[0] + a.heads[1]) * a.d;
}

hipError_t launch_rotary(int dtype, RotaryArgs& a, const RotaryShape& s, RotaryMode mode, float* dw_q, float* dw_k, hipStream_t st) {
  a.inv_d = 1.0f / (float)a.d;
  const bool back = mode == RotaryMode::kNormBackward, sums = back && (dw_q != nullptr || dw_k != nullptr);
  if (!sums) a.partial = nullptr;
  const RotaryPlan p = rotary_plan(s, (long long)a.batch * a.tokens, a.heads[0], a.heads[1], back, a.weight_heads);
  const hipError_t err = dtype == 0 ? launch_rotary_f32(a, s.ve, p, mode, st)
                                    : dtype == 1 ? launch_rotary_f16(a, s.ve, p, mode, st) : launch_rotary_bf16(a, s.ve, p, mode, st);
  if (err != hipSuccess || !sums) return err;
  const int own = a.weight_heads != 0, slots = own ? a.heads[0] + a.heads[1] : 2;
  const int each[2] = {p.blocks * (own ? 1 : p.chunks[0]), p.blocks * (own ? 1 : p.chunks[1])};
  rotary_sum_kernel<<<dim3((unsigned)((a.d + 15) / 16), (unsigned)slots), dim3(1024), 0, st>>>(
      a.partial, (size_t)std::max(each[0], each[1]) * a.d, each[0], each[1], a.d, own ? a.heads[0] : 1, dw_q, dw_k);
  return hipGetLastError();
}

}  // namespace aa
