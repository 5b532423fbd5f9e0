// Softmax attention: launch sequences, and copies of tensors whose rows are no whole 16-byte pieces.
#include "common.h"
#include "kernels.h"

namespace aa {

namespace {

constexpr size_t kAlign = 256;
size_t aligned(size_t bytes) { return (bytes + kAlign - 1) / kAlign * kAlign; }

struct Tensor {
  TokenView* view;
  int heads, tokens;
};

// rows of d elements to dense rows of `width`, with zeros behind them
template <class T>
__global__ __launch_bounds__(256) void softmax_copy_kernel(TokenView from, T* to, int heads, int tokens, int d, int width, long long count) {
  for (long long at = 256 * ((long long)blockIdx.x) + threadIdx.x; at < count; at += 256 * (long long)gridDim.x) {
    const int c = (int)(at % width);
    const long long row = at / width, i = row % tokens, h = row / tokens % heads, b = row / tokens / heads;
    to[at] = c < d ? reinterpret_cast<const T*>(from.data)[b * from.sb + h * from.sh + i * from.sn + c] : (T)0;
  }
}

int padded(int d, int es) { return (d * es + 15) / 16 * 16 / es; }

// whether the kernels can take the tensor as it lies: whole 16-byte pieces, a tile's rows within 2 GiB
bool in_pieces(const TokenView& v, int batch, int heads, int tokens, int d, int es) {
  const unsigned long long strides = (batch > 1 ? v.sb : 0) | (heads > 1 ? v.sh : 0) | (tokens > 1 ? v.sn : 0);
  return d * es % 16 == 0 && (uintptr_t)v.data % 16 == 0 && strides * es % 16 == 0 && (tokens == 1 || v.sn * es < (1 << 24));
}

size_t copy_bytes(const TokenView& v, int batch, int heads, int tokens, int d, int es) {
  if (v.data != nullptr && in_pieces(v, batch, heads, tokens, d, es)) return 0;
  return aligned((size_t)batch * heads * tokens * padded(d, es) * es);
}

hipError_t copy_to(TokenView& v, char*& ws, int batch, int heads, int tokens, int d, int es, hipStream_t st) {
  const size_t bytes = copy_bytes(v, batch, heads, tokens, d, es);
  if (bytes == 0) return hipSuccess;
  const int width = padded(d, es);
  const long long count = (long long)batch * heads * tokens * width;
  const unsigned blocks = (unsigned)std::min<long long>((count + 255) / 256, 1 << 16);
  if (es == 4) softmax_copy_kernel<uint32_t><<<blocks, 256, 0, st>>>(v, (uint32_t*)ws, heads, tokens, d, width, count);
  else softmax_copy_kernel<uint16_t><<<blocks, 256, 0, st>>>(v, (uint16_t*)ws, heads, tokens, d, width, count);
  v = TokenView{ws, (long long)heads * tokens * width, (long long)tokens * width, width};
  ws += bytes;
  return hipGetLastError();
}

hipError_t launch(int dtype, const SoftmaxArgs& a, SoftmaxPass pass, long long tiles, hipStream_t st) {
  const bool back = pass >= SoftmaxPass::kPeaks;
  const auto fn = dtype == 0 ? (back ? launch_softmax_bwd_f32 : launch_softmax_f32)
                             : dtype == 1 ? (back ? launch_softmax_bwd_f16 : launch_softmax_f16) : (back ? launch_softmax_bwd_bf16 : launch_softmax_bf16);
  return fn(a, pass, (int)tiles, st);
}

long long query_rows(const SoftmaxArgs& a) { return (long long)a.batch * a.heads_q * a.tokens_q; }
long long key_rows(const SoftmaxArgs& a) { return (long long)a.batch * a.heads_k * a.tokens_k; }
bool wide_result(const TokenView& v, int batch, int heads, int tokens, int d, int es) {
  const unsigned long long strides = (batch > 1 ? v.sb : 0) | (heads > 1 ? v.sh : 0) | (tokens > 1 ? v.sn : 0);
  return d * es % 16 == 0 && (uintptr_t)v.data % 16 == 0 && strides * es % 16 == 0;
}

}  // namespace

bool softmax_fits(int dtype, const SoftmaxArgs& a) {      // blocks are numbered in 32 bits
  const int es = dtype == 0 ? 4 : 2;
  const SoftmaxPlan p = softmax_plan(a, es);
  const SoftmaxBackPlan q = softmax_back_plan(a, es, false), k = softmax_back_plan(a, es, true);
  const long long outer = a.sequences > 0 ? 1 : a.batch, lim = 1ll << 30;
  return p.tiles * outer * a.heads_q / p.pack * p.splits < lim && q.tiles * outer * a.heads_q * q.splits < lim &&
         k.tiles * outer * a.heads_k * k.splits < lim;
}

size_t softmax_saved_lse(const SoftmaxArgs& a) { return aligned((size_t)query_rows(a) * 4); }
size_t softmax_saved_bytes(int dtype, const SoftmaxArgs& a) {
  return softmax_saved_lse(a) + (dtype == 0 ? 0 : aligned((size_t)query_rows(a) * a.d * 2));
}

size_t softmax_fwd_workspace(int dtype, const SoftmaxArgs& a) {
  const int es = dtype == 0 ? 4 : 2;
  size_t bytes = copy_bytes(a.q, a.batch, a.heads_q, a.tokens_q, a.d, es) + copy_bytes(a.k, a.batch, a.heads_k, a.tokens_k, a.d, es) +
                 copy_bytes(a.v, a.batch, a.heads_k, a.tokens_k, a.d, es);
  const SoftmaxPlan p = softmax_plan(a, es);
  if (p.splits > 1) bytes += aligned((size_t)p.splits * query_rows(a) * a.d * 4) + aligned((size_t)p.splits * query_rows(a) * 8);
  return bytes;
}

hipError_t launch_softmax_fwd(int dtype, SoftmaxArgs a, void* workspace, hipStream_t st) {
  const int es = dtype == 0 ? 4 : 2;
  char* ws = (char*)workspace;
  a.wide = wide_result(a.out, a.batch, a.heads_q, a.tokens_q, a.d, es);
  hipError_t err = copy_to(a.q, ws, a.batch, a.heads_q, a.tokens_q, a.d, es, st);
  if (err == hipSuccess) err = copy_to(a.k, ws, a.batch, a.heads_k, a.tokens_k, a.d, es, st);
  if (err == hipSuccess) err = copy_to(a.v, ws, a.batch, a.heads_k, a.tokens_k, a.d, es, st);
  if (err != hipSuccess) return err;
  const SoftmaxPlan p = softmax_plan(a, es);
  a.waves = p.waves, a.pack = p.pack, a.tile_tokens = p.tile_tokens, a.splits = p.splits;
  if (p.splits > 1) {
    a.part = (float*)ws;
    a.part_ml = (float*)(ws + aligned((size_t)p.splits * query_rows(a) * a.d * 4));
  }
  err = launch(dtype, a, p.columns ? SoftmaxPass::kColumns : SoftmaxPass::kRows, p.tiles, st);
  return err != hipSuccess || p.splits == 1 ? err : launch(dtype, a, SoftmaxPass::kJoin, 0, st);
}

size_t softmax_bwd_workspace(int dtype, const SoftmaxArgs& a) {
  const int es = dtype == 0 ? 4 : 2;
  const size_t q = copy_bytes(a.q, a.batch, a.heads_q, a.tokens_q, a.d, es), k = copy_bytes(a.k, a.batch, a.heads_k, a.tokens_k, a.d, es),
               v = copy_bytes(a.v, a.batch, a.heads_k, a.tokens_k, a.d, es), g = copy_bytes(a.dout, a.batch, a.heads_q, a.tokens_q, a.d, es);
  const int sq = softmax_back_plan(a, es, false).splits, sk = softmax_back_plan(a, es, true).splits;
  // the queries' parts are added up before the keys' are written
  const size_t parts = std::max(sq > 1 ? aligned((size_t)sq * query_rows(a) * a.d * 4) : 0,
                                sk > 1 ? 2 * aligned((size_t)sk * key_rows(a) * a.d * 4) : 0);
  return kAlign + aligned((size_t)query_rows(a) * 8) + q + k + v + g + parts;
}

hipError_t launch_softmax_bwd(int dtype, SoftmaxArgs a, void* workspace, hipStream_t st) {
  const int es = dtype == 0 ? 4 : 2;
  char* ws = (char*)workspace;
  a.peaks = (unsigned*)ws, ws += kAlign;
  a.stats = (float*)ws, ws += aligned((size_t)query_rows(a) * 8);
  a.wide = 1;
  for (const TokenView* v : {&a.out, &a.dq}) a.wide = a.wide && wide_result(*v, a.batch, a.heads_q, a.tokens_q, a.d, es);
  for (const TokenView* v : {&a.dk, &a.dv}) a.wide = a.wide && wide_result(*v, a.batch, a.heads_k, a.tokens_k, a.d, es);
  hipError_t err = copy_to(a.q, ws, a.batch, a.heads_q, a.tokens_q, a.d, es, st);
  if (err == hipSuccess) err = copy_to(a.k, ws, a.batch, a.heads_k, a.tokens_k, a.d, es, st);
  if (err == hipSuccess) err = copy_to(a.v, ws, a.batch, a.heads_k, a.tokens_k, a.d, es, st);
  if (err == hipSuccess) err = copy_to(a.dout, ws, a.batch, a.heads_q, a.tokens_q, a.d, es, st);
  if (err == hipSuccess && dtype == 1) err = launch(dtype, a, SoftmaxPass::kPeaks, 0, st);
  if (err != hipSuccess) return err;
  const SoftmaxBackPlan q = softmax_back_plan(a, es, false), k = softmax_back_plan(a, es, true);
  a.waves = q.waves, a.splits = q.splits;
  a.part_a = (float*)ws;
  err = launch(dtype, a, SoftmaxPass::kQueries, q.tiles, st);
  if (err == hipSuccess && a.splits > 1) err = launch(dtype, a, SoftmaxPass::kSumQueries, 0, st);
  if (err != hipSuccess) return err;
  a.waves = k.waves, a.splits = k.splits;
  a.part_b = (float*)(ws + aligned((size_t)a.splits * key_rows(a) * a.d * 4));
  err = launch(dtype, a, SoftmaxPass::kKeys, k.tiles, st);
  return err != hipSuccess || a.splits == 1 ? err : launch(dtype, a, SoftmaxPass::kSumKeys, 0, st);
}

}  // namespace aa
