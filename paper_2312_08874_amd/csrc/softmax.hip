// Softmax attention: launch sequences, and copies of tensors whose rows are no whole 16-byte pieces.
#include "kernels.h"
#include "softmax_common.inc"

namespace aa {

namespace {

constexpr size_t kAlign = 256;
size_t aligned(size_t bytes) { return (bytes + kAlign - 1) / kAlign * kAlign; }
constexpr size_t kPeakBytes = 2 * kPeakBlocks * sizeof(float);

// Rows of d elements of ES bytes, at any address of an element, to dense rows of whole 16-byte pieces, zeros behind their end: a piece a
// thread; along y the tensors.
struct CopyOf {
  TokenView from;
  char* to;
  int heads, tokens, units;      // units: heads of all batch elements
};
struct CopyArgs {
  CopyOf t[4];
  int d, pieces;
};
template <int ES>
__global__ __launch_bounds__(256) void softmax_copy_kernel(CopyArgs a) {
  typedef uint32_t OffWord __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t OffHalf __attribute__((ext_vector_type(4), aligned(2)));
  using AnyPiece = std::conditional_t<ES == 4, OffWord, OffHalf>;
  using T = std::conditional_t<ES == 4, uint32_t, uint16_t>;
  constexpr int PER = 16 / ES;
  const CopyOf& x = a.t[blockIdx.y];
  const int rows = 256 / a.pieces, slot = threadIdx.x / a.pieces, piece = threadIdx.x - slot * a.pieces;
  if (slot >= rows) return;
  const int at = blockIdx.x * rows + slot, stride = rows * gridDim.x, skip = stride / x.tokens, rest = stride % x.tokens;
  int unit = at / x.tokens, i = at % x.tokens;
  while (unit < x.units) {
    const int b = unit / x.heads, h = unit - b * x.heads;
    const T* p = reinterpret_cast<const T*>(x.from.data) + (long long)b * x.from.sb + (long long)h * x.from.sh + (long long)i * x.from.sn + piece * PER;
    u32x4 v = {0u, 0u, 0u, 0u};
    if ((piece + 1) * PER <= a.d) {
      v = __builtin_bit_cast(u32x4, *reinterpret_cast<const AnyPiece*>(p));
    } else {
#pragma unroll
      for (int n = 0; n < PER - 1; ++n)
        if (piece * PER + n < a.d) v[n * ES / 4] |= (uint32_t)p[n] << (8 * (n * ES % 4));
    }
    *reinterpret_cast<u32x4*>(x.to + (((long long)unit * x.tokens + i) * a.pieces + piece) * 16) = v;
    unit += skip, i += rest;
    if (i >= x.tokens) i -= x.tokens, ++unit;
  }
}
// fp32 rows to dense rows of three terms, 8 * pieces bf16 values each: eight channels a thread; along y the tensors
struct TermsOf {
  TokenView from;
  uint16_t* to;
  int heads, tokens;
  unsigned count;      // threads
};
struct TermsArgs {
  TermsOf t[4];
  int d, pieces;
};
__global__ __launch_bounds__(256) void softmax_terms_kernel(TermsArgs a) {
  const TermsOf& x = a.t[blockIdx.y];
  const bool whole = a.d % 8 == 0 && ((uintptr_t)x.from.data | (x.from.sb | x.from.sh | x.from.sn) * 4) % 16 == 0;
  for (unsigned at = 256 * blockIdx.x + threadIdx.x; at < x.count; at += 256 * gridDim.x) {
    const unsigned row = at / (unsigned)a.pieces, c = 8 * (at - row * a.pieces);
    const unsigned unit = row / (unsigned)x.tokens, i = row - unit * x.tokens, b = unit / (unsigned)x.heads, h = unit - b * x.heads;
    const float* p = reinterpret_cast<const float*>(x.from.data) + b * x.from.sb + h * x.from.sh + i * x.from.sn + c;
    float v[8];
    if (whole) {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int n = 0; n < 4; ++n) v[n] = lo[n], v[4 + n] = hi[n];
    } else {
#pragma unroll
      for (int n = 0; n < 8; ++n) v[n] = (int)c + n < a.d ? p[n] : 0.0f;
    }
    u32x4 t[3];
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      uint32_t w[3];
      three_terms(v[2 * n], v[2 * n + 1], w);
#pragma unroll
      for (int k = 0; k < 3; ++k) t[k][n] = w[k];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<u32x4*>(x.to + (3ull * row + k) * 8 * a.pieces + c) = t[k];
  }
}

int padded(int d, int es) { return (d * es + 15) / 16 * 16 / es; }

// whether the kernels can take the tensor as it lies: whole 16-byte pieces, a tile's rows within 2 GiB
bool in_pieces(const TokenView& v, int batch, int heads, int tokens, int d, int es) {
  const unsigned long long strides = (batch > 1 ? v.sb : 0) | (heads > 1 ? v.sh : 0) | (tokens > 1 ? v.sn : 0);
  return d * es % 16 == 0 && (uintptr_t)v.data % 16 == 0 && strides * es % 16 == 0 && (tokens == 1 || v.sn * es < (1 << 24));
}

// terms > 1: taken apart in any case
size_t copy_bytes(const TokenView& v, int batch, int heads, int tokens, int d, int es, int terms) {
  if (terms > 1) return aligned((size_t)batch * heads * tokens * padded(d, 2) * 2 * terms);
  if (v.data != nullptr && in_pieces(v, batch, heads, tokens, d, es)) return 0;
  return aligned((size_t)batch * heads * tokens * padded(d, es) * es);
}

// q, k, v and, of the backward pass, dout in a form that the kernels can take, in the workspace where they lie in none
hipError_t take_inputs(SoftmaxArgs& a, char*& ws, int es, int terms, bool back, hipStream_t st) {
  TokenView* const views[] = {&a.q, &a.k, &a.v, &a.dout};
  const int count = back ? 4 : 3;
  a.term = 2 * padded(a.d, 2);
  if (terms > 1) {
    TermsArgs t{};
    t.d = a.d, t.pieces = padded(a.d, 2) / 8;
    unsigned most = 0;
    for (int i = 0; i < count; ++i) {
      const bool keys = i == 1 || i == 2;
      const int heads = keys ? a.heads_k : a.heads_q, tokens = keys ? a.tokens_k : a.tokens_q;
      const long long step = terms * padded(a.d, 2), rows = (long long)a.batch * heads * tokens;
      t.t[i] = TermsOf{*views[i], (uint16_t*)ws, heads, tokens, (unsigned)(rows * t.pieces)};
      most = std::max(most, t.t[i].count);
      *views[i] = TokenView{ws, heads * tokens * step, tokens * step, step};
      ws += copy_bytes(*views[i], a.batch, heads, tokens, a.d, es, terms);
    }
    softmax_terms_kernel<<<dim3(std::min((most + 255) / 256, 1u << 13), (unsigned)count), 256, 0, st>>>(t);
    return hipGetLastError();
  }
  CopyArgs c{};
  c.d = a.d, c.pieces = padded(a.d, es) * es / 16;
  int copies = 0;
  long long most = 0;
  for (int i = 0; i < count; ++i) {
    const bool keys = i == 1 || i == 2;
    const int heads = keys ? a.heads_k : a.heads_q, tokens = keys ? a.tokens_k : a.tokens_q, width = padded(a.d, es);
    const size_t bytes = copy_bytes(*views[i], a.batch, heads, tokens, a.d, es, 1);
    if (bytes == 0) continue;
    c.t[copies++] = CopyOf{*views[i], ws, heads, tokens, a.batch * heads};
    most = std::max(most, (long long)a.batch * heads * tokens);
    *views[i] = TokenView{ws, (long long)heads * tokens * width, (long long)tokens * width, width};
    ws += bytes;
  }
  if (copies == 0) return hipSuccess;
  const long long rows = 256 / c.pieces;
  const dim3 grid((unsigned)std::min<long long>((most + rows - 1) / rows, 1 << 12), (unsigned)copies);
  if (es == 4) softmax_copy_kernel<4><<<grid, 256, 0, st>>>(c);
  else softmax_copy_kernel<2><<<grid, 256, 0, st>>>(c);
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
  // and so are the pieces of eight channels that fp32 tensors are taken apart in
  if (es == 4 && std::max(query_rows(a), key_rows(a)) * (padded(a.d, 2) / 8) >= 2 * lim) return false;
  return p.tiles * outer * a.heads_q / p.pack * p.splits < lim && q.tiles * outer * a.heads_q * q.splits < lim &&
         k.tiles * outer * a.heads_k * k.splits < lim;
}

size_t softmax_saved_lse(const SoftmaxArgs& a) { return aligned((size_t)query_rows(a) * 4); }
bool softmax_keeps_low(int dtype, const SoftmaxArgs& a) {
  const bool all_long = a.sequences == 0 && !a.causal && a.lengths_k == nullptr && a.tokens_k > kLowKeys;      // no row sees so few keys
  return dtype != 0 && !all_long;
}
size_t softmax_saved_bytes(int dtype, const SoftmaxArgs& a) {
  return softmax_saved_lse(a) + (softmax_keeps_low(dtype, a) ? aligned((size_t)query_rows(a) * a.d * 2) : 0);
}

size_t softmax_fwd_workspace(int dtype, const SoftmaxArgs& a) {
  const int es = dtype == 0 ? 4 : 2;
  const SoftmaxPlan p = softmax_plan(a, es);
  const int terms = p.columns ? 1 : softmax_terms(es, softmax_width(a.d));
  size_t bytes = copy_bytes(a.q, a.batch, a.heads_q, a.tokens_q, a.d, es, terms) + copy_bytes(a.k, a.batch, a.heads_k, a.tokens_k, a.d, es, terms) +
                 copy_bytes(a.v, a.batch, a.heads_k, a.tokens_k, a.d, es, terms);
  if (p.splits > 1) bytes += aligned((size_t)p.splits * query_rows(a) * a.d * 4) + aligned((size_t)p.splits * query_rows(a) * 12);
  return bytes;
}

hipError_t launch_softmax_fwd(int dtype, SoftmaxArgs a, void* workspace, hipStream_t st) {
  const int es = dtype == 0 ? 4 : 2;
  const SoftmaxPlan p = softmax_plan(a, es);
  const int terms = p.columns ? 1 : softmax_terms(es, softmax_width(a.d));
  char* ws = (char*)workspace;
  a.wide = wide_result(a.out, a.batch, a.heads_q, a.tokens_q, a.d, es);
  hipError_t err = take_inputs(a, ws, es, terms, false, st);
  if (err != hipSuccess) return err;
  a.waves = p.waves, a.shared = p.shared, a.pack = p.pack, a.tile_tokens = p.tile_tokens, a.splits = p.splits;
  if (p.splits > 1) {
    a.part = (float*)ws;
    a.part_stats = (float*)(ws + aligned((size_t)p.splits * query_rows(a) * a.d * 4));
  }
  err = launch(dtype, a, p.columns ? SoftmaxPass::kColumns : SoftmaxPass::kRows, p.tiles, st);
  return err != hipSuccess || p.splits == 1 ? err : launch(dtype, a, SoftmaxPass::kJoin, 0, st);
}

size_t softmax_bwd_workspace(int dtype, const SoftmaxArgs& a) {
  const int es = dtype == 0 ? 4 : 2, terms = softmax_terms(es, softmax_width(a.d));
  const size_t q = copy_bytes(a.q, a.batch, a.heads_q, a.tokens_q, a.d, es, terms), k = copy_bytes(a.k, a.batch, a.heads_k, a.tokens_k, a.d, es, terms),
               v = copy_bytes(a.v, a.batch, a.heads_k, a.tokens_k, a.d, es, terms), g = copy_bytes(a.dout, a.batch, a.heads_q, a.tokens_q, a.d, es, terms);
  const int sq = softmax_back_plan(a, es, false).splits, sk = softmax_back_plan(a, es, true).splits;
  // the queries' parts are added up before the keys' are written
  const size_t parts = std::max(sq > 1 ? aligned((size_t)sq * query_rows(a) * a.d * 4) : 0,
                                sk > 1 ? 2 * aligned((size_t)sk * key_rows(a) * a.d * 4) : 0);
  return (dtype == 1 ? kPeakBytes : 0) + aligned((size_t)query_rows(a) * 8) + q + k + v + g + parts;
}

hipError_t launch_softmax_bwd(int dtype, SoftmaxArgs a, void* workspace, hipStream_t st) {
  const int es = dtype == 0 ? 4 : 2, terms = softmax_terms(es, softmax_width(a.d));
  char* ws = (char*)workspace;
  a.dout_whole = a.dout;
  if (dtype == 1) {
    const long long blocks = (std::max(query_rows(a), key_rows(a)) + 127) / 128;
    a.peaks = (float*)ws, ws += kPeakBytes;
    a.peak_blocks = (int)std::min<long long>((blocks + 7) / 8 * 8, kPeakBlocks);
  }
  a.stats = (float*)ws, ws += aligned((size_t)query_rows(a) * 8);
  a.wide = 1;
  for (const TokenView* v : {&a.out, &a.dq, &a.dout_whole}) a.wide = a.wide && wide_result(*v, a.batch, a.heads_q, a.tokens_q, a.d, es);
  for (const TokenView* v : {&a.dk, &a.dv}) a.wide = a.wide && wide_result(*v, a.batch, a.heads_k, a.tokens_k, a.d, es);
  hipError_t err = take_inputs(a, ws, es, terms, true, st);
  if (err == hipSuccess && dtype == 1) err = launch(dtype, a, SoftmaxPass::kPeaks, 0, st);
  if (err != hipSuccess) return err;
  const SoftmaxBackPlan q = softmax_back_plan(a, es, false), k = softmax_back_plan(a, es, true);
  a.two = softmax_two_roundings(a, es);
  a.waves = q.waves, a.shared = q.shared, a.splits = q.splits;
  a.part_a = (float*)ws;
  err = launch(dtype, a, SoftmaxPass::kQueries, q.tiles, st);
  if (err == hipSuccess && a.splits > 1) err = launch(dtype, a, SoftmaxPass::kSumQueries, 0, st);
  if (err != hipSuccess) return err;
  a.waves = k.waves, a.shared = k.shared, a.splits = k.splits;
  a.part_b = (float*)(ws + aligned((size_t)a.splits * key_rows(a) * a.d * 4));
  err = launch(dtype, a, SoftmaxPass::kKeys, k.tiles, st);
  return err != hipSuccess || a.splits == 1 ? err : launch(dtype, a, SoftmaxPass::kSumKeys, 0, st);
}

}  // namespace aa
