// Launch sequence of the gated feed-forward block, forward and backward, with the small kernels beside its products: rows made
// whole 16-byte pieces, parts of k added up, column sums for the gradients of the biases.
#include <string.h>

#include "kernels.h"
#include "mfma_common.h"

namespace aa {

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
int round_up(int v, int unit) { return (v + unit - 1) / unit * unit; }

template <class E>
__device__ __forceinline__ typename E::T to_elem(float v) {
  if constexpr (sizeof(typename E::T) == 4) return v;
  else return __builtin_bit_cast(typename E::T, (uint16_t)Mx<E>::pack2(v, 0.0f));
}

// Rows copied to a pitch of whole 16-byte pieces, zeros behind them: what the products cannot read where it lies.
struct CopyJob {
  const void* src;
  void* dst;
  long long ld;
  int rows, cols, pitch;
};
struct CopyJobs {
  CopyJob job[5];
  int count;
};
template <class T>
__global__ __launch_bounds__(256) void ffn_copy_kernel(CopyJobs jobs) {
  constexpr int W = 16 / (int)sizeof(T);
  const CopyJob& j = jobs.job[blockIdx.y];
  const long long pieces = (long long)j.rows * (j.pitch / W);
  for (long long p = (long long)blockIdx.x * 256 + threadIdx.x; p < pieces; p += (long long)gridDim.x * 256) {
    const long long row = p / (j.pitch / W);
    const int c = (int)(p - row * (j.pitch / W)) * W;
    const T* src = (const T*)j.src + row * j.ld;
    T v[W];
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = c + i < j.cols ? src[c + i] : T(0);
    *reinterpret_cast<u32x4*>((T*)j.dst + row * j.pitch + c) = __builtin_bit_cast(u32x4, v);
  }
}

// The tiles of a group that were summed in parts: the parts in their order, the bias, one rounding.  A block takes 1024 results.
template <class E>
__global__ __launch_bounds__(256) void ffn_sum_kernel(FfnGroup g, int rows, int cols) {
  using T = typename E::T;
  const unsigned rest = blockIdx.y, tile = g.full + rest, tail = g.tiles - g.full;
  const int q = (int)(blockIdx.x * 256 + threadIdx.x) * 4, in = q / cols, c = q - in * cols;
  FfnProduct a = g.p[0];
  if (tile >= (unsigned)g.first) a = g.p[1];
  int tm, tn;
  ffn_place(tile >= (unsigned)g.first ? tile - g.first : tile, a.grid_m, a.grid_n, tm, tn);
  const int row = tm * rows + in, n = tn * cols + c;
  if (row >= a.M || n >= a.N) return;
  const bool second = a.row_part > 0 && row >= a.row_part;
  const int rr = second ? row - a.row_part : row;
  T* to = (T*)a.out[0];
  if (second) to = (T*)a.out[1];
  if (to == nullptr || (a.row_part > 0 && rr >= a.rows)) return;
  const size_t size = (size_t)rows * cols;
  const float* from = g.partial + rest * size + q;
  f32x4 v = *reinterpret_cast<const f32x4*>(from);
#pragma unroll 4
  for (int p = 1; p < g.parts; ++p) v += *reinterpret_cast<const f32x4*>(from + p * tail * size);
  to += (size_t)rr * a.ldo + n;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (a.bias[0] != nullptr && n + i < a.N) v[i] += E::to_f32(((const T*)a.bias[0])[n + i]);
  if (a.aligned && n + 4 <= a.N) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(to) = v;
    else *reinterpret_cast<u32x2*>(to) = u32x2{Mx<E>::pack2(v[0], v[1]), Mx<E>::pack2(v[2], v[3])};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < a.N) to[i] = to_elem<E>(v[i]);
  }
}

// Sums over the rows, up to three tensors in one launch: partial[part][first + c] = sum over the part's rows of in[row][c].  A block
// takes 64 columns, a thread 16 bytes of a row (rows are whole pieces, zeros behind the columns), 32 or 16 rows side by side.
struct SumJob {
  const void* in;
  long long ld;
  int cols, first;      // columns, and their place in the partial sums, a multiple of 64
  int second;           // elements to their second term, 0: they have one
  void* out;
};
struct SumJobs {
  SumJob job[3];
  int count, rows, rows_each, pitch;
};
__device__ __forceinline__ SumJob sum_job(const SumJobs& jobs, int column) {
  SumJob j = jobs.job[0];
#pragma unroll
  for (int i = 1; i < 3; ++i)
    if (i < jobs.count && column >= jobs.job[i].first) j = jobs.job[i];
  return j;
}
template <class E>
__global__ __launch_bounds__(256) void ffn_column_sum_kernel(SumJobs jobs, float* partial) {
  using T = typename E::T;
  constexpr int W = 16 / (int)sizeof(T), kAcross = 64 / W, kSide = 256 / kAcross;
  __shared__ float sums[kSide][64 + 4];      // + 4: rows on other banks
  const SumJob j = sum_job(jobs, blockIdx.x * 64);
  const int at = threadIdx.x % kAcross * W, side = threadIdx.x / kAcross, c = blockIdx.x * 64 - j.first + at;
  const long long r0 = (long long)blockIdx.y * jobs.rows_each, r1 = min((long long)jobs.rows, r0 + jobs.rows_each);
  float v[W] = {};
  if (c < j.cols) {
    const T* p = (const T*)j.in + c;
#pragma unroll 4
    for (long long r = r0 + side; r < r1; r += kSide) {
      T x[W];
      const u32x4 raw = *reinterpret_cast<const u32x4*>(p + r * j.ld);
      __builtin_memcpy(x, &raw, 16);
#pragma unroll
      for (int i = 0; i < W; ++i) v[i] += E::to_f32(x[i]);
      if (j.second > 0) {
        const u32x4 rest = *reinterpret_cast<const u32x4*>(p + r * j.ld + j.second);
        __builtin_memcpy(x, &rest, 16);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += E::to_f32(x[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < W; ++i) sums[side][at + i] = v[i];
  __syncthreads();
  if (threadIdx.x >= 64) return;
  float s[4] = {};
#pragma unroll
  for (int i = 0; i < kSide; ++i) s[i & 3] += sums[i][threadIdx.x];
  partial[(size_t)blockIdx.y * jobs.pitch + blockIdx.x * 64 + threadIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
}
// out[c] = sum over the parts of partial[part][c], in their order, rounded once
template <class E>
__global__ __launch_bounds__(256) void ffn_column_total_kernel(SumJobs jobs, const float* partial, int parts) {
  const int column = blockIdx.x * 256 + threadIdx.x;
  if (column >= jobs.pitch) return;
  const SumJob j = sum_job(jobs, column);
  if (column - j.first >= j.cols) return;
  float v = 0.0f;
#pragma unroll 8
  for (int p = 0; p < parts; ++p) v += partial[(size_t)p * jobs.pitch + column];
  ((typename E::T*)j.out)[column - j.first] = to_elem<E>(v);
}
constexpr int kSumRows = 256;      // rows of a part, at least; at most 64 parts
int column_parts(int rows) { return (int)std::min(64ll, (rows + (long long)kSumRows - 1) / kSumRows); }

// --- workspaces ---
// stored: the results are, as they are
FfnTile tile_for(const FfnBlock& b, long long M, long long N, long long M2, long long N2, long long k, bool split, bool gated, bool stored) {
  return ffn_tile(M, N, M2, N2, (k * b.es() + 127) / 128, b.es(), split, gated, kComputeUnits, stored);
}
int tiles_of(const FfnTile& t, long long M, long long N) { return (int)((M + t.rows - 1) / t.rows * ((N + t.cols - 1) / t.cols)); }
size_t partial_bytes(const FfnTile& t, int tiles) { return t.parts > 1 ? (size_t)(tiles - t.full) * t.parts * t.rows * t.cols * 4 : 0; }

// The products' tiles and where things lie in the workspace.  Copies of operands whose rows are no whole 16-byte pieces have
// their room always, since the tensors' addresses are not known to a query.
struct ForwardPlan {
  FfnTile gate{}, down{};
  size_t x = 0, w_gate = 0, w_up = 0, w_down = 0, h = 0, partial = 0, total = 0;
};
struct BackwardPlan {
  FfnTile dh{}, dx{}, dw{};
  size_t x = 0, dy = 0, w_gate = 0, w_up = 0, w_down = 0, dgu = 0, partial = 0, total = 0;
};
struct Regions {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t o = at;
    at += align_up(bytes);
    return o;
  }
};

ForwardPlan forward_plan(const FfnBlock& b) {
  const size_t es = b.es(), pitch = ffn_pitch(b.F), C = round_up(b.C, b.unit()), F = round_up(b.F, b.unit());
  ForwardPlan w;
  Regions r;
  if (ffn_few_rows(b.T, b.C, b.F)) {
    w.h = r.take((size_t)b.T * pitch * 4);      // fp32, or two terms
    w.total = r.at;
    return w;
  }
  w.gate = tile_for(b, b.T, pitch, 0, 0, b.C, false, true, false), w.down = tile_for(b, b.T, b.C, 0, 0, b.F, true, false, true);
  w.x = r.take((size_t)b.T * C * es);
  w.w_gate = r.take((size_t)b.F * C * es), w.w_up = r.take((size_t)b.F * C * es), w.w_down = r.take((size_t)b.C * F * es);
  w.h = r.take((size_t)b.T * pitch * es);
  w.partial = r.take(partial_bytes(w.down, tiles_of(w.down, b.T, b.C)));
  w.total = r.at;
  return w;
}

BackwardPlan backward_plan(const FfnBlock& b) {
  const size_t es = b.es(), pitch = ffn_pitch(b.F), C = round_up(b.C, b.unit()), F = round_up(b.F, b.unit());
  BackwardPlan w;
  Regions r;
  const int terms = ffn_terms(b.T, b.C, b.F, b.es());
  w.dh = tile_for(b, b.T, pitch, 0, 0, b.C, false, false, false), w.dx = tile_for(b, b.T, b.C, 0, 0, 2 * pitch * terms, true, false, true);
  w.dw = tile_for(b, 2 * pitch, b.C, b.C, b.F, (long long)b.T * terms, true, false, true);
  w.x = r.take((size_t)b.T * C * es), w.dy = r.take((size_t)b.T * C * es);
  w.w_gate = r.take((size_t)b.F * C * es), w.w_up = r.take((size_t)b.F * C * es), w.w_down = r.take((size_t)b.C * F * es);
  w.dgu = r.take((size_t)b.T * 2 * pitch * es * terms);
  w.partial = r.take(std::max({partial_bytes(w.dx, tiles_of(w.dx, b.T, b.C)),
                               partial_bytes(w.dw, tiles_of(w.dw, 2 * pitch, b.C) + tiles_of(w.dw, b.C, b.F)),
                               (size_t)column_parts(b.T) * (2 * pitch + round_up(b.C, 64)) * 4}));
  w.total = r.at;
  return w;
}

struct Saved {
  size_t h, p_hi, q_hi, p_lo, q_lo, total;
};
Saved saved_plan(const FfnBlock& b) {
  const size_t n = (size_t)b.T * ffn_pitch(b.F);
  Saved s{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align_up(bytes);
    return o;
  };
  s.h = take(n * b.es());
  s.p_hi = take(n * b.es());
  s.q_hi = take(n * b.es());
  if (b.es() == 2) s.p_lo = take(n), s.q_lo = take(n);
  s.total = at;
  return s;
}

struct Rows {
  const void* p;
  long long ld;
};
// Collects the copies that operands need and launches them.
struct Stager {
  const FfnBlock& b;
  char* ws;
  CopyJobs jobs{};
  Rows operand(const void* p, long long ld, int rows, int cols, size_t room) {
    const int unit = b.unit();
    if (((uintptr_t)p & 15) == 0 && ld % unit == 0 && cols % unit == 0) return Rows{p, ld};
    CopyJob& j = jobs.job[jobs.count++];
    j = CopyJob{p, ws + room, ld, rows, cols, round_up(cols, unit)};
    return Rows{j.dst, j.pitch};
  }
  hipError_t launch(hipStream_t st) {
    if (jobs.count == 0) return hipSuccess;
    long long most = 0;
    for (int i = 0; i < jobs.count; ++i) most = std::max(most, (long long)jobs.job[i].rows * (jobs.job[i].pitch / b.unit()));
    const dim3 grid((unsigned)std::min<long long>((most + 255) / 256, 2048), (unsigned)jobs.count);
    if (b.es() == 4) ffn_copy_kernel<float><<<grid, dim3(256), 0, st>>>(jobs);
    else ffn_copy_kernel<uint16_t><<<grid, dim3(256), 0, st>>>(jobs);
    return hipGetLastError();
  }
};

hipError_t launch_group(const FfnBlock& b, FfnGroup& g, FfnForm form, FfnEpilogue epi, const FfnTile& t, float* partial, hipStream_t st) {
  const int cols = epi == FfnEpilogue::kGate ? t.cols / 2 : t.cols;
  int tiles[2] = {0, 0};
  for (int i = 0; i < 2; ++i) {
    FfnProduct& a = g.p[i];
    const int N = epi == FfnEpilogue::kStore ? a.N : a.pitch;      // zeros behind the hidden width
    a.grid_m = (a.M + t.rows - 1) / t.rows, a.grid_n = (N + cols - 1) / cols;
    a.aligned = ((uintptr_t)a.out[0] & 15) == 0 && ((uintptr_t)a.out[1] & 15) == 0 && a.ldo % b.unit() == 0;
    tiles[i] = a.grid_m * a.grid_n;
  }
  g.first = tiles[0], g.tiles = tiles[0] + tiles[1], g.parts = t.parts, g.each = t.each, g.partial = partial;
  g.full = t.parts > 1 ? t.full : g.tiles;
  const hipError_t err = b.dtype == 0   ? launch_ffn_product_f32(g, form, epi, t.rows, t.cols, st)
                         : b.dtype == 1 ? launch_ffn_product_f16(g, form, epi, t.rows, t.cols, st)
                                        : launch_ffn_product_bf16(g, form, epi, t.rows, t.cols, st);
  if (err != hipSuccess || g.full == g.tiles) return err;
  const dim3 grid((unsigned)(t.rows * t.cols / 1024), (unsigned)(g.tiles - g.full)), block(256);
  if (b.dtype == 0) ffn_sum_kernel<ElemF32><<<grid, block, 0, st>>>(g, t.rows, t.cols);
  else if (b.dtype == 1) ffn_sum_kernel<ElemF16><<<grid, block, 0, st>>>(g, t.rows, t.cols);
  else ffn_sum_kernel<ElemBF16><<<grid, block, 0, st>>>(g, t.rows, t.cols);
  return hipGetLastError();
}

hipError_t column_sums(int dtype, SumJobs& jobs, float* partial, hipStream_t st) {
  if (jobs.count == 0) return hipSuccess;
  const int parts = column_parts(jobs.rows);
  jobs.rows_each = (int)((jobs.rows + (long long)parts - 1) / parts);
  const dim3 grid((unsigned)(jobs.pitch / 64), (unsigned)parts), block(256), total((unsigned)((jobs.pitch + 255) / 256));
  if (dtype == 0) ffn_column_sum_kernel<ElemF32><<<grid, block, 0, st>>>(jobs, partial);
  else if (dtype == 1) ffn_column_sum_kernel<ElemF16><<<grid, block, 0, st>>>(jobs, partial);
  else ffn_column_sum_kernel<ElemBF16><<<grid, block, 0, st>>>(jobs, partial);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  if (dtype == 0) ffn_column_total_kernel<ElemF32><<<total, block, 0, st>>>(jobs, partial, parts);
  else if (dtype == 1) ffn_column_total_kernel<ElemF16><<<total, block, 0, st>>>(jobs, partial, parts);
  else ffn_column_total_kernel<ElemBF16><<<total, block, 0, st>>>(jobs, partial, parts);
  return hipGetLastError();
}

}  // namespace

size_t ffn_saved_bytes(const FfnBlock& b) { return saved_plan(b).total; }
size_t ffn_fwd_workspace(const FfnBlock& b) { return forward_plan(b).total; }
size_t ffn_bwd_workspace(const FfnBlock& b) { return backward_plan(b).total; }

#define AA_TRY(call)                          \
  do {                                        \
    const hipError_t err_ = (call);           \
    if (err_ != hipSuccess) return err_;      \
  } while (0)

namespace {

hipError_t launch_rows(int dtype, const FfnRows& a, bool gate, int es, hipStream_t st) {
  const int waves = ffn_rows_waves((a.K * es + 63) / 64);
  if (dtype == 0) return launch_ffn_rows_f32(a, gate, waves, st);
  return dtype == 1 ? launch_ffn_rows_f16(a, gate, waves, st) : launch_ffn_rows_bf16(a, gate, waves, st);
}

hipError_t few_rows_fwd(const FfnBlock& b, char* keep, void* h, hipStream_t st) {
  const Saved s = saved_plan(b);
  FfnRows a{};
  a.w[0] = b.w_gate, a.w[1] = b.w_up, a.x = b.x, a.ldx = b.ldx, a.bias[0] = b.b_gate, a.bias[1] = b.b_up;
  a.M = b.T, a.N = b.F, a.K = b.C, a.pitch = ffn_pitch(b.F), a.activation = b.activation, a.h = h;
  if (keep) {
    a.kept_h = keep + s.h, a.p_hi = (uint16_t*)(keep + s.p_hi), a.q_hi = (uint16_t*)(keep + s.q_hi);
    a.p_lo = (uint8_t*)(keep + s.p_lo), a.q_lo = (uint8_t*)(keep + s.q_lo);
  }
  AA_TRY(launch_rows(b.dtype, a, true, b.es(), st));
  a.w[0] = b.w_down, a.bias[0] = b.b_down, a.N = b.C, a.K = b.F, a.y = b.y, a.ldy = b.ldy;
  return launch_rows(b.dtype, a, false, b.es(), st);
}

}  // namespace

hipError_t launch_ffn_fwd(const FfnBlock& b, void* saved, void* workspace, size_t bytes, bool* room, hipStream_t st) {
  char* ws = (char*)workspace;
  const ForwardPlan w = forward_plan(b);
  *room = bytes >= w.total;
  if (!*room) return hipSuccess;
  if (ffn_few_rows(b.T, b.C, b.F)) return few_rows_fwd(b, (char*)saved, ws + w.h, st);
  const Saved s = saved_plan(b);
  const int pitch = ffn_pitch(b.F), unit = b.unit();
  Stager stage{b, ws};
  const Rows x = stage.operand(b.x, b.ldx, b.T, b.C, w.x), wg = stage.operand(b.w_gate, b.C, b.F, b.C, w.w_gate);
  Rows wu = stage.operand(b.w_up, b.C, b.F, b.C, w.w_up), wd = stage.operand(b.w_down, b.F, b.C, b.F, w.w_down), wg2 = wg;
  if (wg.ld != wu.ld || (wg.p == b.w_gate) != (wu.p == b.w_up)) {      // one of them copied: both, to one pitch
    stage.jobs = CopyJobs{};
    (void)stage.operand(b.x, b.ldx, b.T, b.C, w.x);
    auto copy = [&](const void* src, size_t room) {
      stage.jobs.job[stage.jobs.count++] = CopyJob{src, ws + room, b.C, b.F, b.C, round_up(b.C, unit)};
      return Rows{ws + room, round_up(b.C, unit)};
    };
    wg2 = copy(b.w_gate, w.w_gate);
    wu = copy(b.w_up, w.w_up);
    (void)stage.operand(b.w_down, b.F, b.C, b.F, w.w_down);
  }
  AA_TRY(stage.launch(st));
  char* keep = (char*)saved;
  FfnGroup gate{}, down{};
  FfnProduct& g = gate.p[0];
  g.a = x.p, g.lda = x.ld, g.b[0] = wg2.p, g.b[1] = wu.p, g.ldb = wg2.ld;
  g.M = b.T, g.N = b.F, g.K = round_up(b.C, unit);
  g.bias[0] = b.b_gate, g.bias[1] = b.b_up, g.pitch = pitch, g.hidden = b.F, g.activation = b.activation;
  g.h = keep ? keep + s.h : ws + w.h;
  if (keep) {
    g.p_hi = (uint16_t*)(keep + s.p_hi), g.q_hi = (uint16_t*)(keep + s.q_hi);
    g.p_lo = (uint8_t*)(keep + s.p_lo), g.q_lo = (uint8_t*)(keep + s.q_lo);
  }
  AA_TRY(launch_group(b, gate, FfnForm::kKK, FfnEpilogue::kGate, w.gate, nullptr, st));
  FfnProduct& d = down.p[0];
  d.a = g.h, d.lda = pitch, d.b[0] = wd.p, d.ldb = wd.ld, d.M = b.T, d.N = b.C, d.K = round_up(b.F, unit);
  d.out[0] = b.y, d.ldo = b.ldy, d.bias[0] = b.b_down;
  return launch_group(b, down, FfnForm::kKK, FfnEpilogue::kStore, w.down, (float*)(ws + w.partial), st);
}

hipError_t launch_ffn_bwd(const FfnBlock& b, const void* saved, void* workspace, size_t bytes, bool* room, hipStream_t st) {
  char* ws = (char*)workspace;
  const BackwardPlan w = backward_plan(b);
  *room = bytes >= w.total;
  if (!*room) return hipSuccess;
  const Saved s = saved_plan(b);
  const int pitch = ffn_pitch(b.F), unit = b.unit(), C = round_up(b.C, unit), F = round_up(b.F, unit), terms = ffn_terms(b.T, b.C, b.F, b.es());
  const long long ldg = 2ll * pitch * terms;      // rows of dgate | dup (| their second terms)
  const char* keep = (const char*)saved;
  float* partial = (float*)(ws + w.partial);
  void* dgu = ws + w.dgu;
  Stager stage{b, ws};
  const bool dw_in = b.dw_gate || b.dw_up, want_dx = b.dx != nullptr;
  Rows x{}, wg{}, wu{};
  if (dw_in) x = stage.operand(b.x, b.ldx, b.T, b.C, w.x);
  const Rows dy = stage.operand(b.dy, b.ldy, b.T, b.C, w.dy), wd = stage.operand(b.w_down, b.F, b.C, b.F, w.w_down);
  if (want_dx) {
    const bool copy = ((uintptr_t)b.w_gate & 15) || ((uintptr_t)b.w_up & 15) || b.C % unit;      // both, to one pitch
    wg = wu = Rows{nullptr, b.C};
    wg.p = b.w_gate, wu.p = b.w_up;
    if (copy) {
      wg = Rows{ws + w.w_gate, C}, wu = Rows{ws + w.w_up, C};
      stage.jobs.job[stage.jobs.count++] = CopyJob{b.w_gate, ws + w.w_gate, b.C, b.F, b.C, C};
      stage.jobs.job[stage.jobs.count++] = CopyJob{b.w_up, ws + w.w_up, b.C, b.F, b.C, C};
    }
  }
  AA_TRY(stage.launch(st));
  if (want_dx || dw_in || b.db_gate || b.db_up) {
    FfnGroup group{};
    FfnProduct& g = group.p[0];
    g.a = dy.p, g.lda = dy.ld, g.b[0] = wd.p, g.ldb = wd.ld, g.b_m = F, g.b_rows = b.C, g.M = b.T, g.N = b.F, g.K = C;
    g.pitch = pitch, g.hidden = b.F, g.out[0] = dgu, g.ldo = ldg, g.terms = terms;
    g.p_hi = (uint16_t*)(keep + s.p_hi), g.q_hi = (uint16_t*)(keep + s.q_hi);
    g.p_lo = (uint8_t*)(keep + s.p_lo), g.q_lo = (uint8_t*)(keep + s.q_lo);
    AA_TRY(launch_group(b, group, FfnForm::kKM, FfnEpilogue::kGateGrad, w.dh, nullptr, st));
  }
  if (want_dx) {
    FfnGroup group{};
    FfnProduct& d = group.p[0];
    d.a = dgu, d.lda = ldg, d.terms = terms, d.b[0] = wg.p, d.b[1] = wu.p, d.ldb = wg.ld, d.b_m = C, d.b_rows = b.F, d.b_parts = 2;
    d.k_part = pitch, d.M = b.T, d.N = b.C, d.K = 2 * pitch * terms, d.out[0] = b.dx, d.ldo = b.lddx;
    AA_TRY(launch_group(b, group, FfnForm::kKM, FfnEpilogue::kStore, w.dx, partial, st));
  }
  if (dw_in || b.dw_down) {      // one launch: together they come nearer to whole rounds of the compute units
    FfnGroup group{};
    FfnProduct &d = group.p[0], &e = group.p[1];
    // dgate | dup of a token and their second terms are rows of their own here, both over the token's row of x
    d.a = dgu, d.lda = 2 * pitch, d.a_m = 2 * pitch, d.b[0] = x.p, d.ldb = x.ld, d.b_m = C, d.b_rows = b.T, d.b_twice = terms - 1;
    d.M = dw_in ? 2 * pitch : 0, d.N = b.C, d.K = b.T * terms, d.row_part = pitch, d.rows = b.F, d.out[0] = b.dw_gate, d.out[1] = b.dw_up, d.ldo = b.C;
    e.a = dy.p, e.lda = dy.ld, e.a_m = C, e.b[0] = keep + s.h, e.ldb = pitch, e.b_m = pitch, e.b_rows = b.T;
    e.M = b.dw_down ? b.C : 0, e.N = b.F, e.K = b.T, e.out[0] = b.dw_down, e.ldo = b.F;
    FfnTile t = w.dw;
    if (!dw_in || !b.dw_down)      // one of them alone: its own tiles, no more than the plan has room for
      t = tile_for(b, e.M > 0 ? e.M : d.M, e.M > 0 ? e.N : d.N, 0, 0, e.M > 0 ? e.K : d.K, false, false, true);
    AA_TRY(launch_group(b, group, FfnForm::kMM, FfnEpilogue::kStore, t, partial, st));
  }
  SumJobs sums{};
  sums.rows = b.T;
  auto sum = [&](const void* in, long long ld, int cols, int second, void* out) {
    if (!out) return;
    sums.job[sums.count++] = SumJob{in, ld, cols, sums.pitch, second, out};
    sums.pitch += round_up(cols, 64);
  };
  const int second = terms == 2 ? 2 * pitch : 0;
  sum(dgu, ldg, b.F, second, b.db_gate);
  sum((const char*)dgu + (size_t)pitch * b.es(), ldg, b.F, second, b.db_up);
  sum(dy.p, dy.ld, b.C, 0, b.db_down);
  AA_TRY(column_sums(b.dtype, sums, partial, st));
  return hipSuccess;
}

}  // namespace aa
