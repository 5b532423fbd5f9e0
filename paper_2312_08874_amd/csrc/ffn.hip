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

// out[row][n] = sum over the parts of partial[part][row][n] (+ bias[n]), rounded once; rows from row_part on go to out1, rows of a
// part past `rows` nowhere.  The parts in their order.
struct SumArgs {
  const float* partial;
  int parts, M, N, pitch, row_part, rows;
  long long ldo;
  void *out0, *out1;
  const void* bias;
};
template <class E>
__global__ __launch_bounds__(256) void ffn_sum_kernel(SumArgs a) {
  using T = typename E::T;
  const int quads = (a.N + 3) / 4;
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x, row = at / quads;
  const int n = (int)(at - row * quads) * 4;
  if (row >= a.M) return;
  const bool second = a.row_part > 0 && row >= a.row_part;
  const long long rr = second ? row - a.row_part : row;
  T* to = (T*)(second ? a.out1 : a.out0);
  if (to == nullptr || (a.row_part > 0 && rr >= a.rows)) return;
  const float* from = a.partial + row * a.pitch + n;
  const size_t part = (size_t)a.M * a.pitch;
  f32x4 v = *reinterpret_cast<const f32x4*>(from);
#pragma unroll 4
  for (int p = 1; p < a.parts; ++p) v += *reinterpret_cast<const f32x4*>(from + p * part);
  to += rr * a.ldo + n;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < a.N) to[i] = to_elem<E>(v[i] + (a.bias != nullptr ? E::to_f32(((const T*)a.bias)[n + i]) : 0.0f));
}

// partial[part][c] = sum over the part's rows of in[row][c]: a block takes 64 columns, four rows at a time.
template <class E>
__global__ __launch_bounds__(256) void ffn_column_sum_kernel(const void* in, long long ld, int rows, int cols, int rows_each, int pitch,
                                                             float* partial) {
  __shared__ float sums[4][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), sub = threadIdx.x >> 6;
  const int r0 = blockIdx.y * rows_each, r1 = min(rows, r0 + rows_each);
  float v = 0.0f;
  if (c < cols) {
    const typename E::T* p = (const typename E::T*)in + c;
#pragma unroll 8
    for (int r = r0 + sub; r < r1; r += 4) v += E::to_f32(p[r * ld]);
  }
  sums[sub][threadIdx.x & 63] = v;
  __syncthreads();
  if (sub == 0 && c < cols) {
    const int i = threadIdx.x;
    partial[(size_t)blockIdx.y * pitch + c] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
  }
}
constexpr int kSumRows = 512;      // rows of a part, at least; at most 64 parts
int column_parts(int rows) { return std::min(64, (rows + kSumRows - 1) / kSumRows); }

// --- workspaces ---
// Copies of operands whose rows are no whole 16-byte pieces; their room is always kept, since the tensors' addresses are not
// known to a query.
struct Plan {
  size_t x, dy, w_gate, w_up, w_down;      // copies
  size_t h, dgu, partial, total;
};
struct Products {
  FfnTile gate, down, dh, dx, dw_in, dw_down;
};
int steps_of(const FfnBlock& b, int k) { return (k * b.es() + 127) / 128; }
Products products(const FfnBlock& b) {
  const int pitch = ffn_pitch(b.F), es = b.es();
  auto tile = [&](long long M, long long N, int k, bool split, bool gated) {
    return ffn_tile(M, N, steps_of(b, k), es, split, gated, kComputeUnits);
  };
  return Products{tile(b.T, pitch, b.C, false, true), tile(b.T, b.C, b.F, true, false), tile(b.T, pitch, b.C, false, false),
                  tile(b.T, b.C, 2 * pitch, true, false), tile(2 * pitch, b.C, b.T, true, false), tile(b.C, b.F, b.T, true, false)};
}
size_t partial_bytes(const FfnTile& t, long long M, int N) { return t.splits > 1 ? (size_t)t.splits * M * round_up(N, 8) * 4 : 0; }

Plan make_plan(const FfnBlock& b, bool backward) {
  const size_t es = b.es(), pitch = ffn_pitch(b.F), C = round_up(b.C, b.unit()), F = round_up(b.F, b.unit());
  const Products p = products(b);
  Plan w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += align_up(bytes);
    return o;
  };
  w.x = take((size_t)b.T * C * es);
  if (backward) w.dy = take((size_t)b.T * C * es);
  w.w_gate = take((size_t)b.F * C * es);
  w.w_up = take((size_t)b.F * C * es);
  w.w_down = take((size_t)b.C * F * es);
  if (backward) w.dgu = take((size_t)b.T * 2 * pitch * es);
  else w.h = take((size_t)b.T * pitch * (b.T <= kFfnFewRows ? 4 : es));
  size_t part = 0;
  if (backward) {
    part = std::max({partial_bytes(p.dx, b.T, b.C), partial_bytes(p.dw_in, 2 * (long long)pitch, b.C), partial_bytes(p.dw_down, b.C, b.F),
                     (size_t)column_parts(b.T) * std::max<size_t>(2 * pitch, round_up(b.C, 8)) * 4});
  } else {
    part = partial_bytes(p.down, b.T, b.C);
  }
  w.partial = take(part);
  w.total = std::max(at, kAlign);
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
    const int es = b.es(), unit = b.unit();
    if (((uintptr_t)p & 15) == 0 && ld % unit == 0 && cols % unit == 0) return Rows{p, ld};
    CopyJob& j = jobs.job[jobs.count++];
    j = CopyJob{p, ws + room, ld, rows, cols, round_up(cols, unit)};
    (void)es;
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

hipError_t launch_sum(int dtype, const SumArgs& a, hipStream_t st) {
  const long long threads = (long long)a.M * ((a.N + 3) / 4);
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (dtype == 0) ffn_sum_kernel<ElemF32><<<grid, dim3(256), 0, st>>>(a);
  else if (dtype == 1) ffn_sum_kernel<ElemF16><<<grid, dim3(256), 0, st>>>(a);
  else ffn_sum_kernel<ElemBF16><<<grid, dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_product(int dtype, const FfnProduct& a, FfnForm form, FfnEpilogue epi, const FfnTile& t, hipStream_t st) {
  if (dtype == 0) return launch_ffn_product_f32(a, form, epi, t, st);
  return dtype == 1 ? launch_ffn_product_f16(a, form, epi, t, st) : launch_ffn_product_bf16(a, form, epi, t, st);
}

// kStore, over parts of k where the tile says so
hipError_t store_product(const FfnBlock& b, FfnProduct a, FfnForm form, const FfnTile& t, float* partial, hipStream_t st) {
  a.aligned = ((uintptr_t)a.out[0] & 15) == 0 && ((uintptr_t)a.out[1] & 15) == 0 && a.ldo % b.unit() == 0;
  const int steps = steps_of(b, a.K);
  a.splits = t.splits, a.split_steps = (steps + t.splits - 1) / t.splits;
  if (t.splits == 1) return launch_product(b.dtype, a, form, FfnEpilogue::kStore, t, st);
  a.partial = partial, a.pitch = round_up(a.N, 8);
  const hipError_t err = launch_product(b.dtype, a, form, FfnEpilogue::kPartial, t, st);
  if (err != hipSuccess) return err;
  return launch_sum(b.dtype, SumArgs{partial, t.splits, a.M, a.N, a.pitch, a.row_part, a.rows, a.ldo, a.out[0], a.out[1], a.bias[0]}, st);
}

hipError_t column_sums(int dtype, const void* in, long long ld, int rows, int cols, float* partial, void* out, hipStream_t st) {
  const int parts = column_parts(rows), each = (rows + parts - 1) / parts, pitch = round_up(cols, 8);
  const dim3 grid((unsigned)((cols + 63) / 64), (unsigned)parts), block(256);
  if (dtype == 0) ffn_column_sum_kernel<ElemF32><<<grid, block, 0, st>>>(in, ld, rows, cols, each, pitch, partial);
  else if (dtype == 1) ffn_column_sum_kernel<ElemF16><<<grid, block, 0, st>>>(in, ld, rows, cols, each, pitch, partial);
  else ffn_column_sum_kernel<ElemBF16><<<grid, block, 0, st>>>(in, ld, rows, cols, each, pitch, partial);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  return launch_sum(dtype, SumArgs{partial, parts, 1, cols, pitch, 0, 0, cols, out, nullptr, nullptr}, st);
}

}  // namespace

size_t ffn_saved_bytes(const FfnBlock& b) { return saved_plan(b).total; }
size_t ffn_fwd_workspace(const FfnBlock& b) { return make_plan(b, false).total; }
size_t ffn_bwd_workspace(const FfnBlock& b) { return make_plan(b, true).total; }

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

hipError_t launch_ffn_fwd(const FfnBlock& b, void* saved, void* workspace, hipStream_t st) {
  char* ws = (char*)workspace;
  const Plan w = make_plan(b, false);
  if (b.T <= kFfnFewRows) return few_rows_fwd(b, (char*)saved, ws + w.h, st);
  const Products p = products(b);
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
  FfnProduct g{};
  g.a = x.p, g.lda = x.ld, g.b[0] = wg2.p, g.b[1] = wu.p, g.ldb = wg2.ld;
  g.M = b.T, g.N = b.F, g.K = round_up(b.C, unit), g.splits = 1, g.split_steps = steps_of(b, g.K);
  g.bias[0] = b.b_gate, g.bias[1] = b.b_up, g.pitch = pitch, g.hidden = b.F, g.activation = b.activation;
  g.h = keep ? keep + s.h : ws + w.h;
  if (keep) {
    g.p_hi = (uint16_t*)(keep + s.p_hi), g.q_hi = (uint16_t*)(keep + s.q_hi);
    g.p_lo = (uint8_t*)(keep + s.p_lo), g.q_lo = (uint8_t*)(keep + s.q_lo);
  }
  AA_TRY(launch_product(b.dtype, g, FfnForm::kKK, FfnEpilogue::kGate, p.gate, st));
  FfnProduct d{};
  d.a = g.h, d.lda = pitch, d.b[0] = wd.p, d.ldb = wd.ld, d.M = b.T, d.N = b.C, d.K = round_up(b.F, unit);
  d.out[0] = b.y, d.ldo = b.ldy, d.bias[0] = b.b_down;
  return store_product(b, d, FfnForm::kKK, p.down, (float*)(ws + w.partial), st);
}

hipError_t launch_ffn_bwd(const FfnBlock& b, const void* saved, void* workspace, hipStream_t st) {
  char* ws = (char*)workspace;
  const Plan w = make_plan(b, true);
  const Products p = products(b);
  const Saved s = saved_plan(b);
  const int pitch = ffn_pitch(b.F), unit = b.unit(), C = round_up(b.C, unit), F = round_up(b.F, unit);
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
    FfnProduct g{};
    g.a = dy.p, g.lda = dy.ld, g.b[0] = wd.p, g.ldb = wd.ld, g.b_m = F, g.b_rows = b.C, g.M = b.T, g.N = b.F, g.K = C;
    g.splits = 1, g.split_steps = steps_of(b, C), g.pitch = pitch, g.hidden = b.F, g.out[0] = dgu;
    g.p_hi = (uint16_t*)(keep + s.p_hi), g.q_hi = (uint16_t*)(keep + s.q_hi);
    g.p_lo = (uint8_t*)(keep + s.p_lo), g.q_lo = (uint8_t*)(keep + s.q_lo);
    AA_TRY(launch_product(b.dtype, g, FfnForm::kKM, FfnEpilogue::kGateGrad, p.dh, st));
  }
  if (want_dx) {
    FfnProduct d{};
    d.a = dgu, d.lda = 2 * (long long)pitch, d.b[0] = wg.p, d.b[1] = wu.p, d.ldb = wg.ld, d.b_m = C, d.b_rows = b.F, d.b_parts = 2;
    d.k_part = pitch, d.M = b.T, d.N = b.C, d.K = 2 * pitch, d.out[0] = b.dx, d.ldo = b.lddx;
    AA_TRY(store_product(b, d, FfnForm::kKM, p.dx, partial, st));
  }
  if (dw_in) {
    FfnProduct d{};
    d.a = dgu, d.lda = 2 * (long long)pitch, d.a_m = 2 * pitch, d.b[0] = x.p, d.ldb = x.ld, d.b_m = C, d.b_rows = b.T;
    d.M = 2 * pitch, d.N = b.C, d.K = b.T, d.row_part = pitch, d.rows = b.F, d.out[0] = b.dw_gate, d.out[1] = b.dw_up, d.ldo = b.C;
    AA_TRY(store_product(b, d, FfnForm::kMM, p.dw_in, partial, st));
  }
  if (b.dw_down) {
    FfnProduct d{};
    d.a = dy.p, d.lda = dy.ld, d.a_m = C, d.b[0] = keep + s.h, d.ldb = pitch, d.b_m = pitch, d.b_rows = b.T;
    d.M = b.C, d.N = b.F, d.K = b.T, d.out[0] = b.dw_down, d.ldo = b.F;
    AA_TRY(store_product(b, d, FfnForm::kMM, p.dw_down, partial, st));
  }
  if (b.db_gate) AA_TRY(column_sums(b.dtype, dgu, 2 * (long long)pitch, b.T, b.F, partial, b.db_gate, st));
  if (b.db_up) AA_TRY(column_sums(b.dtype, (const char*)dgu + (size_t)pitch * b.es(), 2 * (long long)pitch, b.T, b.F, partial, b.db_up, st));
  if (b.db_down) AA_TRY(column_sums(b.dtype, dy.p, dy.ld, b.T, b.C, partial, b.db_down, st));
  return hipSuccess;
}

}  // namespace aa
