// 8-bit activation checkpoints and the element-wise operators around them: store, load, GELU forward
// (with checkpoints), and GELU backward (from a checkpoint, with the bias gradient).
// Every value is read and written once.  Store and load are bound by memory, GELU next to it by the instructions a value
// takes (35 forward with two checkpoints, 26 backward).  Measured on 16384 x 4096, among other calls, bf16 / fp32:
//   store 37 / 52 us (0.84 / 1.0 of a copy's rate), load 35 / 72 (0.90 / 0.71),
//   GELU forward with bias and two checkpoints, tanh 89 / 105 (0.70 / 0.98), erf 105 / 214 (0.59 / 0.48: normcdff),
//   GELU backward from a checkpoint with the bias gradient, tanh 78 / 111 (0.67 / 0.83), erf 90 / 194 (0.57 / 0.48).
#include "../../include/fa.h"
#include "fa_columns.cuh"
#include "fa_train.h"

namespace fa {
namespace act8 {

constexpr int kThreads = 256;
constexpr int kPer = 4;              // chunks per thread, loaded before any is worked on

// A launch covers the chunks 0 .. n-1 of its rows, `per_row` (4 a group) each; n < 2^31.
struct Flat {
  uint32_t n;
  int cols, groups, scale_pitch;
  FastDiv per_row;
};
// One of them: chunk c of a row.
struct At {
  uint32_t row;
  int c;
  bool valid;
  __device__ __forceinline__ At(const Flat& f, uint32_t i) : valid(i < f.n) {
    if (!valid) i = 0;
    row = f.per_row.div(i);
    c = static_cast<int>(i - row * f.per_row.d);
  }
};

template <typename T>
__device__ __forceinline__ void put_chunk(const Act8& ck, const Flat& f, const At& at, const Raw8<T>& raw) {
  const int g = at.c >> 2;
  act8_put(ck.codes + (size_t)at.row * f.groups * 32 + (size_t)at.c * 8, ck.scales + (size_t)at.row * f.scale_pitch + g, raw,
           (at.c & 3) == 0, g == f.groups - 1 ? -f.groups & 3 : 0, at.valid);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_flat(T* out, long long ld, const Flat& f, const At& at, const Raw8<T>& raw) {
  const int lane = threadIdx.x & 31;
  store_chunk<T, VEC>(out + at.row * ld, at.c * 8, f.cols, raw, at.valid, at.c > 0 && lane > 0,
                      at.c + 1 < static_cast<int>(f.per_row.d) && lane < 31);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) store_kernel(Source<T> x, Act8 ck, Flat f) {
  const uint32_t first = blockIdx.x * (kThreads * kPer) + threadIdx.x;
  Chunk<T, VEC> in[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const At at(f, first + k * kThreads);
    in[k].fetch(x, x.p + at.row * x.ld, at.c * 8, f.cols);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const At at(f, first + k * kThreads);
    put_chunk(ck, f, at, in[k].raw(at.c * 8 < f.cols));
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) load_kernel(Act8 ck, T* __restrict__ out, long long ldo, Flat f) {
  const uint32_t first = blockIdx.x * (kThreads * kPer) + threadIdx.x;
  RawAct8 q[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const At at(f, first + k * kThreads);
    q[k].load(ck, (long long)at.row * f.groups * 32 + at.c * 8, (long long)at.row * f.scale_pitch + (at.c >> 2), true);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    F2 v[4];
    q[k].get(v);
    Raw8<T> raw;
    raw.put(v);
    store_flat<T, VEC>(out, ldo, f, At(f, first + k * kThreads), raw);
  }
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// tanh form: z (1 + tanh u) / 2 = z S(2u) with the logistic function S and u = sqrt(2/pi) (z + 0.044715 z^3).
// S is formed as 1 / (1 + 2^t), t = -2u log2(e): without the cancellation of 1 + tanh, two instructions of the
// special function unit, off by a few units of 2^-23 wherever z S is not negligible.  z^2 is cut at 1000, where
// 2^t has long run out of range, so that no product below overflows.
constexpr float kT0 = -2.302208198144325f;            // -2 sqrt(2/pi) log2(e)
constexpr float kT1 = kT0 * 0.044715f;
constexpr float kU0 = 1.5957691216057308f;            // 2 sqrt(2/pi), of the derivative of 2u
constexpr float kU1 = 3.f * 0.044715f * kU0;
__device__ __forceinline__ F2 cut_square(F2 z) {
  float a, b;
  apart(mul2(z, z), &a, &b);
  return two(fminf(a, 1000.f), fminf(b, 1000.f));
}
__device__ __forceinline__ F2 logistic_2u(F2 z, F2 z2) {
  float a, b;
  apart(mul2(z, fma2(z2, two(kT1), two(kT0))), &a, &b);
  apart(add2(two(exp2_approx(a), exp2_approx(b)), two(1.f)), &a, &b);
  return two(rcp_approx(a), rcp_approx(b));
}

// erf form: z Phi(z).  In bf16 Phi comes from Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26
// (off by at most 1.5e-7, half of which reaches Phi), which shares its exponential with the density; in fp32 from
// CUDA's normcdff.  `density` receives exp(-z^2 / 2) / sqrt(2 pi).
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float* density) {
  const float e = exp2_approx(-0.7213475204444817f * z * z);      // exp(-z^2 / 2)
  *density = e * 0.3989422804014327f;
  if constexpr (sizeof(T) == 4) return normcdff(z);
  const float t = rcp_approx(fmaf(0.3275911f * 0.7071067811865476f, fabsf(z), 1.f));
  float q = fmaf(t, 1.061405429f, -1.453152027f);
  q = fmaf(t, q, 1.421413741f);
  q = fmaf(t, q, -0.284496736f);
  q = fmaf(t, q, 0.254829592f);
  q *= 0.5f * t * e;
  return z >= 0.f ? 1.f - q : q;
}

template <typename T, int APPROX>
__device__ __forceinline__ void gelu(float& a, float& b) {
  if constexpr (APPROX == kGeluTanh) {
    const F2 z = two(a, b);
    apart(mul2(z, logistic_2u(z, cut_square(z))), &a, &b);
  } else {
    float density;
    a *= normal_cdf<T>(a, &density);
    b *= normal_cdf<T>(b, &density);
  }
}
// tanh form: S + z S (1 - S) (2u)'; erf form: Phi + z phi.
template <typename T, int APPROX>
__device__ __forceinline__ F2 gelu_slope(float a, float b) {
  const F2 z = two(a, b);
  if constexpr (APPROX == kGeluTanh) {
    const F2 z2 = cut_square(z), s = logistic_2u(z, z2);
    const F2 t = fma2(mul2(s, two(-1.f)), s, s);
    return fma2(mul2(t, z), fma2(z2, two(kU1), two(kU0)), s);
  } else {
    float da, db;
    const float pa = normal_cdf<T>(a, &da), pb = normal_cdf<T>(b, &db);
    return fma2(z, two(da, db), two(pa, pb));
  }
}

template <typename T, bool VEC, int APPROX>
__global__ void __launch_bounds__(kThreads) gelu_forward_kernel(Source<T> x, ParamVec bias,
                                                                T* __restrict__ y, long long ldy, Act8 ck_x, Act8 ck_y,
                                                                Flat f) {
  const uint32_t first = blockIdx.x * (kThreads * kPer) + threadIdx.x;
  Chunk<T, VEC> in[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const At at(f, first + k * kThreads);
    in[k].fetch(x, x.p + at.row * x.ld, at.c * 8, f.cols);
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const At at(f, first + k * kThreads);
    float z[8], b[8];
    Raw8<T> raw = in[k].raw(at.c * 8 < f.cols);
    raw.get(z);
    if (bias.p) {
      load_param(bias, at.c * 8, f.cols, 0.f, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] += b[j];
    }
    if (ck_x.codes) {
      Raw8<float> exact;                  // before any rounding
      exact.put(z);
      put_chunk(ck_x, f, at, exact);
    }
#pragma unroll
    for (int j = 0; j < 8; j += 2) gelu<T, APPROX>(z[j], z[j + 1]);
    raw.put(z);
    store_flat<T, VEC>(y, ldy, f, at, raw);
    if (ck_y.codes) put_chunk(ck_y, f, at, raw);          // y as it is stored (zeros past the row's end: gelu(0) = 0)
  }
}

// ---- column kernels: a thread owns the 8 columns of a chunk and walks over rows; its sums stay in registers.  A block
// has 256 / lanes rows side by side, `lanes` (a power of two; not VEC: 32, a warp) chunks wide.  Rows are taken kAhead
// at a time, loads first.
template <bool VEC> constexpr int kAhead = VEC ? 4 : 2;      // (an unaligned chunk takes more registers on its way)
struct Columns {
  long long rows;
  int chunks, lanes_log2;
  float* partials;           // [gridDim.y][chunks * 8], or null
};

template <class Op>
__global__ void __launch_bounds__(kThreads) column_kernel(Op op, Columns g) {
  constexpr int kAhead = act8::kAhead<Op::kVec>;
  const int lanes = 1 << g.lanes_log2, side = kThreads >> g.lanes_log2;
  const int rl = threadIdx.x >> g.lanes_log2, lane = threadIdx.x & (lanes - 1);
  const int c = blockIdx.x * lanes + lane;
  float acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
  op.begin(c);
  const long long step = (long long)gridDim.y * side;
  for (long long r = (long long)blockIdx.y * side + rl; r < g.rows; r += step * kAhead) {
    typename Op::In in[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (r + k * step < g.rows) op.load(r + k * step, c, in[k]);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (r + k * step < g.rows) op.row(r + k * step, c, lane, in[k], acc);
  }
  if (!g.partials) return;
  __shared__ float sums[kThreads * 9];       // 9 floats apart: the threads of a column group spread over the banks
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[threadIdx.x * 9 + i] = acc[i];
  __syncthreads();
  const int width = g.chunks * 8;
  float* out = g.partials + (size_t)blockIdx.y * width;
  for (int j = threadIdx.x; j < lanes * 8; j += kThreads) {
    const int col = blockIdx.x * lanes * 8 + j;
    if (col >= width) continue;
    float s = 0.f;
    for (int k = 0; k < side; ++k) s += sums[(k * lanes + (j >> 3)) * 9 + (j & 7)];
    out[col] = s;
  }
}

template <typename T, bool VEC, int APPROX, bool CK>
struct GeluBackward {
  static constexpr bool kVec = VEC;
  Source<T> dy, x;
  ParamVec bias;
  Act8 ck;
  int cols, groups, scale_pitch;
  T* dx; long long lddx;
  float b[8];
  struct In {
    Chunk<T, VEC> dy, x;
    RawAct8 q;
  };
  __device__ __forceinline__ void begin(int c) {
    if (!CK) load_param(bias, c * 8, cols, 0.f, b);
  }
  __device__ __forceinline__ void load(long long r, int c, In& in) const {
    in.dy.fetch(dy, dy.p + r * dy.ld, c * 8, cols);
    if constexpr (CK)
      in.q.load(ck, r * groups * 32 + c * 8, r * scale_pitch + (c >> 2), c < groups * 4);
    else in.x.fetch(x, x.p + r * x.ld, c * 8, cols);
  }
  __device__ __forceinline__ void row(long long r, int c, int lane, const In& in, float (&acc)[8]) const {
    float g[8], z[8];
    in.dy.raw(c * 8 < cols).get(g);
    if constexpr (CK) {
      F2 v[4];
      in.q.get(v);
#pragma unroll
      for (int i = 0; i < 4; ++i) apart(v[i], &z[2 * i], &z[2 * i + 1]);
    } else {
      in.x.raw(c * 8 < cols).get(z);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] += b[i];
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const F2 d = mul2(two(g[i], g[i + 1]), gelu_slope<T, APPROX>(z[i], z[i + 1]));
      apart(d, &g[i], &g[i + 1]);
      apart(add2(d, two(acc[i], acc[i + 1])), &acc[i], &acc[i + 1]);
    }
    Raw8<T> o;
    o.put(g);
    store_chunk<T, VEC>(dx + r * lddx, c * 8, cols, o, true, c > 0 && lane > 0, lane < 31);
  }
};

}  // namespace act8

// A block adds 32 columns of one sum, a warp taking every kFinishWarps-th part; the warps' sums are added in order.
constexpr int kFinishWarps = 16;
__global__ void __launch_bounds__(32 * kFinishWarps) finish_columns_kernel(const float* __restrict__ partials, int parts,
                                                                           int sums, long long width, long long cols,
                                                                           void* out0, void* out1, int gbf16) {
  __shared__ float s[kFinishWarps][32];
  cudaGridDependencySynchronize();         // launched while the partial sums are still being written
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.y;
  const long long col = (long long)blockIdx.x * 32 + lane;
  void* out = k ? out1 : out0;
  if (!out) return;
  float v = 0.f;
  if (col < cols) {
    const float* p = partials + (size_t)k * width + col;
    const size_t step = (size_t)sums * width;
#pragma unroll 8
    for (int b = warp; b < parts; b += kFinishWarps) v += p[b * step];
  }
  s[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && col < cols) {
    v = 0.f;
#pragma unroll
    for (int j = 0; j < kFinishWarps; ++j) v += s[j][lane];
    if (gbf16) static_cast<bf16*>(out)[col] = __float2bfloat16_rn(v);
    else static_cast<float*>(out)[col] = v;
  }
}

cudaError_t launch_finish_columns(const float* partials, int parts, int sums, long long width, long long cols,
                                  void* out0, void* out1, int gdtype, cudaStream_t st) {
  const dim3 grid((unsigned)((cols + 31) / 32), sums);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(32 * kFinishWarps);
  cfg.stream = st;
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, finish_columns_kernel, partials, parts, sums, width, cols, out0, out1,
                            (int)(gdtype == FA_BF16));
}

// ---- host side
namespace {

// One launch per piece of at most 2^30 chunks (or one row, which has fewer than 2^28).
template <class Launch>
cudaError_t for_flat(long long rows, long long cols, Launch launch) {
  const long long groups = act8_groups(cols), per_row = groups * 4;
  const long long piece = (1LL << 30) / per_row;
  for (long long r0 = 0; r0 < rows; r0 += piece) {
    const long long n = rows - r0 < piece ? rows - r0 : piece;
    act8::Flat f{};
    f.n = static_cast<uint32_t>(n * per_row);
    f.cols = static_cast<int>(cols);
    f.groups = static_cast<int>(groups);
    f.scale_pitch = static_cast<int>(act8_scale_pitch(cols));
    f.per_row = FastDiv(static_cast<uint32_t>(per_row));
    const unsigned blocks = (f.n + act8::kThreads * act8::kPer - 1) / (act8::kThreads * act8::kPer);
    launch(blocks, f, r0);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <typename T>
cudaError_t store_t(Mat x, long long rows, long long cols, void* ck, cudaStream_t st) {
  const bool vec = mat_vec<T>(x, cols);
  return for_flat(rows, cols, [&](unsigned blocks, const act8::Flat& f, long long r0) {
    if (vec) act8::store_kernel<T, true><<<blocks, act8::kThreads, 0, st>>>(source_of<T>(x, r0, rows - r0, cols), act8_at(ck, rows, cols, r0), f);
    else act8::store_kernel<T, false><<<blocks, act8::kThreads, 0, st>>>(source_of<T>(x, r0, rows - r0, cols), act8_at(ck, rows, cols, r0), f);
  });
}
template <typename T>
cudaError_t load_t(const void* ck, long long rows, long long cols, Mat out, cudaStream_t st) {
  const bool vec = mat_vec<T>(out, cols);
  return for_flat(rows, cols, [&](unsigned blocks, const act8::Flat& f, long long r0) {
    if (vec) act8::load_kernel<T, true><<<blocks, act8::kThreads, 0, st>>>(act8_at(ck, rows, cols, r0), row_of<T>(out, r0), out.ld, f);
    else act8::load_kernel<T, false><<<blocks, act8::kThreads, 0, st>>>(act8_at(ck, rows, cols, r0), row_of<T>(out, r0), out.ld, f);
  });
}
template <typename T, bool VEC, int APPROX>
cudaError_t gelu_forward_t(Mat x, long long rows, long long cols, Param bias, Mat y, void* ck_x, void* ck_y,
                           cudaStream_t st) {
  const ParamVec b = param_vec(bias);
  return for_flat(rows, cols, [&](unsigned blocks, const act8::Flat& f, long long r0) {
    act8::gelu_forward_kernel<T, VEC, APPROX><<<blocks, act8::kThreads, 0, st>>>(
        source_of<T>(x, r0, rows - r0, cols), b, row_of<T>(y, r0), y.ld, act8_at(ck_x, rows, cols, r0),
        act8_at(ck_y, rows, cols, r0), f);
  });
}
template <typename T>
cudaError_t gelu_forward_d(Mat x, long long rows, long long cols, Param bias, int approx, Mat y, void* ck_x, void* ck_y,
                           cudaStream_t st) {
  const bool vec = mat_vec<T>(x, cols) && mat_vec<T>(y, cols);
  if (approx == kGeluTanh)
    return vec ? gelu_forward_t<T, true, kGeluTanh>(x, rows, cols, bias, y, ck_x, ck_y, st)
               : gelu_forward_t<T, false, kGeluTanh>(x, rows, cols, bias, y, ck_x, ck_y, st);
  return vec ? gelu_forward_t<T, true, kGeluErf>(x, rows, cols, bias, y, ck_x, ck_y, st)
             : gelu_forward_t<T, false, kGeluErf>(x, rows, cols, bias, y, ck_x, ck_y, st);
}

// Grid of a column kernel: sixteen blocks per SM, several times what is resident, so that the last ones to run leave
// little of the GPU idle; but at least eight rows for every thread as long as there are SMs to fill.
struct ColumnGrid {
  int lanes_log2;
  unsigned x, y;
  long long chunks;
};
ColumnGrid column_grid(bool vec, long long rows, long long cols) {
  ColumnGrid g{};
  const long long groups = act8_groups(cols);
  g.chunks = groups * 4;
  g.lanes_log2 = 5;
  while (vec && g.lanes_log2 > 2 && (1LL << (g.lanes_log2 - 1)) >= g.chunks) --g.lanes_log2;
  const long long lanes = 1LL << g.lanes_log2, side = act8::kThreads / lanes;
  const long long x = (g.chunks + lanes - 1) / lanes;
  const long long once = (2LL * sm_count() + x - 1) / x;
  long long y = (16LL * sm_count() + x - 1) / x;
  const long long full = (rows + side * 8 - 1) / (side * 8), most = (rows + side - 1) / side;
  if (y > full) y = full > once ? full : once;
  if (y > most) y = most;
  if (y < 1) y = 1;
  g.x = static_cast<unsigned>(x);
  g.y = static_cast<unsigned>(y);
  return g;
}

template <class Op>
cudaError_t run_columns(const Op& op, long long rows, long long cols, void* out, int gdtype, float* partials,
                        cudaStream_t st) {
  const ColumnGrid g = column_grid(Op::kVec, rows, cols);
  if (rows > 0) {
    act8::Columns p{};
    p.rows = rows;
    p.chunks = static_cast<int>(g.chunks);
    p.lanes_log2 = g.lanes_log2;
    p.partials = out ? partials : nullptr;
    act8::column_kernel<Op><<<dim3(g.x, g.y), act8::kThreads, 0, st>>>(op, p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!out) return cudaSuccess;
  return launch_finish_columns(partials, rows > 0 ? (int)g.y : 0, 1, g.chunks * 8, cols, out, nullptr, gdtype, st);
}

struct GeluBackwardArgs {
  Mat dy, x;
  Param bias;
  const void* ck;
  long long rows, cols;
  Mat dx;
  void* dbias;
  int gdtype;
  float* partials;
};
template <typename T, bool VEC, int APPROX, bool CK>
cudaError_t gelu_backward_t(const GeluBackwardArgs& a, cudaStream_t st) {
  act8::GeluBackward<T, VEC, APPROX, CK> op{};
  op.dy = source_of<T>(a.dy, 0, a.rows, a.cols);
  op.x = source_of<T>(a.x, 0, a.rows, a.cols);
  op.bias = param_vec(a.bias);
  op.ck = act8_at(a.ck, a.rows, a.cols, 0);
  op.cols = static_cast<int>(a.cols);
  op.groups = static_cast<int>(act8_groups(a.cols));
  op.scale_pitch = static_cast<int>(act8_scale_pitch(a.cols));
  op.dx = row_of<T>(a.dx, 0); op.lddx = a.dx.ld;
  return run_columns(op, a.rows, a.cols, a.dbias, a.gdtype, a.partials, st);
}
template <typename T, bool VEC>
cudaError_t gelu_backward_v(const GeluBackwardArgs& a, int approx, cudaStream_t st) {
  if (approx == kGeluTanh)
    return a.ck ? gelu_backward_t<T, VEC, kGeluTanh, true>(a, st) : gelu_backward_t<T, VEC, kGeluTanh, false>(a, st);
  return a.ck ? gelu_backward_t<T, VEC, kGeluErf, true>(a, st) : gelu_backward_t<T, VEC, kGeluErf, false>(a, st);
}
template <typename T>
cudaError_t gelu_backward_d(const GeluBackwardArgs& a, int approx, cudaStream_t st) {
  const bool vec = mat_vec<T>(a.dy, a.cols) && mat_vec<T>(a.x, a.cols) && mat_vec<T>(a.dx, a.cols);
  return vec ? gelu_backward_v<T, true>(a, approx, st) : gelu_backward_v<T, false>(a, approx, st);
}
}  // namespace

cudaError_t launch_act8_store(Mat x, int dtype, long long rows, long long cols, void* ck, cudaStream_t st) {
  return dtype == FA_BF16 ? store_t<bf16>(x, rows, cols, ck, st) : store_t<float>(x, rows, cols, ck, st);
}
cudaError_t launch_act8_load(const void* ck, long long rows, long long cols, Mat out, int dtype, cudaStream_t st) {
  return dtype == FA_BF16 ? load_t<bf16>(ck, rows, cols, out, st) : load_t<float>(ck, rows, cols, out, st);
}
cudaError_t launch_gelu_forward(Mat x, int dtype, long long rows, long long cols, Param bias, int approx, Mat y,
                                void* ck_x, void* ck_y, cudaStream_t st) {
  return dtype == FA_BF16 ? gelu_forward_d<bf16>(x, rows, cols, bias, approx, y, ck_x, ck_y, st)
                          : gelu_forward_d<float>(x, rows, cols, bias, approx, y, ck_x, ck_y, st);
}
size_t column_partials_bytes(long long rows, long long cols) {
  const ColumnGrid v = column_grid(true, rows, cols), e = column_grid(false, rows, cols);   // known at the call
  return (size_t)(v.y > e.y ? v.y : e.y) * v.chunks * 8 * sizeof(float);
}
cudaError_t launch_gelu_backward(Mat dy, Mat x, Param bias, const void* ck, int dtype, long long rows, long long cols,
                                 int approx, Mat dx, void* dbias, int gdtype, float* partials, cudaStream_t st) {
  const GeluBackwardArgs a{dy, x, bias, ck, rows, cols, dx, dbias, gdtype, partials};
  return dtype == FA_BF16 ? gelu_backward_d<bf16>(a, approx, st) : gelu_backward_d<float>(a, approx, st);
}
}  // namespace fa
