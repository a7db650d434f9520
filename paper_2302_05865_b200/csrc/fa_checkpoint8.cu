// 8-bit activation checkpoints and the element-wise operators around them: store, load, GELU forward
// (with checkpoints), and the column kernels: GELU backward (from a checkpoint) and column sums.
#include "../../include/fa.h"
#include "fa_columns.cuh"
#include "fa_train.h"

namespace fa {
namespace act8 {

constexpr int kThreads = 256;
constexpr int kPer = 4;              // chunks per thread, loaded before any is worked on

// A launch covers the chunks 0 .. n-1 of `rows` rows, `per_row` (a multiple of 4) chunks each; n < 2^31.
struct Flat {
  uint32_t n;
  int cols, groups, scale_pitch;
  FastDiv per_row;
};

__device__ __forceinline__ void split(const Flat& f, uint32_t i, uint32_t* row, int* c) {
  *row = f.per_row.div(i);
  *c = static_cast<int>(i - *row * f.per_row.d);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) store_kernel(const T* __restrict__ x, long long ldx, Act8 ck, Flat f) {
  const uint32_t first = blockIdx.x * (kThreads * kPer) + threadIdx.x;
  Raw8<T> raw[kPer];
  uint32_t row[kPer];
  int c[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const uint32_t i = first + k * kThreads;
    split(f, i < f.n ? i : 0u, &row[k], &c[k]);
    if (i < f.n) raw[k] = load_chunk<T, VEC>(x + row[k] * ldx, c[k], f.cols);
    else raw[k].zero();
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    float v[8];
    raw[k].get(v);
    act8_put(ck.codes + (size_t)row[k] * f.groups * 32, ck.scales + (size_t)row[k] * f.scale_pitch, c[k], f.groups, v,
             first + k * kThreads < f.n);
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) load_kernel(Act8 ck, T* __restrict__ out, long long ldo, Flat f) {
  const uint32_t first = blockIdx.x * (kThreads * kPer) + threadIdx.x;
  uint2 q[kPer];
  uint32_t byte[kPer], row[kPer];
  int c[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const uint32_t i = first + k * kThreads;
    split(f, i < f.n ? i : 0u, &row[k], &c[k]);
    if (i < f.n) {
      q[k] = *reinterpret_cast<const uint2*>(ck.codes + (size_t)row[k] * f.groups * 32 + (size_t)c[k] * 8);
      byte[k] = ck.scales[(size_t)row[k] * f.scale_pitch + (c[k] >> 2)];
    }
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (first + k * kThreads >= f.n) continue;
    float v[8];
    act8_decode(q[k], byte[k], v);
    store_chunk<T, VEC>(out + row[k] * ldo, c[k], f.cols, v);
  }
}

// tanh form: z (1 + tanh u) / 2 = z * S(2u) with the logistic function S, u = sqrt(2/pi) (z + 0.044715 z^3)
constexpr float kTwoU = 1.5957691216057308f;      // 2 sqrt(2/pi)
__device__ __forceinline__ float logistic(float t, float) { return 1.f / (1.f + expf(-t)); }
__device__ __forceinline__ float logistic(float t, bf16) { return __fdividef(1.f, 1.f + __expf(-t)); }

template <typename T, int APPROX>
__device__ __forceinline__ float gelu(float z) {
  if constexpr (APPROX == kGeluTanh) return z * logistic(kTwoU * (z + 0.044715f * z * z * z), T());
  else return z * normcdff(z);
}
template <typename T, int APPROX>
__device__ __forceinline__ float gelu_slope(float z) {
  if constexpr (APPROX == kGeluTanh) {
    const float z2 = z * z;
    const float s = logistic(kTwoU * (z + 0.044715f * z2 * z), T());
    const float t = s * (1.f - s);
    // far out t is zero while the other factors may overflow
    return t == 0.f ? s : s + z * t * (kTwoU * (1.f + 3.f * 0.044715f * z2));
  } else {
    const float e = expf(-0.5f * z * z) * 0.3989422804014327f;
    return e == 0.f ? normcdff(z) : normcdff(z) + z * e;
  }
}

template <typename T, bool VEC, int APPROX>
__global__ void __launch_bounds__(kThreads) gelu_forward_kernel(const T* __restrict__ x, long long ldx, ParamVec bias,
                                                                T* __restrict__ y, long long ldy, Act8 ck_x, Act8 ck_y,
                                                                Flat f) {
  const uint32_t first = blockIdx.x * (kThreads * kPer) + threadIdx.x;
  Raw8<T> raw[kPer];
  uint32_t row[kPer];
  int c[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const uint32_t i = first + k * kThreads;
    split(f, i < f.n ? i : 0u, &row[k], &c[k]);
    if (i < f.n) raw[k] = load_chunk<T, VEC>(x + row[k] * ldx, c[k], f.cols);
    else raw[k].zero();
  }
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const bool valid = first + k * kThreads < f.n;
    float z[8], b[8];
    raw[k].get(z);
    if (bias.p) {
      load_param(bias, c[k], f.cols, 0.f, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] += b[i];
    }
    if (ck_x.codes)
      act8_put(ck_x.codes + (size_t)row[k] * f.groups * 32, ck_x.scales + (size_t)row[k] * f.scale_pitch, c[k],
               f.groups, z, valid);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = gelu<T, APPROX>(z[i]);
    if (valid) store_chunk<T, VEC>(y + row[k] * ldy, c[k], f.cols, z);
    if (ck_y.codes) {
      round_to<T>(z);                     // the checkpoint holds y as it is stored
      act8_put(ck_y.codes + (size_t)row[k] * f.groups * 32, ck_y.scales + (size_t)row[k] * f.scale_pitch, c[k],
               f.groups, z, valid);
    }
  }
}

// ---- column kernels: a thread owns the 8 columns of one chunk and walks over rows; its sums stay in
// registers.  A block has 256 / lanes rows side by side, `lanes` (a power of two) chunks wide.
struct Columns {
  long long rows;
  int cols, chunks, lanes_log2;
  float* partials;           // [gridDim.y][chunks * 8], or null
};

template <class Op>
__global__ void __launch_bounds__(kThreads) column_kernel(Op op, Columns g) {
  const int lanes = 1 << g.lanes_log2, side = kThreads >> g.lanes_log2;
  const int rl = threadIdx.x >> g.lanes_log2;
  const int c = blockIdx.x * lanes + (threadIdx.x & (lanes - 1));
  float acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
  if (c < g.chunks) {
    op.begin(c);
    for (long long r = (long long)blockIdx.y * side + rl; r < g.rows; r += (long long)gridDim.y * side) op.row(r, c, acc);
  }
  if (!g.partials) return;
  __shared__ float sums[kThreads * 9];       // 9 floats apart: the threads of a column group spread over the banks
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[threadIdx.x * 9 + i] = acc[i];
  __syncthreads();
  for (int j = threadIdx.x; j < lanes * 8; j += kThreads) {
    const int cc = blockIdx.x * lanes + (j >> 3);
    if (cc >= g.chunks) continue;
    float s = 0.f;
    for (int k = 0; k < side; ++k) s += sums[(k * lanes + (j >> 3)) * 9 + (j & 7)];
    g.partials[(size_t)blockIdx.y * g.chunks * 8 + (size_t)cc * 8 + (j & 7)] = s;
  }
}

template <typename T, bool VEC, int APPROX>
struct GeluBackward {
  const T* dy; long long lddy;
  const T* x; long long ldx;
  ParamVec bias;
  Act8 ck;
  int cols, groups, scale_pitch;
  T* dx; long long lddx;
  float b[8];
  __device__ __forceinline__ void begin(int c) { load_param(bias, c, cols, 0.f, b); }
  __device__ __forceinline__ void row(long long r, int c, float (&acc)[8]) {
    float g[8], z[8];
    load_chunk<T, VEC>(dy + r * lddy, c, cols).get(g);
    if (ck.codes) {
      act8_decode(*reinterpret_cast<const uint2*>(ck.codes + (size_t)r * groups * 32 + (size_t)c * 8),
                  ck.scales[(size_t)r * scale_pitch + (c >> 2)], z);
    } else {
      load_chunk<T, VEC>(x + r * ldx, c, cols).get(z);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] += b[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g[i] *= gelu_slope<T, APPROX>(z[i]);
      acc[i] += g[i];
    }
    store_chunk<T, VEC>(dx + r * lddx, c, cols, g);
  }
};

template <typename T, bool VEC>
struct ColumnSum {
  const T* x; long long ldx;
  int cols;
  __device__ __forceinline__ void begin(int) {}
  __device__ __forceinline__ void row(long long r, int c, float (&acc)[8]) {
    float v[8];
    load_chunk<T, VEC>(x + r * ldx, c, cols).get(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] += v[i];
  }
};

}  // namespace act8

__global__ void __launch_bounds__(256) finish_columns_kernel(const float* __restrict__ partials, int parts, int sums,
                                                             long long width, long long cols, void* out0, void* out1,
                                                             int gbf16) {
  __shared__ float s[8][32];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const long long col = (long long)blockIdx.x * 32 + lane;
  for (int k = 0; k < sums; ++k) {
    void* out = k ? out1 : out0;
    if (!out) continue;
    float v = 0.f;
    if (col < cols) {
      const float* p = partials + (size_t)k * width + col;
#pragma unroll 8
      for (int b = slice; b < parts; b += 8) v += p[(size_t)b * sums * width];
    }
    s[slice][lane] = v;
    __syncthreads();
    if (slice == 0 && col < cols) {
      v = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) v += s[j][lane];
      if (gbf16) static_cast<bf16*>(out)[col] = __float2bfloat16_rn(v);
      else static_cast<float*>(out)[col] = v;
    }
    __syncthreads();
  }
}

cudaError_t launch_finish_columns(const float* partials, int parts, int sums, long long width, long long cols,
                                  void* out0, void* out1, int gdtype, cudaStream_t st) {
  const long long blocks = (cols + 31) / 32;
  finish_columns_kernel<<<(unsigned)blocks, 256, 0, st>>>(partials, parts, sums, width, cols, out0, out1,
                                                          gdtype == FA_BF16);
  return cudaGetLastError();
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
    if (vec) act8::store_kernel<T, true><<<blocks, act8::kThreads, 0, st>>>(row_of<T>(x, r0), x.ld, act8_at(ck, rows, cols, r0), f);
    else act8::store_kernel<T, false><<<blocks, act8::kThreads, 0, st>>>(row_of<T>(x, r0), x.ld, act8_at(ck, rows, cols, r0), f);
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
  const ParamVec b = param_vec(bias, cols);
  return for_flat(rows, cols, [&](unsigned blocks, const act8::Flat& f, long long r0) {
    act8::gelu_forward_kernel<T, VEC, APPROX><<<blocks, act8::kThreads, 0, st>>>(
        row_of<T>(x, r0), x.ld, b, row_of<T>(y, r0), y.ld, act8_at(ck_x, rows, cols, r0),
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

// Grid of a column kernel: about four blocks per SM in all, no block without rows.
struct ColumnGrid {
  int lanes_log2;
  unsigned x, y;
  long long chunks;
};
ColumnGrid column_grid(long long rows, long long cols) {
  ColumnGrid g{};
  g.chunks = act8_groups(cols) * 4;
  g.lanes_log2 = 5;
  while (g.lanes_log2 > 2 && (1LL << (g.lanes_log2 - 1)) >= g.chunks) --g.lanes_log2;
  const long long lanes = 1LL << g.lanes_log2, side = act8::kThreads / lanes;
  const long long x = (g.chunks + lanes - 1) / lanes;
  long long y = (4LL * sm_count() + x - 1) / x;
  const long long most = (rows + side - 1) / side;
  if (y > most) y = most;
  if (y < 1) y = 1;
  g.x = static_cast<unsigned>(x);
  g.y = static_cast<unsigned>(y);
  return g;
}

template <class Op>
cudaError_t run_columns(const Op& op, long long rows, long long cols, void* out, int gdtype, float* partials,
                        cudaStream_t st) {
  const ColumnGrid g = column_grid(rows, cols);
  if (rows > 0) {
    act8::Columns p{};
    p.rows = rows;
    p.cols = static_cast<int>(cols);
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

template <typename T, bool VEC, int APPROX>
cudaError_t gelu_backward_t(Mat dy, Mat x, Param bias, const void* ck, long long rows, long long cols, Mat dx,
                            void* dbias, int gdtype, float* partials, cudaStream_t st) {
  act8::GeluBackward<T, VEC, APPROX> op{};
  op.dy = row_of<T>(dy, 0); op.lddy = dy.ld;
  op.x = row_of<T>(x, 0); op.ldx = x.ld;
  op.bias = param_vec(bias, cols);
  op.ck = act8_at(ck, rows, cols, 0);
  op.cols = static_cast<int>(cols);
  op.groups = static_cast<int>(act8_groups(cols));
  op.scale_pitch = static_cast<int>(act8_scale_pitch(cols));
  op.dx = row_of<T>(dx, 0); op.lddx = dx.ld;
  return run_columns(op, rows, cols, dbias, gdtype, partials, st);
}
template <typename T>
cudaError_t gelu_backward_d(Mat dy, Mat x, Param bias, const void* ck, long long rows, long long cols, int approx,
                            Mat dx, void* dbias, int gdtype, float* partials, cudaStream_t st) {
  const bool vec = mat_vec<T>(dy, cols) && mat_vec<T>(x, cols) && mat_vec<T>(dx, cols);
  if (approx == kGeluTanh)
    return vec ? gelu_backward_t<T, true, kGeluTanh>(dy, x, bias, ck, rows, cols, dx, dbias, gdtype, partials, st)
               : gelu_backward_t<T, false, kGeluTanh>(dy, x, bias, ck, rows, cols, dx, dbias, gdtype, partials, st);
  return vec ? gelu_backward_t<T, true, kGeluErf>(dy, x, bias, ck, rows, cols, dx, dbias, gdtype, partials, st)
             : gelu_backward_t<T, false, kGeluErf>(dy, x, bias, ck, rows, cols, dx, dbias, gdtype, partials, st);
}
template <typename T>
cudaError_t column_sum_d(Mat x, long long rows, long long cols, void* out, int gdtype, float* partials,
                         cudaStream_t st) {
  if (mat_vec<T>(x, cols)) {
    act8::ColumnSum<T, true> op{row_of<T>(x, 0), x.ld, static_cast<int>(cols)};
    return run_columns(op, rows, cols, out, gdtype, partials, st);
  }
  act8::ColumnSum<T, false> op{row_of<T>(x, 0), x.ld, static_cast<int>(cols)};
  return run_columns(op, rows, cols, out, gdtype, partials, st);
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
  const ColumnGrid g = column_grid(rows, cols);
  return (size_t)g.y * g.chunks * 8 * sizeof(float);
}
cudaError_t launch_gelu_backward(Mat dy, Mat x, Param bias, const void* ck, int dtype, long long rows, long long cols,
                                 int approx, Mat dx, void* dbias, int gdtype, float* partials, cudaStream_t st) {
  return dtype == FA_BF16
             ? gelu_backward_d<bf16>(dy, x, bias, ck, rows, cols, approx, dx, dbias, gdtype, partials, st)
             : gelu_backward_d<float>(dy, x, bias, ck, rows, cols, approx, dx, dbias, gdtype, partials, st);
}
cudaError_t launch_column_sum(Mat x, int dtype, long long rows, long long cols, void* out, int gdtype, float* partials,
                              cudaStream_t st) {
  return dtype == FA_BF16 ? column_sum_d<bf16>(x, rows, cols, out, gdtype, partials, st)
                          : column_sum_d<float>(x, rows, cols, out, gdtype, partials, st);
}

}  // namespace fa
