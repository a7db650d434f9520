// Layer norm over the rows of a matrix, forward and backward.
//   forward : s = x + r, mean and rstd = 1 / sqrt(mean((s - mean)^2) + eps) of a row, y = (s - mean) rstd w + b
//   backward: h = (s - mean) rstd, g = dy w;  dx = rstd (g - mean(g) - h mean(g h)) + dr,
//             dw = column sums of dy h, db = column sums of dy
// A team of threads holds a row in registers, `K` chunks of 8 values per thread (chunk t + k * team), so
// the variance is formed from centred values and nothing is read twice.  Rows of more than
// kMaxThreads * kMaxK chunks go through the `long` kernels, which read a row several times.
#include "../../include/fa.h"
#include "fa_columns.cuh"
#include "fa_train.h"

namespace fa {
namespace ln {

constexpr int kMaxK = 4;
constexpr int kMaxThreads = 512;                  // 128 registers a thread
constexpr long long kMaxChunks = (long long)kMaxThreads * kMaxK;

struct Shape {
  long long rows;
  int cols, chunks, groups, scale_pitch;
  int team;            // threads per row: a power of two up to 32, or a multiple of 32
  float n;               // cols: means are quotients, so a constant row has its own value as the mean
};

// Sums of N values over the team.  Teams wider than a warp are the whole block; `buf` has two sets of
// kMaxThreads/32 slots per value, used in turn (`phase`), so that one barrier per call is enough.
template <int N>
__device__ __forceinline__ void team_sum(float (&v)[N], int team, float* buf, int* phase) {
  const int top = team < 32 ? team : 32;
  for (int o = top >> 1; o > 0; o >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  }
  if (team <= 32) return;
  constexpr int kWarps = kMaxThreads / 32;
  float* b = buf + *phase * N * kWarps;
  *phase ^= 1;
  const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) b[i * kWarps + warp] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float s = 0.f;
    for (int w = 0; w < warps; ++w) s += b[i * kWarps + w];
    v[i] = s;
  }
}

template <typename T>
struct Forward {
  const T* x; long long ldx;
  const T* residual; long long ldr;
  ParamVec weight, bias;
  float eps;
  T* y; long long ldy;
  T* sum_out; long long lds;
  float* mean;
  float* rstd;
  Act8 ck_sum, ck_y;
};

template <typename T, bool VEC, int K>
__global__ void __launch_bounds__(kMaxThreads) forward_kernel(Forward<T> a, Shape s) {
  __shared__ float buf[2 * kMaxThreads / 32];
  int phase = 0;
  const int teams = blockDim.x / s.team, t = threadIdx.x % s.team, mine = threadIdx.x / s.team;
  const long long stride = (long long)gridDim.x * teams;
  const long long turns = (s.rows + stride - 1) / stride;       // the same for every thread: all take part in the sums
  for (long long i = 0; i < turns; ++i) {
    const long long r = i * stride + (long long)blockIdx.x * teams + mine;
    const bool live = r < s.rows;
    float v[K][8];
    float sum[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = t + k * s.team;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[k][j] = 0.f;
      if (live && c < s.chunks) {
        load_chunk<T, VEC>(a.x + r * a.ldx, c, s.cols).get(v[k]);
        if (a.residual) {
          float u[8];
          load_chunk<T, VEC>(a.residual + r * a.ldr, c, s.cols).get(u);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[k][j] += u[j];
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] += v[k][j];
    }
    team_sum(sum, s.team, buf, &phase);
    const float mean = sum[0] / s.n;
    sum[0] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int left = s.cols - (t + k * s.team) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = j < left ? v[k][j] - mean : 0.f;
        sum[0] = fmaf(d, d, sum[0]);
      }
    }
    team_sum(sum, s.team, buf, &phase);
    const float rstd = 1.f / sqrtf(sum[0] / s.n + a.eps);
    if (live && t == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = t + k * s.team;
      const bool valid = live && c < s.chunks;
      float w[8], b[8], y[8];
      load_param(a.weight, c, s.cols, 1.f, w);
      load_param(a.bias, c, s.cols, 0.f, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = fmaf((v[k][j] - mean) * rstd, w[j], b[j]);
      if (valid) {
        if (a.sum_out) store_chunk<T, VEC>(a.sum_out + r * a.lds, c, s.cols, v[k]);
        store_chunk<T, VEC>(a.y + r * a.ldy, c, s.cols, y);
      }
      const size_t code_row = (size_t)(live ? r : 0) * s.groups * 32, scale_row = (size_t)(live ? r : 0) * s.scale_pitch;
      if (a.ck_sum.codes) {               // checkpoints hold the values as they are stored
        round_to<T>(v[k]);
        act8_put(a.ck_sum.codes + code_row, a.ck_sum.scales + scale_row, c, s.groups, v[k], valid);
      }
      if (a.ck_y.codes) {
        round_to<T>(y);
        const int left = s.cols - c * 8;  // past the row's end the formula gives (0 - mean) rstd
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = j < left ? y[j] : 0.f;
        act8_put(a.ck_y.codes + code_row, a.ck_y.scales + scale_row, c, s.groups, y, valid);
      }
    }
  }
}

// Rows of any length: one block per row, three reads.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kMaxThreads) forward_long_kernel(Forward<T> a, Shape s) {
  __shared__ float buf[2 * kMaxThreads / 32];
  int phase = 0;
  const int turns = (s.chunks + kMaxThreads - 1) / kMaxThreads;
  for (long long r = blockIdx.x; r < s.rows; r += gridDim.x) {
    auto value = [&](int c, float (&v)[8]) {
      load_chunk<T, VEC>(a.x + r * a.ldx, c, s.cols).get(v);
      if (a.residual) {
        float u[8];
        load_chunk<T, VEC>(a.residual + r * a.ldr, c, s.cols).get(u);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += u[j];
      }
    };
    float sum[1] = {0.f};
    for (int c = threadIdx.x; c < s.chunks; c += kMaxThreads) {
      float v[8];
      value(c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] += v[j];
    }
    team_sum(sum, kMaxThreads, buf, &phase);
    const float mean = sum[0] / s.n;
    sum[0] = 0.f;
    for (int c = threadIdx.x; c < s.chunks; c += kMaxThreads) {
      float v[8];
      value(c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = c * 8 + j < s.cols ? v[j] - mean : 0.f;
        sum[0] = fmaf(d, d, sum[0]);
      }
    }
    team_sum(sum, kMaxThreads, buf, &phase);
    const float rstd = 1.f / sqrtf(sum[0] / s.n + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    for (int i = 0; i < turns; ++i) {
      const int c = threadIdx.x + i * kMaxThreads;
      const bool valid = c < s.chunks;
      float v[8], w[8], b[8], y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.f;
      if (valid) value(c, v);
      load_param(a.weight, c, s.cols, 1.f, w);
      load_param(a.bias, c, s.cols, 0.f, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = c * 8 + j < s.cols ? fmaf((v[j] - mean) * rstd, w[j], b[j]) : 0.f;
      if (valid) {
        if (a.sum_out) store_chunk<T, VEC>(a.sum_out + r * a.lds, c, s.cols, v);
        store_chunk<T, VEC>(a.y + r * a.ldy, c, s.cols, y);
      }
      const size_t code_row = (size_t)r * s.groups * 32, scale_row = (size_t)r * s.scale_pitch;
      if (a.ck_sum.codes) {
        round_to<T>(v);
        act8_put(a.ck_sum.codes + code_row, a.ck_sum.scales + scale_row, c, s.groups, v, valid);
      }
      if (a.ck_y.codes) {
        round_to<T>(y);
        act8_put(a.ck_y.codes + code_row, a.ck_y.scales + scale_row, c, s.groups, y, valid);
      }
    }
  }
}

template <typename T>
struct Backward {
  const T* dy; long long lddy;
  const T* x; long long ldx;          // null: read the checkpoint
  Act8 ck;
  ParamVec weight;
  const float* mean;
  const float* rstd;
  const T* residual; long long ldr;
  T* dx; long long lddx;
  float* partials;                    // [gridDim.x][2][chunks * 8], or null
};

// Values of chunk c of row r of the normalised input; zeros past the row's end.
template <typename T, bool VEC>
__device__ __forceinline__ void input_chunk(const Backward<T>& a, const Shape& s, long long r, int c, float (&v)[8]) {
  if (a.x) {
    load_chunk<T, VEC>(a.x + r * a.ldx, c, s.cols).get(v);
  } else {
    act8_decode(*reinterpret_cast<const uint2*>(a.ck.codes + (size_t)r * s.groups * 32 + (size_t)c * 8),
                a.ck.scales[(size_t)r * s.scale_pitch + (c >> 2)], v);
  }
}

// Persistent: a team walks over rows, its share of the column sums stays in registers.
template <typename T, bool VEC, int K>
__global__ void __launch_bounds__(kMaxThreads) backward_kernel(Backward<T> a, Shape s) {
  extern __shared__ float dyn[];             // [teams - 1][chunks * 8]: column sums of the block's other teams
  __shared__ float buf[2 * 2 * kMaxThreads / 32];
  int phase = 0;
  const int teams = blockDim.x / s.team, t = threadIdx.x % s.team, mine = threadIdx.x / s.team;
  const long long stride = (long long)gridDim.x * teams;
  const long long turns = (s.rows + stride - 1) / stride;
  float dw[K][8], db[K][8];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[k][j] = db[k][j] = 0.f;
  for (long long i = 0; i < turns; ++i) {
    const long long r = i * stride + (long long)blockIdx.x * teams + mine;
    const bool live = r < s.rows;
    const float mean = live ? a.mean[r] : 0.f, rstd = live ? a.rstd[r] : 0.f;
    Raw8<T> dyr[K];
    float h[K][8];
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = t + k * s.team;
      dyr[k].zero();
#pragma unroll
      for (int j = 0; j < 8; ++j) h[k][j] = 0.f;
      if (live && c < s.chunks) {
        dyr[k] = load_chunk<T, VEC>(a.dy + r * a.lddy, c, s.cols);
        input_chunk<T, VEC>(a, s, r, c, h[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = t + k * s.team, left = live ? s.cols - c * 8 : 0;
      float w[8], dy[8];
      load_param(a.weight, c, s.cols, 1.f, w);
      dyr[k].get(dy);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        h[k][j] = j < left ? (h[k][j] - mean) * rstd : 0.f;
        const float g = dy[j] * w[j];
        sum[0] += g;
        sum[1] = fmaf(g, h[k][j], sum[1]);
        dw[k][j] = fmaf(dy[j], h[k][j], dw[k][j]);
        db[k][j] += dy[j];
      }
    }
    team_sum(sum, s.team, buf, &phase);
    const float mg = sum[0] / s.n, mgh = sum[1] / s.n;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = t + k * s.team;
      if (!live || c >= s.chunks) continue;
      float w[8], dy[8], o[8];
      load_param(a.weight, c, s.cols, 1.f, w);
      dyr[k].get(dy);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = rstd * (dy[j] * w[j] - mg - h[k][j] * mgh);
      if (a.residual) {
        float u[8];
        load_chunk<T, VEC>(a.residual + r * a.ldr, c, s.cols).get(u);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] += u[j];
      }
      store_chunk<T, VEC>(a.dx + r * a.lddx, c, s.cols, o);
    }
  }
  if (!a.partials) return;
  const int width = s.chunks * 8;
  float* out = a.partials + (size_t)blockIdx.x * 2 * width;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (teams > 1) {
      __syncthreads();
      if (mine > 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
          const int c = t + k * s.team;
          if (c < s.chunks) {
#pragma unroll
            for (int j = 0; j < 8; ++j) dyn[(mine - 1) * width + j * s.chunks + c] = half ? db[k][j] : dw[k][j];
          }
        }
      }
      __syncthreads();
    }
    if (mine == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = t + k * s.team;
        if (c >= s.chunks) continue;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] = half ? db[k][j] : dw[k][j];
          for (int q = 0; q < teams - 1; ++q) v[j] += dyn[q * width + j * s.chunks + c];
        }
        Raw8<float> o;
        o.put(v);
        o.store(out + half * width + c * 8);
      }
    }
  }
}

// Long rows, first step: mean(g) and mean(g h) of every row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kMaxThreads) backward_stats_kernel(Backward<T> a, Shape s, float* stats) {
  __shared__ float buf[2 * 2 * kMaxThreads / 32];
  int phase = 0;
  for (long long r = blockIdx.x; r < s.rows; r += gridDim.x) {
    const float mean = a.mean[r], rstd = a.rstd[r];
    float sum[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < s.chunks; c += kMaxThreads) {
      float dy[8], v[8], w[8];
      load_chunk<T, VEC>(a.dy + r * a.lddy, c, s.cols).get(dy);
      input_chunk<T, VEC>(a, s, r, c, v);
      load_param(a.weight, c, s.cols, 1.f, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float g = dy[j] * w[j];
        sum[0] += g;
        sum[1] = fmaf(g, c * 8 + j < s.cols ? (v[j] - mean) * rstd : 0.f, sum[1]);
      }
    }
    team_sum(sum, kMaxThreads, buf, &phase);
    if (threadIdx.x == 0) {
      stats[2 * r] = sum[0] / s.n;
      stats[2 * r + 1] = sum[1] / s.n;
    }
  }
}

// Second step: a block owns 32 chunks of columns and a share of the rows.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) backward_long_kernel(Backward<T> a, Shape s, const float* stats) {
  __shared__ float part[8][32 * 8 + 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.y * 32 + lane;
  float dw[8], db[8], w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) dw[j] = db[j] = 0.f;
  load_param(a.weight, c, s.cols, 1.f, w);
  if (c < s.chunks) {
    for (long long r = (long long)blockIdx.x * 8 + warp; r < s.rows; r += (long long)gridDim.x * 8) {
      const float mean = a.mean[r], rstd = a.rstd[r], mg = stats[2 * r], mgh = stats[2 * r + 1];
      float dy[8], v[8], o[8];
      load_chunk<T, VEC>(a.dy + r * a.lddy, c, s.cols).get(dy);
      input_chunk<T, VEC>(a, s, r, c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float h = c * 8 + j < s.cols ? (v[j] - mean) * rstd : 0.f;
        o[j] = rstd * (dy[j] * w[j] - mg - h * mgh);
        dw[j] = fmaf(dy[j], h, dw[j]);
        db[j] += dy[j];
      }
      if (a.residual) {
        load_chunk<T, VEC>(a.residual + r * a.ldr, c, s.cols).get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] += v[j];
      }
      store_chunk<T, VEC>(a.dx + r * a.lddx, c, s.cols, o);
    }
  }
  if (!a.partials) return;
  float* out = a.partials + (size_t)blockIdx.x * 2 * s.chunks * 8;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int j = 0; j < 8; ++j) part[warp][j * 33 + lane] = half ? db[j] : dw[j];
    __syncthreads();
    const int j = threadIdx.x & 7, l = threadIdx.x >> 3, cc = blockIdx.y * 32 + l;
    if (cc < s.chunks) {
      float v = 0.f;
      for (int q = 0; q < 8; ++q) v += part[q][j * 33 + l];
      out[(size_t)half * s.chunks * 8 + (size_t)cc * 8 + j] = v;
    }
    __syncthreads();
  }
}

}  // namespace ln

namespace {

ln::Shape ln_shape(long long rows, long long cols) {
  ln::Shape s{};
  s.rows = rows;
  s.cols = static_cast<int>(cols);
  s.groups = static_cast<int>(act8_groups(cols));
  s.chunks = s.groups * 4;
  s.scale_pitch = static_cast<int>(act8_scale_pitch(cols));
  s.n = static_cast<float>(cols);
  return s;
}

// Threads per row and chunks per thread, for rows that fit in registers.
void ln_team(ln::Shape* s, int* K) {
  if (s->chunks <= 32) {
    int t = 4;
    while (t < s->chunks) t *= 2;
    s->team = t;
    *K = 1;
  } else if (s->chunks <= 32 * ln::kMaxK) {
    s->team = 32;
    *K = (s->chunks + 31) / 32;
  } else {
    *K = ln::kMaxK;
    s->team = (s->chunks + 32 * ln::kMaxK - 1) / (32 * ln::kMaxK) * 32;
  }
}

template <typename T>
cudaError_t ln_forward_t(const ln::Forward<T>& a, bool vec, long long rows, long long cols, cudaStream_t st) {
  ln::Shape s = ln_shape(rows, cols);
  if (s.chunks > ln::kMaxChunks) {
    s.team = ln::kMaxThreads;
    const unsigned grid = static_cast<unsigned>(rows < (1 << 30) ? rows : 1 << 30);
    if (vec) ln::forward_long_kernel<T, true><<<grid, ln::kMaxThreads, 0, st>>>(a, s);
    else ln::forward_long_kernel<T, false><<<grid, ln::kMaxThreads, 0, st>>>(a, s);
    return cudaGetLastError();
  }
  int K = 1;
  ln_team(&s, &K);
  const int threads = s.team <= 32 ? 128 : s.team, teams = threads / s.team;
  const long long want = (rows + teams - 1) / teams;
  const unsigned grid = static_cast<unsigned>(want < (1 << 30) ? want : 1 << 30);
  auto go = [&](auto kernel) { kernel<<<grid, threads, 0, st>>>(a, s); };
  if (vec) {
    if (K == 1) go(ln::forward_kernel<T, true, 1>);
    else if (K == 2) go(ln::forward_kernel<T, true, 2>);
    else if (K == 3) go(ln::forward_kernel<T, true, 3>);
    else go(ln::forward_kernel<T, true, 4>);
  } else {
    if (K == 1) go(ln::forward_kernel<T, false, 1>);
    else if (K == 2) go(ln::forward_kernel<T, false, 2>);
    else if (K == 3) go(ln::forward_kernel<T, false, 3>);
    else go(ln::forward_kernel<T, false, 4>);
  }
  return cudaGetLastError();
}

template <typename T>
cudaError_t ln_forward_d(Mat x, Mat residual, long long rows, long long cols, Param weight, Param bias, float eps,
                         Mat y, Mat sum_out, float* mean, float* rstd, void* ck_sum, void* ck_y, cudaStream_t st) {
  if (rows == 0) return cudaSuccess;
  ln::Forward<T> a{};
  a.x = row_of<T>(x, 0); a.ldx = x.ld;
  a.residual = row_of<T>(residual, 0); a.ldr = residual.ld;
  a.weight = param_vec(weight, cols); a.bias = param_vec(bias, cols);
  a.eps = eps;
  a.y = row_of<T>(y, 0); a.ldy = y.ld;
  a.sum_out = row_of<T>(sum_out, 0); a.lds = sum_out.ld;
  a.mean = mean; a.rstd = rstd;
  a.ck_sum = act8_at(ck_sum, rows, cols, 0); a.ck_y = act8_at(ck_y, rows, cols, 0);
  const bool vec = mat_vec<T>(x, cols) && mat_vec<T>(residual, cols) && mat_vec<T>(y, cols) && mat_vec<T>(sum_out, cols);
  return ln_forward_t<T>(a, vec, rows, cols, st);
}

// Blocks of the backward kernels: what is resident at once, as far as there are rows.
struct LnBackwardGrid {
  ln::Shape s;
  int K, threads, teams;
  unsigned grid;
  bool is_long;
};
LnBackwardGrid ln_backward_grid(long long rows, long long cols) {
  LnBackwardGrid g{};
  g.s = ln_shape(rows, cols);
  g.is_long = g.s.chunks > ln::kMaxChunks;
  long long want;
  if (g.is_long) {
    const long long tiles = (g.s.chunks + 31) / 32;
    g.threads = 256; g.teams = 8; g.K = 1;
    want = (4LL * sm_count() + tiles - 1) / tiles;
  } else {
    ln_team(&g.s, &g.K);
    g.threads = g.s.team <= 32 ? 256 : g.s.team;
    g.teams = g.threads / g.s.team;
    want = (long long)sm_count() * (g.threads <= 256 ? 512 / g.threads : 1);
  }
  const long long most = (rows + g.teams - 1) / g.teams;
  if (want > most) want = most;
  g.grid = static_cast<unsigned>(want < 1 ? 1 : want);
  return g;
}

template <typename T>
cudaError_t ln_backward_d(Mat dy, Mat x, const void* ck, long long rows, long long cols, Param weight,
                          const float* mean, const float* rstd, Mat residual, Mat dx, void* dweight, void* dbias,
                          int gdtype, float* partials, float* row_stats, cudaStream_t st) {
  const LnBackwardGrid g = ln_backward_grid(rows, cols);
  const bool sums = dweight || dbias;
  if (rows > 0) {
    ln::Backward<T> a{};
    a.dy = row_of<T>(dy, 0); a.lddy = dy.ld;
    a.x = row_of<T>(x, 0); a.ldx = x.ld;
    a.ck = act8_at(ck, rows, cols, 0);
    a.weight = param_vec(weight, cols);
    a.mean = mean; a.rstd = rstd;
    a.residual = row_of<T>(residual, 0); a.ldr = residual.ld;
    a.dx = row_of<T>(dx, 0); a.lddx = dx.ld;
    a.partials = sums ? partials : nullptr;
    const bool vec = mat_vec<T>(dy, cols) && mat_vec<T>(x, cols) && mat_vec<T>(residual, cols) && mat_vec<T>(dx, cols);
    cudaError_t e = cudaSuccess;
    if (g.is_long) {
      const unsigned row_grid = static_cast<unsigned>(rows < (1 << 30) ? rows : 1 << 30);
      const dim3 grid(g.grid, (g.s.chunks + 31) / 32);
      if (vec) {
        ln::backward_stats_kernel<T, true><<<row_grid, ln::kMaxThreads, 0, st>>>(a, g.s, row_stats);
        ln::backward_long_kernel<T, true><<<grid, 256, 0, st>>>(a, g.s, row_stats);
      } else {
        ln::backward_stats_kernel<T, false><<<row_grid, ln::kMaxThreads, 0, st>>>(a, g.s, row_stats);
        ln::backward_long_kernel<T, false><<<grid, 256, 0, st>>>(a, g.s, row_stats);
      }
    } else {
      const size_t smem = (size_t)(g.teams - 1) * g.s.chunks * 8 * sizeof(float);
      auto go = [&](auto kernel) { kernel<<<g.grid, g.threads, smem, st>>>(a, g.s); };
      if (vec) {
        if (g.K == 1) go(ln::backward_kernel<T, true, 1>);
        else if (g.K == 2) go(ln::backward_kernel<T, true, 2>);
        else if (g.K == 3) go(ln::backward_kernel<T, true, 3>);
        else go(ln::backward_kernel<T, true, 4>);
      } else {
        if (g.K == 1) go(ln::backward_kernel<T, false, 1>);
        else if (g.K == 2) go(ln::backward_kernel<T, false, 2>);
        else if (g.K == 3) go(ln::backward_kernel<T, false, 3>);
        else go(ln::backward_kernel<T, false, 4>);
      }
    }
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!sums) return cudaSuccess;
  return launch_finish_columns(partials, rows > 0 ? (int)g.grid : 0, 2, (long long)g.s.chunks * 8, cols, dweight, dbias,
                               gdtype, st);
}

}  // namespace

size_t layer_norm_partials_bytes(long long rows, long long cols) {
  const LnBackwardGrid g = ln_backward_grid(rows, cols);
  return (size_t)g.grid * 2 * g.s.chunks * 8 * sizeof(float);
}
bool layer_norm_needs_row_stats(long long cols) { return act8_groups(cols) * 4 > ln::kMaxChunks; }

cudaError_t launch_layer_norm_forward(Mat x, Mat residual, int dtype, long long rows, long long cols, Param weight,
                                      Param bias, float eps, Mat y, Mat sum_out, float* mean, float* rstd, void* ck_sum,
                                      void* ck_y, cudaStream_t st) {
  return dtype == FA_BF16
             ? ln_forward_d<bf16>(x, residual, rows, cols, weight, bias, eps, y, sum_out, mean, rstd, ck_sum, ck_y, st)
             : ln_forward_d<float>(x, residual, rows, cols, weight, bias, eps, y, sum_out, mean, rstd, ck_sum, ck_y, st);
}

cudaError_t launch_layer_norm_backward(Mat dy, Mat x, const void* ck, int dtype, long long rows, long long cols,
                                       Param weight, const float* mean, const float* rstd, Mat residual_grad, Mat dx,
                                       void* dweight, void* dbias, int gdtype, float* partials, float* row_stats,
                                       cudaStream_t st) {
  return dtype == FA_BF16 ? ln_backward_d<bf16>(dy, x, ck, rows, cols, weight, mean, rstd, residual_grad, dx, dweight,
                                                dbias, gdtype, partials, row_stats, st)
                          : ln_backward_d<float>(dy, x, ck, rows, cols, weight, mean, rstd, residual_grad, dx, dweight,
                                                 dbias, gdtype, partials, row_stats, st);
}

}  // namespace fa
