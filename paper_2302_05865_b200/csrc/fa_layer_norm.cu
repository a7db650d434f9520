// Layer norm over the rows of a matrix, forward and backward.
//   forward : s = x + r, mean and rstd = 1 / sqrt(mean((s - mean)^2) + eps) of a row, y = (s - mean) rstd w + b
//   backward: h = (s - mean) rstd, g = dy w;  dx = rstd (g - mean(g) - h mean(g h)) + dr,
//             dw = column sums of dy h, db = column sums of dy
// A team of threads holds a row in registers, `K` chunks of 8 values per thread, so the variance is formed from
// centred values and nothing is read twice; the next row's loads are issued before the current row's sums, which
// are what a row waits for.  One block per SM walks over the rows; the backward pass keeps its share of the column sums
// in registers.  Rows that do not fit (more than 16384 columns forward, 8192 backward) go through the `long` kernels,
// which read a row several times.
// Memory is the floor; what holds the kernels above it is the number of instructions a row takes besides its values
// (sums across lanes and warps, the scales of checkpoints): measured on bf16, 16384 rows of 4096, among other calls,
//   forward with residual, sum and two checkpoints 137 us (0.76 of a copy's rate; 44 instructions a value, 63 % of the
//   issue slots), backward from a checkpoint with residual gradient and column sums 109 us (0.66; 33 a value),
// and of 768: 31 and 31 us (0.63, 0.43); fp32 rows of 4096 196 and 162 us (0.95, 0.83).  Unaligned rows of 4001, whose
// shifts are instructions as well: bf16 300 and 290 us, fp32 368 and 340; rows of the `long` kernels (2048 x 20000 bf16,
// three reads) 144 and 142 us (0.44, 0.31).  More chunks a thread spread those instructions over more values, fewer leave
// registers for more warps: four (three) chunks are best in the forward pass (768 columns: 33 us, with one 41), one
// (bf16 up to 1024 columns, fp32 up to 4096) or two, with two sums a column to keep, in the backward pass.
#include "../../include/fa.h"
#include "fa_columns.cuh"
#include "fa_train.h"

namespace fa {
namespace ln {

constexpr int kBlock = 512;             // most threads per row and block
// One block per SM, as many threads as their registers allow: its teams' column sums are added in shared memory, so
// that there are as few partial sums as SMs.
template <int K> constexpr int kForwardThreads = K == 1 ? 768 : kBlock;
template <typename T, int K> constexpr int kBackwardThreads = K == 1 && sizeof(T) == 2 ? 768 : kBlock;
constexpr int kMaxKForward = 4, kMaxKBackward = 2;

struct Shape {
  long long rows;
  int cols, groups, scale_pitch;
  int width;           // groups * 32
  int team;            // threads per row: a power of two up to 32 (not VEC: 32), or a multiple of 32
  float n, inv;        // cols and its reciprocal
};

constexpr int kSlots = 16;              // warps of the widest team
constexpr int kMaxTeams = 768 / 32;
// Room for the sums of the warps of a team, two sets used in turn so that one barrier per call is enough; slots past
// the team's warps stay zero, so that four are read at once.
template <int N>
struct TeamSums {
  alignas(16) float slot[2][N][kMaxTeams][kSlots];
};
template <int N>
__device__ __forceinline__ void clear_sums(TeamSums<N>& buf) {
  for (int i = threadIdx.x; i < 2 * N * kMaxTeams * kSlots; i += blockDim.x) (&buf.slot[0][0][0][0])[i] = 0.f;
  __syncthreads();
}

// Sums of N values over the team.  A team of several warps has a barrier of its own.
template <int N>
__device__ __forceinline__ void team_sum(float (&v)[N], int team, TeamSums<N>& buf, int* phase) {
  if (team < 32) {
    for (int o = team >> 1; o > 0; o >>= 1) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
    return;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  }
  if (team == 32) return;
  const int warps = team >> 5, warp = threadIdx.x >> 5, mine = warp / warps;
  const int set = *phase;
  *phase ^= 1;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) buf.slot[set][i][mine][warp - mine * warps] = v[i];
  }
  asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "r"(team) : "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float4* b = reinterpret_cast<const float4*>(buf.slot[set][i][mine]);
    float4 q = b[0];
    v[i] = (q.x + q.y) + (q.z + q.w);
    if (warps > 4) {
      q = b[1];
      v[i] += (q.x + q.y) + (q.z + q.w);
    }
    if (warps > 8) {
      q = b[2];
      v[i] += (q.x + q.y) + (q.z + q.w);
      q = b[3];
      v[i] += (q.x + q.y) + (q.z + q.w);
    }
  }
}

// A parameter vector as floats in shared memory, zeros past its end: element 4 i + j of a half, the first four
// elements of every chunk in one half and the last four in the other, so that neighbouring lanes read neighbours.
struct ParamCache {
  float4* half[2];
  __device__ __forceinline__ void get(int chunk, F2 (&v)[4]) const {
    const float4 a = half[0][chunk], b = half[1][chunk];
    v[0] = two(a.x, a.y); v[1] = two(a.z, a.w); v[2] = two(b.x, b.y); v[3] = two(b.z, b.w);
  }
};
// Fills it; the caller synchronises.  `room`: 8 floats per chunk, 16-byte aligned.
__device__ __forceinline__ ParamCache cache_param(float* room, const ParamVec& w, const Shape& s, float none) {
  const int chunks = s.width / 8;
  ParamCache c;
  c.half[0] = reinterpret_cast<float4*>(room);
  c.half[1] = c.half[0] + chunks;
#pragma unroll 4
  for (int i = threadIdx.x; i < chunks; i += blockDim.x) {
    float v[8];
    load_param(w, i * 8, s.cols, none, v);
    c.half[0][i] = make_float4(v[0], v[1], v[2], v[3]);
    c.half[1][i] = make_float4(v[4], v[5], v[6], v[7]);
  }
  return c;
}

// Quotient of a sum and the number of columns, to the last bit but for rare ties; exact where it is a float.  That of an
// infinite sum has no remainder.
__device__ __forceinline__ float mean_of(float sum, const Shape& s) {
  const float q = sum * s.inv;
  return fabsf(q) <= 3.402823466e38f ? fmaf(fmaf(-q, s.n, sum), s.inv, q) : q;
}

// 1 / sqrt(v), rounded to nearest but for rare ties: an error of rstd is shared by its whole row, and rsqrtf's is up to
// two units.  One step of Newton's iteration, r + r (1 - v r^2) / 2 with the residual to twice the precision.  (Rounded
// root and division instead take a subroutine and its registers: forward 16384 x 768 32 -> 46 us.)  0 and Inf, which
// rsqrtf has right, have no residual.
__device__ __forceinline__ float rstd_of(float v) {
  const float r = rsqrtf(v), h = v * r;
  const float e = fmaf(-fmaf(v, r, -h), r, fmaf(-h, r, 1.f));
  return v > 0.f && v <= 3.402823466e38f ? fmaf(0.5f * r, e, r) : r;
}

template <typename T>
struct Forward {
  Source<T> x, residual;              // residual.p may be null
  ParamVec weight, bias;
  float eps;
  T* y; long long ldy;
  T* sum_out; long long lds;
  float* mean;
  float* rstd;
  Act8 ck_sum, ck_y;
};

// What bounds it next to memory is the number of instructions, so they work on two values each where there is one that
// does, and addresses are stepped.
template <typename T, bool VEC, int K>
__global__ void __launch_bounds__(kForwardThreads<K>, 1) forward_kernel(Forward<T> a, Shape s) {
  extern __shared__ float4 dyn4[];          // weight and bias
  float* room = reinterpret_cast<float*>(dyn4);
  __shared__ TeamSums<1> buf;
  int phase = 0;
  const int teams = blockDim.x / s.team, t = threadIdx.x % s.team, mine = threadIdx.x / s.team, lane = threadIdx.x & 31;
  const bool prev = lane > 0 && t > 0, next = lane < 31 && t + 1 < s.team;      // neighbours of the same row
  const long long stride = (long long)gridDim.x * teams;
  const int turns = static_cast<int>((s.rows + stride - 1) / stride);   // the same for every thread: all take part in the sums
  long long r = (long long)blockIdx.x * teams + mine;
  const int first = t * 8, apart_by = s.team * 8;               // chunk k starts at first + k * apart_by
  const T* xp = a.x.p + r * a.x.ld;
  const T* up = a.residual.p ? a.residual.p + r * a.residual.ld : nullptr;
  T* yp = a.y + r * a.ldy;
  T* sp = a.sum_out ? a.sum_out + r * a.lds : nullptr;
  long long code = r * s.width + first, scale = r * s.scale_pitch + (first >> 5);
  const int pad = (first & 31) == 0 ? -s.groups & 3 : 0;
  Chunk<T, VEC> x[K], u[K];
  auto load = [&](bool live) {
    const int cols = live ? s.cols : 0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      x[k].fetch(a.x, xp, first + k * apart_by, cols);
      if (up) u[k].fetch(a.residual, up, first + k * apart_by, cols);
    }
  };
  load(r < s.rows);
  const ParamCache weight = cache_param(room, a.weight, s, 1.f), bias = cache_param(room + s.width, a.bias, s, 0.f);
  clear_sums(buf);
  for (int i = 0; i < turns; ++i) {
    const bool live = r < s.rows;
    F2 v[K][4], part = two(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool in = first + k * apart_by < s.cols;
      x[k].raw(in).get(v[k]);
      if (up) {
        F2 w[4];
        u[k].raw(in).get(w);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k][j] = add2(v[k][j], w[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) part = add2(part, v[k][j]);
    }
    xp += stride * a.x.ld;
    if (up) up += stride * a.residual.ld;
    load(r + stride < s.rows);
    float sum[1] = {sum_of(part)};
    team_sum(sum, s.team, buf, &phase);
    const float mean = mean_of(sum[0], s);
    const F2 minus_mean = two(-mean);
    part = two(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int left = s.cols - (first + k * apart_by);
      if (left <= 0) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        F2 d = add2(v[k][j], minus_mean);
        if (!VEC && left < 2 * j + 2) {                   // past the row's end: zeros that count as nothing
          float lo, hi;
          apart(d, &lo, &hi);
          d = two(left > 2 * j ? lo : 0.f, 0.f);
        }
        part = fma2(d, d, part);
      }
    }
    sum[0] = sum_of(part);
    team_sum(sum, s.team, buf, &phase);
    const float rstd = rstd_of(mean_of(sum[0], s) + a.eps);
    if (live && t == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    const F2 rstd2 = two(rstd);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int at = first + k * apart_by, g = at >> 5, left = s.cols - at;
      const bool keep = live && g < s.groups;
      Raw8<T> raw;
      if (sp || a.ck_sum.codes) {
        raw.put(v[k]);
        if (sp) store_chunk<T, VEC>(sp, at, s.cols, raw, live, prev, next);
        if (a.ck_sum.codes)               // the values as they are stored
          act8_put(a.ck_sum.codes + code + k * apart_by, a.ck_sum.scales + scale + k * (apart_by >> 5), raw, (at & 31) == 0,
                   g == s.groups - 1 ? pad : 0, keep);
      }
      raw.zero();
      if (left > 0) {
        F2 w[4], b[4];
        weight.get(at >> 3, w);
        bias.get(at >> 3, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[k][j] = fma2(mul2(add2(v[k][j], minus_mean), rstd2), w[j], b[j]);
          if (!VEC && left < 2 * j + 2) {
            float lo, hi;
            apart(v[k][j], &lo, &hi);
            v[k][j] = two(left > 2 * j ? lo : 0.f, 0.f);
          }
        }
        raw.put(v[k]);
      }
      store_chunk<T, VEC>(yp, at, s.cols, raw, live, prev, next);
      if (a.ck_y.codes)
        act8_put(a.ck_y.codes + code + k * apart_by, a.ck_y.scales + scale + k * (apart_by >> 5), raw, (at & 31) == 0,
                 g == s.groups - 1 ? pad : 0, keep);
    }
    r += stride;
    yp += stride * a.ldy;
    if (sp) sp += stride * a.lds;
    code += stride * s.width;
    scale += stride * s.scale_pitch;
  }
}

// Rows of any length: one block per row, three reads.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kBlock) forward_long_kernel(Forward<T> a, Shape s) {
  __shared__ TeamSums<1> buf;
  clear_sums(buf);
  int phase = 0;
  const int turns = (s.width / 8 + kBlock - 1) / kBlock, lane = threadIdx.x & 31;
  for (long long r = blockIdx.x; r < s.rows; r += gridDim.x) {
    auto value = [&](int first, float (&v)[8]) {
      Chunk<T, VEC> in;
      in.fetch(a.x, a.x.p + r * a.x.ld, first, s.cols);
      in.raw(first < s.cols).get(v);
      if (a.residual.p) {
        float u[8];
        in.fetch(a.residual, a.residual.p + r * a.residual.ld, first, s.cols);
        in.raw(first < s.cols).get(u);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += u[j];
      }
    };
    float sum[1] = {0.f};
    for (int i = 0; i < turns; ++i) {
      float v[8];
      value((threadIdx.x + i * kBlock) * 8, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] += v[j];
    }
    team_sum(sum, kBlock, buf, &phase);
    const float mean = mean_of(sum[0], s);
    sum[0] = 0.f;
    for (int i = 0; i < turns; ++i) {
      const int first = (threadIdx.x + i * kBlock) * 8;
      float v[8];
      value(first, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = first + j < s.cols ? v[j] - mean : 0.f;
        sum[0] = fmaf(d, d, sum[0]);
      }
    }
    team_sum(sum, kBlock, buf, &phase);
    const float rstd = rstd_of(mean_of(sum[0], s) + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    for (int i = 0; i < turns; ++i) {
      const int first = (threadIdx.x + i * kBlock) * 8, g = first >> 5;
      const int pad = g == s.groups - 1 ? -s.groups & 3 : 0;
      float v[8], w[8], b[8], y[8];
      value(first, v);
      load_param(a.weight, first, s.cols, 1.f, w);
      load_param(a.bias, first, s.cols, 0.f, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = first + j < s.cols ? fmaf((v[j] - mean) * rstd, w[j], b[j]) : 0.f;
      Raw8<T> rs, ry;
      rs.put(v);
      ry.put(y);
      if (a.sum_out) store_chunk<T, VEC>(a.sum_out + r * a.lds, first, s.cols, rs, true, lane > 0, lane < 31);
      store_chunk<T, VEC>(a.y + r * a.ldy, first, s.cols, ry, true, lane > 0, lane < 31);
      const long long code = r * s.width + first, scale = r * s.scale_pitch + g;
      if (a.ck_sum.codes) act8_put(a.ck_sum.codes + code, a.ck_sum.scales + scale, rs, (first & 31) == 0, pad, g < s.groups);
      if (a.ck_y.codes) act8_put(a.ck_y.codes + code, a.ck_y.scales + scale, ry, (first & 31) == 0, pad, g < s.groups);
    }
  }
}

template <typename T>
struct Backward {
  Source<T> dy, x;                    // x.p null: read the checkpoint
  Act8 ck;
  ParamVec weight;
  const float* mean;
  const float* rstd;
  Source<T> residual;
  T* dx; long long lddx;
  float* partials;                    // [gridDim.x][2][width], or null
};

// The normalised input as it lies in memory: values, or a checkpoint's codes.
template <typename T, bool VEC, bool CK>
struct Input {
  Chunk<T, VEC> x;
  // the first `cols` elements of row r exist
  __device__ __forceinline__ void load(const Backward<T>& a, const Shape&, long long r, int first, int cols) {
    x.fetch(a.x, a.x.p + r * a.x.ld, first, cols);
  }
  __device__ __forceinline__ void get(F2 (&v)[4]) const { x.raw(true).get(v); }
};
template <typename T, bool VEC>
struct Input<T, VEC, true> {
  RawAct8 x;
  __device__ __forceinline__ void load(const Backward<T>& a, const Shape& s, long long r, int first, int cols) {
    x.load(a.ck, r * s.width + first, r * s.scale_pitch + (first >> 5), first < cols);
  }
  __device__ __forceinline__ void get(F2 (&v)[4]) const { x.get(v); }
};

// The block's column sums (thread t of a team: chunks t + k * team) into its partial sums.  `dyn`: [teams - 1] of the
// team's values, element j of chunk k of thread t at (k * 8 + j) * team + t: neighbouring threads, neighbouring words.
template <int K>
__device__ __forceinline__ void write_partials(float* out, float* dyn, const Shape& s, int teams, int t, int mine,
                                               const F2 (&dw)[K][4], const F2 (&db)[K][4]) {
  const int all = s.team * 8 * K;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    float v[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) apart(half ? db[k][j] : dw[k][j], &v[k][2 * j], &v[k][2 * j + 1]);
    if (teams > 1) {
      __syncthreads();
      if (mine > 0) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int j = 0; j < 8; ++j) dyn[(mine - 1) * all + (k * 8 + j) * s.team + t] = v[k][j];
      }
      __syncthreads();
    }
    if (mine > 0) continue;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int first = (t + k * s.team) * 8;
      if (first >= s.width) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        for (int q = 0; q < teams - 1; ++q) v[k][j] += dyn[q * all + (k * 8 + j) * s.team + t];
      Raw8<float> o;
      o.put(v[k]);
      o.store(out + half * s.width + first);
    }
  }
}

// Persistent: a team walks over rows, its share of the column sums stays in registers.
template <typename T, bool VEC, int K, bool CK>
__global__ void __launch_bounds__((kBackwardThreads<T, K>), 1) backward_kernel(Backward<T> a, Shape s) {
  extern __shared__ float4 dyn4[];          // the weight; then the column sums of the block's other teams
  float* dyn = reinterpret_cast<float*>(dyn4) + s.width;
  __shared__ TeamSums<2> buf;
  int phase = 0;
  const int teams = blockDim.x / s.team, t = threadIdx.x % s.team, mine = threadIdx.x / s.team, lane = threadIdx.x & 31;
  const bool prev = lane > 0 && t > 0, next = lane < 31 && t + 1 < s.team;
  const long long stride = (long long)gridDim.x * teams;
  const int turns = static_cast<int>((s.rows + stride - 1) / stride);
  long long r = (long long)blockIdx.x * teams + mine;
  const int first = t * 8, apart_by = s.team * 8;
  const T* dyp = a.dy.p + r * a.dy.ld;
  const T* xp = CK ? nullptr : a.x.p + r * a.x.ld;
  long long code = r * s.width + first, scale = r * s.scale_pitch + (first >> 5);
  const T* up = a.residual.p ? a.residual.p + r * a.residual.ld : nullptr;
  T* dxp = a.dx + r * a.lddx;
  F2 dw[K][4], db[K][4];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[k][j] = db[k][j] = two(0.f);
  constexpr bool kResidualAhead = VEC && (sizeof(T) == 2 || K == 1);        // (elsewhere it would not fit the registers)
  Chunk<T, VEC> in_dy[K], in_x[CK ? 1 : K], in_u[K], next_u[K];
  RawAct8 in_q[CK ? K : 1];
  float mean = 0.f, rstd = 0.f;
  auto load = [&](long long row) {
    const bool live = row < s.rows;
    const int cols = live ? s.cols : 0;
    mean = live ? a.mean[row] : 0.f;
    rstd = live ? a.rstd[row] : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int at = first + k * apart_by;
      in_dy[k].fetch(a.dy, dyp, at, cols);
      if constexpr (CK) in_q[k].load(a.ck, code + k * apart_by, scale + k * (apart_by >> 5), at < cols);
      else in_x[k].fetch(a.x, xp, at, cols);
      if (kResidualAhead && up) next_u[k].fetch(a.residual, up, at, cols);
    }
  };
  load(r);
  const ParamCache weight = cache_param(reinterpret_cast<float*>(dyn4), a.weight, s, 1.f);
  clear_sums(buf);
  for (int i = 0; i < turns; ++i) {
    const bool live = r < s.rows;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (kResidualAhead) in_u[k] = next_u[k];
      else if (up) in_u[k].fetch(a.residual, up, first + k * apart_by, live ? s.cols : 0);
    }
    const F2 rstd2 = two(rstd), minus_mean = two(-mean);
    F2 g[K][4], h[K][4], sg = two(0.f), sgh = two(0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int left = live ? s.cols - (first + k * apart_by) : 0;
      if (left <= 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) g[k][j] = h[k][j] = two(0.f);
        continue;
      }
      F2 w[4], dy[4];
      weight.get((first + k * apart_by) >> 3, w);
      in_dy[k].raw(true).get(dy);
      if constexpr (CK) in_q[k].get(h[k]);
      else in_x[k].raw(true).get(h[k]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // (past the row's end dy is zero, and h only ever meets it or is not stored)
        h[k][j] = mul2(add2(h[k][j], minus_mean), rstd2);
        g[k][j] = mul2(dy[j], w[j]);
        sg = add2(sg, g[k][j]);
        sgh = fma2(g[k][j], h[k][j], sgh);
        dw[k][j] = fma2(dy[j], h[k][j], dw[k][j]);
        db[k][j] = add2(db[k][j], dy[j]);
      }
    }
    dyp += stride * a.dy.ld;
    if constexpr (CK) {
      code += stride * s.width;
      scale += stride * s.scale_pitch;
    } else {
      xp += stride * a.x.ld;
    }
    if (up) up += stride * a.residual.ld;
    load(r + stride);
    float sum[2] = {sum_of(sg), sum_of(sgh)};
    team_sum(sum, s.team, buf, &phase);
    const F2 mg = two(-sum[0] * s.inv), mgh = two(-sum[1] * s.inv);
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < 4; ++j) g[k][j] = mul2(fma2(h[k][j], mgh, add2(g[k][j], mg)), rstd2);
      if (up) {
        F2 u[4];
        in_u[k].raw(true).get(u);
#pragma unroll
        for (int j = 0; j < 4; ++j) g[k][j] = add2(g[k][j], u[j]);
      }
      Raw8<T> o;
      o.put(g[k]);
      store_chunk<T, VEC>(dxp, first + k * apart_by, s.cols, o, live, prev, next);
    }
    r += stride;
    dxp += stride * a.lddx;
  }
  if (a.partials) write_partials<K>(a.partials + (size_t)blockIdx.x * 2 * s.width, dyn, s, teams, t, mine, dw, db);
}

// Long rows, first step: mean(g) and mean(g h) of every row.
template <typename T, bool VEC, bool CK>
__global__ void __launch_bounds__(kBlock) backward_stats_kernel(Backward<T> a, Shape s, float* stats) {
  __shared__ TeamSums<2> buf;
  clear_sums(buf);
  int phase = 0;
  const int turns = (s.width / 8 + kBlock - 1) / kBlock;
  for (long long r = blockIdx.x; r < s.rows; r += gridDim.x) {
    const float mean = a.mean[r], rstd = a.rstd[r];
    float sum[2] = {0.f, 0.f};
    for (int i = 0; i < turns; ++i) {
      const int first = (threadIdx.x + i * kBlock) * 8;
      Input<T, VEC, CK> in;
      F2 v2[4];
      float dy[8], v[8], w[8];
      in.load(a, s, r, first, s.cols);
      Chunk<T, VEC> in_dy;
      in_dy.fetch(a.dy, a.dy.p + r * a.dy.ld, first, s.cols);
      in_dy.raw(first < s.cols).get(dy);
      in.get(v2);
      load_param(a.weight, first, s.cols, 1.f, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) apart(v2[j], &v[2 * j], &v[2 * j + 1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {        // (past the row's end dy is zero)
        const float g = dy[j] * w[j];
        sum[0] += g;
        sum[1] = first + j < s.cols ? fmaf(g, (v[j] - mean) * rstd, sum[1]) : sum[1];
      }
    }
    team_sum(sum, kBlock, buf, &phase);
    if (threadIdx.x == 0) {
      stats[2 * r] = mean_of(sum[0], s);
      stats[2 * r + 1] = mean_of(sum[1], s);
    }
  }
}

// Second step: a block owns 256 columns and a share of the rows.
template <typename T, bool VEC, bool CK>
__global__ void __launch_bounds__(256) backward_long_kernel(Backward<T> a, Shape s, const float* stats) {
  __shared__ float part[8][8 * 33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int first = (blockIdx.y * 32 + lane) * 8;
  float dw[8], db[8], w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) dw[j] = db[j] = 0.f;
  load_param(a.weight, first, s.cols, 1.f, w);
  for (long long r = (long long)blockIdx.x * 8 + warp; r < s.rows; r += (long long)gridDim.x * 8) {
    const float mean = a.mean[r], rstd = a.rstd[r], mg = stats[2 * r], mgh = stats[2 * r + 1];
    Input<T, VEC, CK> in;
    F2 v2[4];
    float dy[8], v[8], o[8];
    in.load(a, s, r, first, s.cols);
    Chunk<T, VEC> other;
    other.fetch(a.dy, a.dy.p + r * a.dy.ld, first, s.cols);
    other.raw(first < s.cols).get(dy);
    in.get(v2);
#pragma unroll
    for (int j = 0; j < 4; ++j) apart(v2[j], &v[2 * j], &v[2 * j + 1]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float h = first + j < s.cols ? (v[j] - mean) * rstd : 0.f;
      o[j] = rstd * (fmaf(dy[j], w[j], -mg) - h * mgh);
      dw[j] = fmaf(dy[j], h, dw[j]);
      db[j] += dy[j];
    }
    if (a.residual.p) {
      other.fetch(a.residual, a.residual.p + r * a.residual.ld, first, s.cols);
      other.raw(first < s.cols).get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] += v[j];
    }
    Raw8<T> raw;
    raw.put(o);
    store_chunk<T, VEC>(a.dx + r * a.lddx, first, s.cols, raw, true, lane > 0, lane < 31);
  }
  if (!a.partials) return;
  float* out = a.partials + (size_t)blockIdx.x * 2 * s.width;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int j = 0; j < 8; ++j) part[warp][j * 33 + lane] = half ? db[j] : dw[j];
    __syncthreads();
    const int j = threadIdx.x & 7, l = threadIdx.x >> 3;
    const int col = blockIdx.y * 256 + threadIdx.x;
    if (col < s.width) {
      float v = 0.f;
      for (int q = 0; q < 8; ++q) v += part[q][j * 33 + l];
      out[(size_t)half * s.width + col] = v;
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
  s.width = s.groups * 32;
  s.scale_pitch = static_cast<int>(act8_scale_pitch(cols));
  s.n = static_cast<float>(cols);
  s.inv = 1.f / s.n;
  return s;
}

// Threads per row and chunks (8 values) per thread; false: the row does not fit.  `few` and `many`: chunks per
// thread of rows of up to `limit` chunks, and of longer ones.
bool ln_team(ln::Shape* s, bool vec, int limit, int few, int many, int max_k, int* K) {
  const int chunks = s->width / 8;
  if (chunks > ln::kBlock * max_k) return false;
  // up to one row per SM there is only the one row's latency to shorten: as many threads as it has chunks
  *K = s->rows <= sm_count() ? 1 : chunks <= limit ? few : many;
  while (*K * ln::kBlock < chunks) *K *= 2;
  while (*K > 1 && chunks <= 32 * (*K / 2)) *K /= 2;
  auto places = [&](int k) { return ((chunks + k - 1) / k + 31) / 32 * 32 * k; };
  if (*K == 4 && places(3) < places(4) && 3 * ln::kBlock >= chunks) *K = 3;
  const int threads = (chunks + *K - 1) / *K;
  if (vec && threads <= 32) {
    int t = 4;
    while (t < threads) t *= 2;
    s->team = t;
  } else {
    s->team = (threads + 31) / 32 * 32;
  }
  return true;
}
// Block size: whole teams, a multiple of 32 threads, and no more teams than bring the rows to all SMs.
int ln_block(const ln::Shape& s, int most) {
  const int unit = s.team < 32 ? 32 : s.team, per_unit = unit / s.team;
  const long long rows_per_sm = (s.rows + sm_count() - 1) / sm_count();
  long long units = (rows_per_sm + per_unit - 1) / per_unit;
  if (units > most / unit) units = most / unit;
  return unit * static_cast<int>(units < 1 ? 1 : units);
}

template <typename T, bool VEC>
cudaError_t ln_forward_t(const ln::Forward<T>& a, long long rows, long long cols, cudaStream_t st) {
  ln::Shape s = ln_shape(rows, cols);
  int K = 1;
  const int few = sizeof(T) == 4 ? 1 : VEC ? 4 : 2, many = sizeof(T) == 2 && VEC ? 4 : 2;
  if (!ln_team(&s, VEC, 256, few, many, ln::kMaxKForward, &K)) {
    const unsigned grid = static_cast<unsigned>(rows < (1 << 30) ? rows : 1 << 30);
    ln::forward_long_kernel<T, VEC><<<grid, ln::kBlock, 0, st>>>(a, s);
    return cudaGetLastError();
  }
  const int threads = ln_block(s, K == 1 ? 768 : ln::kBlock), teams = threads / s.team;
  const long long want = (rows + teams - 1) / teams, most = sm_count();
  const unsigned grid = static_cast<unsigned>(want < most ? want : most);
  const size_t smem = 2 * (size_t)s.width * sizeof(float);
  // The attribute belongs to the kernel: always what its widest row takes, so that calls of several threads agree.
  auto go = [&](auto kernel, int k) {
    const size_t most = 2 * (size_t)k * ln::kBlock * 8 * sizeof(float);
    if (most > 32 << 10) {
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
      if (e != cudaSuccess) return e;
    }
    kernel<<<grid, threads, smem, st>>>(a, s);
    return cudaGetLastError();
  };
  return K == 1   ? go(ln::forward_kernel<T, VEC, 1>, 1)
         : K == 2 ? go(ln::forward_kernel<T, VEC, 2>, 2)
         : K == 3 ? go(ln::forward_kernel<T, VEC, 3>, 3)
                  : go(ln::forward_kernel<T, VEC, 4>, 4);
}

template <typename T>
cudaError_t ln_forward_d(Mat x, Mat residual, long long rows, long long cols, Param weight, Param bias, float eps,
                         Mat y, Mat sum_out, float* mean, float* rstd, void* ck_sum, void* ck_y, cudaStream_t st) {
  if (rows == 0) return cudaSuccess;
  ln::Forward<T> a{};
  a.x = source_of<T>(x, 0, rows, cols);
  a.residual = source_of<T>(residual, 0, rows, cols);
  a.weight = param_vec(weight); a.bias = param_vec(bias);
  a.eps = eps;
  a.y = row_of<T>(y, 0); a.ldy = y.ld;
  a.sum_out = row_of<T>(sum_out, 0); a.lds = sum_out.ld;
  a.mean = mean; a.rstd = rstd;
  a.ck_sum = act8_at(ck_sum, rows, cols, 0); a.ck_y = act8_at(ck_y, rows, cols, 0);
  const bool vec = mat_vec<T>(x, cols) && mat_vec<T>(residual, cols) && mat_vec<T>(y, cols) && mat_vec<T>(sum_out, cols);
  return vec ? ln_forward_t<T, true>(a, rows, cols, st) : ln_forward_t<T, false>(a, rows, cols, st);
}

// Blocks of the backward kernels: what is resident at once, as far as there are rows.
struct LnBackwardGrid {
  ln::Shape s;
  int K, threads, teams;
  unsigned grid;
  bool is_long;
};
LnBackwardGrid ln_backward_grid(bool vec, int dtype, long long rows, long long cols) {
  LnBackwardGrid g{};
  g.s = ln_shape(rows, cols);
  // One chunk a thread up to so many of them, two beyond; from a checkpoint, 16384 rows.  Aligned bf16: of 1024 columns
  // 39.9 us with one and 37.6 with two, 1536 56.0 and 50.0, 2048 70.3 and 60.4.  Aligned fp32, whose chunk takes twice the
  // registers: 2048 78.6 and 92.9, 2304 (the least good for one) 120 and 108, 2816 126 and 132, 4096 149 and 196.
  // Unaligned: fp32 2001 134 and 141, 2305 224 and 173, 4001 282 and 271; bf16 2001 124 and 126, 2305 169 and 155.
  const int limit = !vec ? 256 : dtype == FA_BF16 ? 128 : 512;
  g.is_long = !ln_team(&g.s, vec, limit, 1, 2, ln::kMaxKBackward, &g.K);
  long long want;
  if (g.is_long) {
    const long long tiles = (g.s.width + 255) / 256;
    g.threads = 256; g.teams = 8;
    want = (4LL * sm_count() + tiles - 1) / tiles;
  } else {
    g.threads = ln_block(g.s, g.K == 1 && dtype == FA_BF16 ? 768 : ln::kBlock);
    g.teams = g.threads / g.s.team;
    want = sm_count();
  }
  const long long most = (rows + g.teams - 1) / g.teams;
  if (want > most) want = most;
  g.grid = static_cast<unsigned>(want < 1 ? 1 : want);
  return g;
}

template <typename T, bool VEC, bool CK>
cudaError_t ln_backward_t(const ln::Backward<T>& a, const LnBackwardGrid& g, float* row_stats, cudaStream_t st) {
  if (g.is_long) {
    const unsigned row_grid = static_cast<unsigned>(g.s.rows < (1 << 30) ? g.s.rows : 1 << 30);
    ln::backward_stats_kernel<T, VEC, CK><<<row_grid, ln::kBlock, 0, st>>>(a, g.s, row_stats);
    const dim3 grid(g.grid, (g.s.width + 255) / 256);
    ln::backward_long_kernel<T, VEC, CK><<<grid, 256, 0, st>>>(a, g.s, row_stats);
  } else {
    // a team's row has at most 8 K values a thread: at most 32 KB with 512 threads of K = 2 and less with others, which
    // needs no attribute
    static_assert(ln::kBlock * 8 * ln::kMaxKBackward * sizeof(float) <= 32 << 10 && 768 * 8 * sizeof(float) <= 32 << 10, "");
    const size_t smem = (size_t)g.s.width * sizeof(float) +
                        (a.partials ? (size_t)(g.teams - 1) * g.s.team * 8 * g.K * sizeof(float) : 0);
    auto go = [&](auto kernel) { kernel<<<g.grid, g.threads, smem, st>>>(a, g.s); };
    if (g.K == 1) go(ln::backward_kernel<T, VEC, 1, CK>);
    else go(ln::backward_kernel<T, VEC, 2, CK>);
  }
  return cudaGetLastError();
}

template <typename T>
cudaError_t ln_backward_d(Mat dy, Mat x, const void* ck, long long rows, long long cols, Param weight,
                          const float* mean, const float* rstd, Mat residual, Mat dx, void* dweight, void* dbias,
                          int gdtype, float* partials, float* row_stats, cudaStream_t st) {
  const bool vec = mat_vec<T>(dy, cols) && mat_vec<T>(x, cols) && mat_vec<T>(residual, cols) && mat_vec<T>(dx, cols);
  const LnBackwardGrid g = ln_backward_grid(vec, sizeof(T) == 2 ? FA_BF16 : FA_F32, rows, cols);
  const bool sums = dweight || dbias;
  if (rows > 0) {
    ln::Backward<T> a{};
    a.dy = source_of<T>(dy, 0, rows, cols);
    a.x = source_of<T>(x, 0, rows, cols);
    a.ck = act8_at(ck, rows, cols, 0);
    a.weight = param_vec(weight);
    a.mean = mean; a.rstd = rstd;
    a.residual = source_of<T>(residual, 0, rows, cols);
    a.dx = row_of<T>(dx, 0); a.lddx = dx.ld;
    a.partials = sums ? partials : nullptr;
    const cudaError_t e = ck ? (vec ? ln_backward_t<T, true, true>(a, g, row_stats, st)
                                    : ln_backward_t<T, false, true>(a, g, row_stats, st))
                             : (vec ? ln_backward_t<T, true, false>(a, g, row_stats, st)
                                    : ln_backward_t<T, false, false>(a, g, row_stats, st));
    if (e != cudaSuccess) return e;
  }
  if (!sums) return cudaSuccess;
  return launch_finish_columns(partials, rows > 0 ? (int)g.grid : 0, 2, g.s.width, cols, dweight, dbias, gdtype, st);
}

}  // namespace

size_t layer_norm_partials_bytes(long long rows, long long cols) {
  // type and alignment are known at the call: no grid has more blocks than there are SMs, or than 4 per SM for long rows
  const LnBackwardGrid g = ln_backward_grid(true, FA_F32, rows, cols);
  const long long most = g.is_long ? g.grid : sm_count();
  return (size_t)(most < rows ? most : rows < 1 ? 1 : rows) * 2 * g.s.width * sizeof(float);
}
bool layer_norm_needs_row_stats(long long cols) { return act8_groups(cols) * 4 > ln::kBlock * ln::kMaxKBackward; }

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
