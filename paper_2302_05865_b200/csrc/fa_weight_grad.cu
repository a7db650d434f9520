// Weight gradient of a linear layer from the 8-bit checkpoint of its input:
//   dW[o][i] = sum over tokens t of dY[t][o] * X[t][i],   X read back from the checkpoint.
#include "../../include/fa.h"
#include "fa_columns.cuh"
#include "fa_train.h"

namespace fa {
namespace wgrad {

constexpr int kTile = 64, kTokens = 16;

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) simple_kernel(const T* __restrict__ dy, long long lddy, Act8 ck, long long rows,
                                                     int outs, int ins, int groups, int scale_pitch, void* dw,
                                                     int gbf16) {
  __shared__ float a[kTokens][kTile], b[kTokens][kTile];
  const int o0 = blockIdx.y * kTile, i0 = blockIdx.x * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  const int half = threadIdx.x >> 7, k = (threadIdx.x & 127) >> 3, c = threadIdx.x & 7;
  for (long long t0 = 0; t0 < rows; t0 += kTokens) {
    const long long t = t0 + k;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.f;
    if (half == 0) {
      if (t < rows && o0 + c * 8 < outs) load_chunk<T, VEC>(dy + t * lddy, o0 / 8 + c, outs).get(v);
    } else if (t < rows && i0 + c * 8 < groups * 32) {
      act8_decode(*reinterpret_cast<const uint2*>(ck.codes + (size_t)t * groups * 32 + i0 + c * 8),
                  ck.scales[(size_t)t * scale_pitch + (i0 + c * 8) / 32], v);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) (half ? b : a)[k][c * 8 + j] = v[j];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kTokens; ++q)
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[y][x] = fmaf(a[q][ty * 4 + y], b[q][tx + 16 * x], acc[y][x]);
  }
#pragma unroll
  for (int y = 0; y < 4; ++y)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int o = o0 + ty * 4 + y, i = i0 + tx + 16 * x;
      if (o >= outs || i >= ins) continue;
      const size_t at = (size_t)o * ins + i;
      if (gbf16) static_cast<bf16*>(dw)[at] = __float2bfloat16_rn(acc[y][x]);
      else static_cast<float*>(dw)[at] = acc[y][x];
    }
}

}  // namespace wgrad

size_t linear_weight_grad_scratch_bytes(long long, long long, long long, int) { return 0; }

template <typename T>
static cudaError_t weight_grad_t(Mat dy, long long rows, long long outs, long long ins, const void* ck, void* dweight,
                                 int gdtype, cudaStream_t st) {
  const dim3 grid((ins + wgrad::kTile - 1) / wgrad::kTile, (outs + wgrad::kTile - 1) / wgrad::kTile);
  auto go = [&](auto kernel) {
    kernel<<<grid, 256, 0, st>>>(row_of<T>(dy, 0), dy.ld, act8_at(ck, rows, ins, 0), rows, (int)outs, (int)ins,
                                 (int)act8_groups(ins), (int)act8_scale_pitch(ins), dweight, gdtype == FA_BF16);
  };
  if (mat_vec<T>(dy, outs)) go(wgrad::simple_kernel<T, true>);
  else go(wgrad::simple_kernel<T, false>);
  return cudaGetLastError();
}

cudaError_t launch_linear_weight_grad(Mat dy, int dtype, long long rows, long long outs, long long ins, const void* ck,
                                      void* dweight, int gdtype, void*, cudaStream_t st) {
  return dtype == FA_BF16 ? weight_grad_t<bf16>(dy, rows, outs, ins, ck, dweight, gdtype, st)
                          : weight_grad_t<float>(dy, rows, outs, ins, ck, dweight, gdtype, st);
}

}  // namespace fa
