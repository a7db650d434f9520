// Internal launch interface of the training operators (fa_train_api.cu checks the arguments).
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>

namespace fa {

constexpr int kGeluErf = 0, kGeluTanh = 1;

// A rows x cols matrix of activations with unit column stride.
struct Mat {
  const void* p;
  long long ld;      // elements from row to row
};
struct Param {
  const void* p;     // may be null
  int dtype;
};

cudaError_t launch_act8_store(Mat x, int dtype, long long rows, long long cols, void* ck, cudaStream_t st);
cudaError_t launch_act8_load(const void* ck, long long rows, long long cols, Mat out, int dtype, cudaStream_t st);

// y = gelu(x + bias), checkpoints of x + bias and of y where wanted
cudaError_t launch_gelu_forward(Mat x, int dtype, long long rows, long long cols, Param bias, int approx, Mat y,
                                void* ck_x, void* ck_y, cudaStream_t st);

// Column sums over the rows are formed in two steps: partial sums per block, then one kernel that adds
// them in a fixed order.  Bytes of the partial sums of one sum per column (layer norm: its own two).
size_t column_partials_bytes(long long rows, long long cols);

// dx = dy * gelu'(z), dbias = column sums of dx (null: not wanted); z = x + bias or read back from ck
cudaError_t launch_gelu_backward(Mat dy, Mat x, Param bias, const void* ck, int dtype, long long rows, long long cols,
                                 int approx, Mat dx, void* dbias, int gdtype, float* partials, cudaStream_t st);

cudaError_t launch_layer_norm_forward(Mat x, Mat residual, int dtype, long long rows, long long cols, Param weight,
                                      Param bias, float eps, Mat y, Mat sum_out, float* mean, float* rstd, void* ck_sum,
                                      void* ck_y, cudaStream_t st);

size_t layer_norm_partials_bytes(long long rows, long long cols);
// row_stats: 2 * rows floats, used when layer_norm_needs_row_stats(cols)
bool layer_norm_needs_row_stats(long long cols);
cudaError_t launch_layer_norm_backward(Mat dy, Mat x, const void* ck, int dtype, long long rows, long long cols,
                                       Param weight, const float* mean, const float* rstd, Mat residual_grad, Mat dx,
                                       void* dweight, void* dbias, int gdtype, float* partials, float* row_stats,
                                       cudaStream_t st);

cudaError_t launch_linear_weight_grad(Mat dy, int dtype, long long rows, long long outs, long long ins, const void* ck,
                                      void* dweight, void* dbias, int gdtype, void* scratch, cudaStream_t st);
// whether dY is bf16 and TMA can address its rows
bool linear_weight_grad_direct(Mat dy, int dtype, long long outs);
size_t linear_weight_grad_scratch_bytes(long long rows, long long outs, long long ins, int dtype, bool direct);

}  // namespace fa
