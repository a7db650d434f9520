// Column sums over many rows in a fixed order: blocks write partial sums, finish_columns adds them.
#pragma once
#include "../../include/fa.h"
#include "fa_act8.cuh"
#include "fa_kernels.h"
#include "fa_train.h"

namespace fa {

// partials: [parts][sums][width] floats; out0 / out1 (null: not wanted) receive sum 0 / 1 of columns < cols.
cudaError_t launch_finish_columns(const float* partials, int parts, int sums, long long width, long long cols,
                                  void* out0, void* out1, int gdtype, cudaStream_t st);

// ---- host side: operands of a launch
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
template <typename T> inline bool mat_vec(const Mat& m, long long cols) {
  return !m.p || (aligned16(m.p) && cols % 8 == 0 && (m.ld * (long long)sizeof(T)) % 16 == 0);
}
inline ParamVec param_vec(const Param& w) {
  ParamVec v{};
  v.p = w.p;
  v.is_bf16 = w.dtype == FA_BF16;
  v.vec = aligned16(w.p);
  return v;
}
inline Act8 act8_at(const void* ck, long long rows, long long cols, long long row) {
  Act8 a{};
  if (ck) {
    uint8_t* base = static_cast<uint8_t*>(const_cast<void*>(ck));
    a.codes = base + row * act8_groups(cols) * 32;
    a.scales = base + act8_scale_offset(rows, cols) + row * act8_scale_pitch(cols);
  }
  return a;
}
template <typename T> inline T* row_of(const Mat& m, long long row) {
  return m.p ? static_cast<T*>(const_cast<void*>(m.p)) + row * m.ld : nullptr;
}

template <typename T> inline Source<T> source_of(const Mat& m, long long row, long long rows, long long cols) {
  Source<T> s{row_of<const T>(m, row), m.ld, nullptr};
  if (s.p) s.end = s.p + (rows - 1) * m.ld + cols;
  return s;
}

}  // namespace fa
