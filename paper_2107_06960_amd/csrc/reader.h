// reader.h -- argument blocks and launchers of the reader's operators
// (reader.cpp checks the calls; norm.hip, linear.hip and cross.hip hold the
// kernels).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/mafat_reader.h"

namespace mafat {

struct NormArgs {
  const void* x;
  const void* res;
  const float* gain;
  void* sum;
  void* y;
  float* y_scale;
  int64_t x_stride, res_stride, sum_stride, y_stride;
  int64_t rows;
  int32_t cols;
  float eps;
};
hipError_t launch_norm(int dtype, int out_dtype, const NormArgs& a, hipStream_t stream);

}  // namespace mafat
