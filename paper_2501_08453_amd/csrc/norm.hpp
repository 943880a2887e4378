// Layer norm: kernel arguments and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vcja {

struct NormArgs {
  const void *x, *w, *b;  // w, b may be NULL (1 and 0)
  void* y;
  float *mean, *rstd;     // [rows]; the backward reads them
  const void* dout;       // backward
  void *dx, *dw, *db;     // backward; dw, db may be NULL
  float* part;            // backward: [2][groups][cols] partial column sums (dw, db)
  int rows, cols;
  int64_t stride;         // elements between the rows of x (and of dout: dout_stride)
  int64_t dout_stride;
  float eps;
  bool x_f32, p_f32;      // element types: bf16 or fp32
  int groups;             // backward: runs of rows whose column sums are kept apart
};
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s);
// Most rows of a call (2^30; rows too wide for registers take a workgroup each, and a launch less than 2^32 threads).
int64_t norm_max_rows(int cols);
// Runs of rows of the backward's column sums.
int norm_groups(int64_t rows, int cols);

}  // namespace vcja
