// Gated residual with the norms before and after a block: kernel arguments and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vcja {

constexpr int kResidualCols = 8192;  // widest row: 1,024 threads of eight columns

struct ResidualArgs {
  const void *x, *a;                          // stream and block output, [rows, cols]; a may be NULL
  const void *gate, *scale, *shift, *wp;      // parameters, NULL: 1, (1 or 0), 0, 1
  void *h, *y;                                // forward; y without a norm NULL, h without a block output NULL
  float *mean, *rstd, *pmean, *prstd;         // [rows]: statistics of h and of a
  int8_t *h8, *a8;                            // checkpoints (NULL: none) and their scales
  float *h8s, *a8s;
  const void *dh, *dy;                        // backward; either may be NULL
  const void* h_in;                           // backward: h and a as the forward left them, or in 8 bits (h8, a8)
  void *dx, *da;
  void *dgate, *dscale, *dshift, *dwp;        // NULL: not wanted
  float* part;                                // [groups + samples][3][cols]: each run's sums of H xa, dy xh, dy
  float* sums;                                // [samples][3][cols], where sums over samples are wanted
  const int32_t *cu, *lens;
  int64_t x_stride, a_stride, dh_stride, dy_stride, h_stride;  // h_stride: of h_in
  int64_t gate_stride, scale_stride, shift_stride;  // elements between samples; 0: one for all of them
  int rows, cols, samples, per;               // per: rows of a sample's slot (without cu)
  int groups, chunk;                          // workgroups, and the rows of each
  float c, eps;
  int norm, post;                             // VC_NORM_*
  bool plus_one, p_f32, x_f32, y_f32, clear;
  bool flat;                                  // backward: one set of sums over all rows, no vector is a sample's own
};

// Rows of one workgroup, and how many of these there are (the same forward and backward).
void residual_groups(int64_t rows, int cols, bool backward, int* groups, int* chunk);
hipError_t launch_residual_fwd(const ResidualArgs& a, hipStream_t s);
hipError_t launch_residual_bwd(const ResidualArgs& a, bool kept, hipStream_t s);

}  // namespace vcja
