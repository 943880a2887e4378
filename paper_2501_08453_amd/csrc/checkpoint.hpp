// Checkpoints in 8 bits: kernel arguments and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vcja {

struct CheckpointArgs {
  const void* x;     // pack: the values; [rows, cols], rows `stride` elements apart
  void* y;           // unpack: the values, contiguous
  int8_t* q;         // [rows, cols]
  float* scales;     // [rows, blocks]
  int64_t rows;
  int64_t stride;
  int cols, blocks;  // blocks of 128 columns of a row
  bool f32;          // type of x or y
};
hipError_t launch_checkpoint_pack(const CheckpointArgs& a, hipStream_t s);
hipError_t launch_checkpoint_unpack(const CheckpointArgs& a, hipStream_t s);

}  // namespace vcja
