// Embedding of tokens: kernel arguments and launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vcja {

struct EmbeddingArgs {
  const void* ids;           // int32 or int64 [tokens]
  const void* table;         // forward: [vocab, cols]
  void* out;                 // forward: [tokens, cols], contiguous
  const void* dout;          // backward: [tokens, cols], rows dout_stride elements apart
  void* grad;                // backward: [vocab, cols], contiguous
  int64_t tokens, vocab, padding, dout_stride, table_stride;
  int cols;
  float scale;
  bool ids64, table_f32, out_f32, grad_f32, add;
  bool once;                 // backward: zeros and dout past the caches
  // backward: the tokens' ids in order, and where they stand; two of each, as a pass of the sort goes from one to the other
  uint32_t *keys[2], *pos[2];
  uint32_t* hist;            // [blocks][512] digits of a pass, where several workgroups sort
  float* part;               // [chunks][2][cols]
  int digits, passes;        // bits of a pass, passes
  int chunk, chunks;         // sorted tokens of a share, and shares
  int64_t filled;            // rows from here on have been written as zeros beside the sort
};

constexpr int64_t kEmbeddingTokens = (int64_t)1 << 24;  // most tokens of a backward
constexpr int64_t kEmbeddingVocab = (int64_t)1 << 27;   // most rows of a table: three passes of nine bits, of 2^27 itself (keys go up to it) four of seven
struct EmbeddingPlan {
  int passes, digits, blocks, chunk, chunks;
};
EmbeddingPlan embedding_plan(int64_t tokens, int64_t vocab, int cols);
hipError_t launch_embedding_fwd(const EmbeddingArgs& a, hipStream_t s);
hipError_t launch_embedding_bwd(EmbeddingArgs a, hipStream_t s);

}  // namespace vcja
