// Attention over caches in 4 bits on the tensor cores: what k_chunk.cu's launches take from k_chunk4.cu.
#pragma once

#include "k_chunk_dev.cuh"

namespace tlf {

// CTAs that an SM holds of the kernel for `rows` (8 or 16) rows, and its launch (a.rows of them).
int chunk4_per_sm(int hd, int rows);
cudaError_t launch_chunk4(const ChunkAttn& a, cudaStream_t st);

}  // namespace tlf
