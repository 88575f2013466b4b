// Attention over caches in 4 bits on the tensor cores: what k_chunk.cu's launches take from k_chunk4.cu.
#pragma once

#include "k_chunk_dev.cuh"

namespace tlf {

// 3-D map over q: {head_dim, Hq, tokens}, boxes of 64 elements x the heads of a kv head x 128 / G tokens, one column of a tile
// of 128 rows; tokens past the last read as zeros.
bool chunk_q_map(CUtensorMap* m, const ChunkAttn& a);

// CTAs that an SM holds of the kernel for `rows` (8 or 16) rows; the launch for a.rows of them (8, 16 or PAIR_ROWS).
int chunk4_per_sm(int hd, int rows);
cudaError_t launch_chunk4(const ChunkAttn& a, cudaStream_t st);

}  // namespace tlf
