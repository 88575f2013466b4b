// The 4-bit cache's layout (include/tlf.h), as its kernels take it.
#pragma once

#include "k_serve.cuh"

namespace tlf {

template <int HD>
struct Kv4 {
  static constexpr int GS = HD < 64 ? HD : 64, NG = HD / GS;              // values and number of an entry's groups
  static constexpr int CODES = SV_PAGE * HD / 2, PAIRS = SV_PAGE * NG * 4;  // bytes of a block's two parts
  static constexpr int BLOCK = CODES + PAIRS;
};
inline int kv4_block_bytes(int hd) { return SV_PAGE * (hd / 2 + 4 * (hd > 64 ? hd / 64 : 1)); }

// (d, lo) of a group.
__device__ __forceinline__ float2 kv4_pair(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

// The eight values of a word of codes: one rounding of d n, which is exact in float32, plus lo.
__device__ __forceinline__ void kv4_values(uint32_t w, float2 p, float* x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = fmaf(p.x, (float)((w >> (4 * i)) & 15u), p.y);
}

cudaError_t launch_kv4_append(const ChunkDev& c, int dtype, const tlf_rope_args& a, int num_sms, cudaStream_t st);
cudaError_t launch_kv4_read(const ChunkDev& c, int dtype, const tlf_kv4_read_args& a, int num_sms, cudaStream_t st);

}  // namespace tlf
