// Shared by the operators on a caller's paged caches (k_rope.cu, k_chunk.cu, k_evict.cu) and on logits (k_sample.cu).
#pragma once

#include "tlf_internal.cuh"

namespace tlf {

constexpr int SV_PAGE = 64;
constexpr int SV_MAX_ROWS = 1024;

// A tlf_chunk as the kernels take it (checked by the host; cu, lens, page_table hold what the device finds there).
struct ChunkDev {
  int n, T, max_chunk, Hq, Hkv, G, hd, J, layer, max_pages;
  long long n_pages, page_elems;
  void* pool;
  const int* page_table;
  const int* cu;
  const int* lens;
  uint32_t* err;  // may be NULL
};

// Bits of a caller's error word beside those of the library's own (DEVERR_WAIT, DEVERR_INDEX).
enum : uint32_t { SVERR_VALUE = 8u, SVERR_PAGES = 16u };

__device__ __forceinline__ void sv_report(uint32_t* err, uint32_t bit) {
  if (err) atomicOr(err, bit);
}

// New tokens t0 .. t0 + ql - 1 and cache entries of row b. What is out of range is reported and cut, so that nothing below
// reads past the arrays: a row with bad offsets has no tokens, a bad length no more entries than the page table's row.
struct ChunkRow {
  int t0, ql, len;
};
__device__ __forceinline__ ChunkRow chunk_row(const ChunkDev& c, int b) {
  ChunkRow r;
  const int a = c.cu[b], e = c.cu[b + 1];
  r.t0 = a;
  r.ql = e - a;
  if (a < 0 || e < a || e > c.T) {
    sv_report(c.err, DEVERR_INDEX);
    r.t0 = r.ql = 0;
  }
  if (r.ql > c.max_chunk) {
    sv_report(c.err, DEVERR_INDEX);
    r.ql = c.max_chunk;
  }
  r.len = c.lens[b];
  if (r.len < 0 || r.len > c.max_pages * SV_PAGE) {
    sv_report(c.err, DEVERR_INDEX);
    r.len = r.len < 0 ? 0 : c.max_pages * SV_PAGE;
  }
  return r;
}

// Page p of row b, -1 (reported) when the table holds no page of the pool.
__device__ __forceinline__ int chunk_page(const int* table, int max_pages, long long n_pages, int b, int p, uint32_t* err) {
  const int page = table[(size_t)b * max_pages + p];
  if (page >= 0 && page < n_pages) return page;
  sv_report(err, DEVERR_INDEX);
  return -1;
}

// 2^x with the hardware approximation (relative error about 2^-22).
__device__ __forceinline__ float ex2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two floats in a register pair: one instruction works on both, where the issue slots bound a loop.
__device__ __forceinline__ uint64_t f2_pack(float x, float y) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 f2_unpack(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <typename T>
__device__ __forceinline__ T block_sum(T v, T* red) {  // every thread gets the sum; red: 33 values; fixed order
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (lane == 0) red[warp] = v;
  __syncthreads();
  if (warp == 0) {
    T x = lane < warps ? red[lane] : T(0);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (lane == 0) red[32] = x;
  }
  __syncthreads();
  return red[32];
}
// Exclusive prefix over the block; *total gets the sum.
template <typename T>
__device__ __forceinline__ T block_scan(T v, T* red, T* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  T x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) red[warp] = x;
  __syncthreads();
  if (warp == 0) {
    T w = lane < warps ? red[lane] : T(0), s = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    red[lane] = s - w;
    if (lane == 31) red[32] = s;
  }
  __syncthreads();
  if (total) *total = red[32];
  return red[warp] + x - v;
}

// launch_k with clusters of cs CTAs.
template <typename... KArgs, typename... Args>
inline cudaError_t launch_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, int cs, size_t smem, cudaStream_t st,
                                  Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cs;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = g_use_pdl ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

// ---- launchers ----
cudaError_t launch_rope_scaled_table(const tlf_rope_config& cfg, int max_pos, float* table, cudaStream_t st);
cudaError_t launch_rope_chunk(const ChunkDev& c, int dtype, const tlf_rope_args& a, int num_sms, cudaStream_t st);

// Attention of chunks: scratch (0 bytes: refused) and launch.
size_t chunk_attn_scratch(const ChunkDev& c, int dtype, const tlf_attn_chunk_args& a, int num_sms);
cudaError_t launch_chunk_attn(const ChunkDev& c, int dtype, const tlf_attn_chunk_args& a, void* scratch, int num_sms,
                              cudaStream_t st);

// The same under a window, or over a cache in 4 bits (c's page_elems then counts bytes).
size_t window_attn_scratch(const ChunkDev& c, int dtype, const tlf_attn_window_args& a, int num_sms);
cudaError_t launch_window_attn(const ChunkDev& c, int dtype, const tlf_attn_window_args& a, void* scratch, int num_sms,
                               cudaStream_t st);

size_t evict_scratch(const tlf_evict_args& a);
cudaError_t launch_evict(const tlf_evict_args& a, void* scratch, int num_sms, cudaStream_t st);

size_t fork_scratch(const tlf_fork_args& a);
cudaError_t launch_fork(const tlf_fork_args& a, void* scratch, int num_sms, cudaStream_t st);
size_t compact_scratch(const tlf_compact_args& a);
cudaError_t launch_compact(const tlf_compact_args& a, void* scratch, int num_sms, cudaStream_t st);

cudaError_t launch_sample(const tlf_sample_args& a, int num_sms, cudaStream_t st);

}  // namespace tlf
