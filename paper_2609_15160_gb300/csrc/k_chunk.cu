// Attention of chunks of new tokens over paged caches (tlf_attn_chunk).
//
// A work item is a tile of queries of one row with the G query heads of one kv head (MMA or thread row r = query * G + head);
// its keys are the row's cache up to the tile's last query. The items' key blocks are dealt out evenly (k_chunk.cuh). A CTA
// runs an online softmax over its blocks of an item: running maximum m and sum l of 2^(s - m) (scores times log2 e), and
// O = sum 2^(s - m) v, all in float32. An item inside one CTA's share is written out; the parts of a shared one go to the
// scratch, and k_chunk_join adds them: M = max m_c, O = sum 2^(m_c - M) O_c / sum 2^(m_c - M) l_c.
//
// k_chunk_simt   float32 caches: tiles in shared memory, products on the CUDA cores.
// k_chunk_weigh  with weights: adds up exp(s - lse) of every entry over the queries that see it.
#include <algorithm>
#include <type_traits>

#include "k_chunk.cuh"
#include "k_serve.cuh"

namespace tlf {

struct ChunkAttn {
  ChunkDev c;
  ChunkSplit sp;
  const void* q;
  long long qs;
  void* out;
  long long os;
  float* lse;      // [T][Hq] or NULL
  float scale;     // of the scores, times log2 e
  int ctas, rows;  // CTAs that share the blocks; rows of a part
  long long min_blocks;  // least share of a CTA
  float* part_o;   // [2 ctas][rows][hd]
  float2* part_ml; // [2 ctas][rows]
};

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// base[b] = blocks of the rows before b; base[n] = all. By the whole block.
__device__ __forceinline__ void chunk_plan(const ChunkDev& c, const ChunkSplit& sp, long long* base, long long* red) {
  long long carry = 0;
  for (int b0 = 0; b0 < c.n; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    long long u = 0;
    if (b < c.n) {
      const ChunkRow r = chunk_row(c, b);
      u = sp.before(r.len - r.ql, r.ql, sp.tiles(r.ql)) * c.Hkv;
    }
    long long total;
    const long long at = carry + block_scan(u, red, &total);
    if (b < c.n) base[b] = at;
    carry += total;
  }
  if (threadIdx.x == 0) base[c.n] = carry;
  __syncthreads();
}

__device__ __forceinline__ long long chunk_share(const ChunkAttn& a, long long all) {
  const long long per = (all + a.ctas - 1) / a.ctas;
  return per > a.min_blocks ? per : a.min_blocks;
}

// The item that holds block `pos` of the flat order.
struct ChunkItem {
  int b, h, t, nb;     // row, kv head, tile, its blocks
  int t0, s0, ql, len; // the row's first new token, old entries, new tokens, entries
  long long first;     // the item's first block in the flat order
};
__device__ __forceinline__ ChunkItem chunk_item(const ChunkDev& c, const ChunkSplit& sp, const long long* base, long long pos) {
  int lo = 0, hi = c.n;  // largest b with base[b] <= pos (rows without tokens have no blocks)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (base[mid] <= pos) lo = mid;
    else hi = mid;
  }
  const ChunkRow r = chunk_row(c, lo);
  ChunkItem it;
  it.b = lo;
  it.t0 = r.t0;
  it.ql = r.ql;
  it.len = r.len;
  it.s0 = r.len - r.ql;
  const long long rel = pos - base[lo], per = (base[lo + 1] - base[lo]) / c.Hkv;
  it.h = (int)(rel / per);
  const long long at = rel - it.h * per;
  it.t = sp.tile_of(it.s0, it.ql, at);
  it.nb = sp.blocks(it.s0, it.ql, it.t);
  it.first = base[lo] + it.h * per + sp.before(it.s0, it.ql, it.t);
  return it;
}

// ----------------------------------------------------------------------------
// Joining the parts of shared items
// ----------------------------------------------------------------------------
// blockIdx.x + 1 = a CTA whose share starts inside an item; the first such CTA of an item joins it. CTA c's first item has
// its part at 2c if it began in an earlier share, the part of an item that goes on past its share is at 2c + 1. A warp a row.
template <typename T>
__global__ void __launch_bounds__(256) k_chunk_join(ChunkAttn a) {
  pdl_wait();
  extern __shared__ long long s_base[];
  __shared__ long long s_red[33];
  chunk_plan(a.c, a.sp, s_base, s_red);
  const long long all = s_base[a.c.n], per = chunk_share(a, all), pos = (blockIdx.x + 1) * per;
  if (pos >= all) return;
  const ChunkItem it = chunk_item(a.c, a.sp, s_base, pos);
  if (it.first == pos || it.first / per != blockIdx.x) return;
  const int c0 = blockIdx.x, c1 = (int)((it.first + it.nb - 1) / per), parts = c1 - c0 + 1;
  const int qt = 1 << a.sp.qt_log, rows = min(qt, it.ql - it.t * qt) * a.c.G, lane = threadIdx.x & 31, hd = a.c.hd;
  const int row = blockIdx.y * 8 + (threadIdx.x >> 5);
  if (row >= rows) return;
  auto slot = [&](int i) { return (size_t)(i == 0 ? 2 * c0 + 1 : 2 * (c0 + i)) * a.rows + row; };
  float m = -INFINITY;
  for (int i = lane; i < parts; i += 32) m = fmaxf(m, a.part_ml[slot(i)].x);
  m = warp_max(m);
  float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < parts; i0 += 32) {
    float w = 0.f;
    if (i0 + lane < parts) {
      const float2 ml = a.part_ml[slot(i0 + lane)];
      w = exp2f(ml.x - (m == -INFINITY ? 0.f : m));
      l += w * ml.y;
    }
    const int n = min(32, parts - i0);
    for (int i = 0; i < n; ++i) {
      const float wi = __shfl_sync(0xffffffffu, w, i);
      const float* p = a.part_o + slot(i0 + i) * hd;
      if (wi != 0.f)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (lane + 32 * k < hd) o[k] += wi * p[lane + 32 * k];
    }
  }
  l = warp_sum(l);
  const int token = it.t0 + it.t * qt + row / a.c.G, head = it.h * a.c.G + row % a.c.G;
  T* out = static_cast<T*>(a.out) + token * a.os + (long long)head * hd;
  const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (lane + 32 * k < hd) out[lane + 32 * k] = from_f32<T>(o[k] * inv);
  if (lane == 0 && a.lse) a.lse[(long long)token * a.c.Hq + head] = l != 0.f ? (m + log2f(l)) * LN2 : -INFINITY;
}

// ----------------------------------------------------------------------------
// CUDA cores
// ----------------------------------------------------------------------------
template <int RT, int HD>
struct SimtShape {
  static constexpr int THREADS = 256, BK = 64, RW = RT / 16;  // rows of a thread
  static constexpr int DW = HD / 16, KS = HD + 4, PS = BK + 4;
  static constexpr int OFF_K = RT * HD, OFF_V = OFF_K + BK * KS, OFF_P = OFF_V + BK * HD, FLOATS = OFF_P + RT * PS;
  static int bytes(int n) { return FLOATS * 4 + (n + 1) * 8; }
};

// 16 lanes share a row: lane x has keys x, x + 16, .. of a block in the first product and dims DW x .. in the second, so a
// row's statistics and probabilities never leave its half warp.
template <typename T, int RT, int HD>
__global__ void __launch_bounds__(256) k_chunk_simt(ChunkAttn a) {
  using Sh = SimtShape<RT, HD>;
  constexpr int RW = Sh::RW, DW = Sh::DW, KS = Sh::KS, PS = Sh::PS;
  pdl_wait();
  extern __shared__ float4 smem4[];
  __shared__ long long s_red[33];
  float* sm = reinterpret_cast<float*>(smem4);
  float *sQ = sm, *sK = sm + Sh::OFF_K, *sV = sm + Sh::OFF_V, *sP = sm + Sh::OFF_P;
  long long* s_base = reinterpret_cast<long long*>(sm + Sh::FLOATS);
  const ChunkDev& c = a.c;
  chunk_plan(c, a.sp, s_base, s_red);
  const long long all = s_base[c.n], per = chunk_share(a, all);
  long long pos = blockIdx.x * per;
  const long long end = pos + per < all ? pos + per : all;
  const int tid = threadIdx.x, x = tid & 15, y = tid >> 4, G = c.G, qt = 1 << a.sp.qt_log;
  while (pos < end) {
    const ChunkItem it = chunk_item(c, a.sp, s_base, pos);
    const int kb0 = (int)(pos - it.first), kb1 = (int)(end - it.first < it.nb ? end - it.first : it.nb);
    const int nq = min(qt, it.ql - it.t * qt), rows = nq * G;
    const int token0 = it.t0 + it.t * qt, see0 = it.s0 + it.t * qt;  // the tile's first query sees entries 0..see0
    __syncthreads();
    for (int i = tid; i < RT * HD; i += 256) {
      const int r = i / HD, d = i % HD;
      float v = 0.f;
      if (r < rows)
        v = to_f32(static_cast<const T*>(a.q)[(token0 + r / G) * a.qs + (long long)(it.h * G + r % G) * HD + d]) * a.scale;
      sQ[i] = v;
    }
    int see[RW];
    float m[RW], l[RW], o[RW][DW];
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      const int r = y + 16 * i;
      see[i] = r < rows ? see0 + r / G : -1;
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int d = 0; d < DW; ++d) o[i][d] = 0.f;
    }
    for (int kb = kb0; kb < kb1; ++kb) {
      const int page = kb * 64 < it.len ? chunk_page(c.page_table, c.max_pages, c.n_pages, it.b, kb, c.err) : -1;
      if (page < 0) continue;  // nothing to see there
      const T* pk = static_cast<const T*>(c.pool) + page * c.page_elems + ((long long)c.layer * 2 * c.Hkv + it.h) * 64 * HD;
      const T* pv = pk + (long long)c.Hkv * 64 * HD;
      __syncthreads();
      constexpr int VEC = Vec16<T>::N;
      for (int i = tid * VEC; i < 64 * HD; i += 256 * VEC) {
        float kk[VEC], vv[VEC];
        Vec16<T>::load(pk + i, kk);
        Vec16<T>::load(pv + i, vv);
        float* dk = sK + (i / HD) * KS + i % HD;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          dk[e] = kk[e];
          sV[i + e] = vv[e];
        }
      }
      __syncthreads();
      float s[RW][4];
#pragma unroll
      for (int i = 0; i < RW; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
      for (int d = 0; d < HD; d += 4) {
        float4 kv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kv[j] = *reinterpret_cast<const float4*>(sK + (x + 16 * j) * KS + d);
#pragma unroll
        for (int i = 0; i < RW; ++i) {
          const float4 q = *reinterpret_cast<const float4*>(sQ + (y + 16 * i) * HD + d);
#pragma unroll
          for (int j = 0; j < 4; ++j) s[i][j] += q.x * kv[j].x + q.y * kv[j].y + q.z * kv[j].z + q.w * kv[j].w;
        }
      }
      int most = 64;  // keys that some row of this half warp sees, and whether all rows see all of them
      bool mixed = false;
#pragma unroll
      for (int i = 0; i < RW; ++i) {
        const int vis = see[i] - kb * 64;  // keys 0..vis of the block
        mixed |= vis < 63;
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (x + 16 * j > vis) s[i][j] = -INFINITY;
          mx = fmaxf(mx, s[i][j]);
        }
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : mn, cr = exp2f(m[i] - ref);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = x + 16 * j > vis ? 0.f : exp2f(s[i][j] - ref);
          sP[(y + 16 * i) * PS + x + 16 * j] = p;
          sum += p;
        }
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        l[i] = l[i] * cr + sum;
        m[i] = mn;
#pragma unroll
        for (int d = 0; d < DW; ++d) o[i][d] *= cr;
      }
      __syncwarp();
      if (!mixed) {
#pragma unroll 4
        for (int key = 0; key < most; ++key) {
          float v[DW];
#pragma unroll
          for (int d = 0; d < DW; ++d) v[d] = sV[key * HD + x * DW + d];
#pragma unroll
          for (int i = 0; i < RW; ++i) {
            const float p = sP[(y + 16 * i) * PS + key];
#pragma unroll
            for (int d = 0; d < DW; ++d) o[i][d] += p * v[d];
          }
        }
      } else {  // 0 times what a row may not see need not be 0
#pragma unroll
        for (int i = 0; i < RW; ++i) {
          const int vis = min(63, see[i] - kb * 64);
          for (int key = 0; key <= vis; ++key) {
            const float p = sP[(y + 16 * i) * PS + key];
#pragma unroll
            for (int d = 0; d < DW; ++d) o[i][d] += p * sV[key * HD + x * DW + d];
          }
        }
      }
    }
    const bool whole = kb0 == 0 && kb1 == it.nb;
    const size_t part = (size_t)(2 * blockIdx.x + (kb0 == 0)) * a.rows;
#pragma unroll
    for (int i = 0; i < RW; ++i) {
      const int r = y + 16 * i;
      if (r >= rows) continue;
      if (whole) {
        const long long token = token0 + r / G;
        const int head = it.h * G + r % G;
        const float inv = l[i] != 0.f ? 1.f / l[i] : 0.f;
        T* out = static_cast<T*>(a.out) + token * a.os + (long long)head * HD + x * DW;
#pragma unroll
        for (int d = 0; d < DW; ++d) out[d] = from_f32<T>(o[i][d] * inv);
        if (x == 0 && a.lse) a.lse[token * c.Hq + head] = l[i] != 0.f ? (m[i] + log2f(l[i])) * LN2 : -INFINITY;
      } else {
#pragma unroll
        for (int d = 0; d < DW; ++d) a.part_o[(part + r) * HD + x * DW + d] = o[i][d];
        if (x == 0) a.part_ml[part + r] = make_float2(m[i], l[i]);
      }
    }
    pos = it.first + kb1;
  }
  pdl_trigger();
}

// ----------------------------------------------------------------------------
// Weights
// ----------------------------------------------------------------------------
// An item is a page of a row, with all heads and all queries that see one of its entries; one writer an entry, and a fixed
// order of the sums. Four threads a key, each with every fourth query row.
template <typename T, int HD>
__global__ void __launch_bounds__(256) k_chunk_weigh(ChunkAttn a, const float* w_in, float* w_out) {
  constexpr int KS = HD + 4, QR = HD == 128 ? 16 : 32;
  pdl_wait();
  extern __shared__ long long s_base[];
  __shared__ long long s_red[33];
  __shared__ __align__(16) float sK[64 * KS];
  __shared__ __align__(16) float sQ[QR * HD];
  __shared__ float s_lse[QR];
  __shared__ int s_see[QR];
  __shared__ float s_sum[4][64];
  const ChunkDev& c = a.c;
  const int tid = threadIdx.x, key = tid & 63, part = tid >> 6, G = c.G;
  long long carry = 0;
  for (int b0 = 0; b0 < c.n; b0 += 256) {
    const int b = b0 + tid;
    long long total;
    const long long pages = b < c.n ? (chunk_row(c, b).len + 63) / 64 : 0, at = carry + block_scan(pages, s_red, &total);
    if (b < c.n) s_base[b] = at;
    carry += total;
  }
  if (tid == 0) s_base[c.n] = carry;
  __syncthreads();
  for (long long item = blockIdx.x; item < carry; item += gridDim.x) {
    int lo = 0, hi = c.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_base[mid] <= item) lo = mid;
      else hi = mid;
    }
    const int pg = (int)(item - s_base[lo]), page = chunk_page(c.page_table, c.max_pages, c.n_pages, lo, pg, c.err);
    if (page < 0) continue;
    const ChunkRow r = chunk_row(c, lo);
    const int s0 = r.len - r.ql, e0 = pg * 64, i0 = max(0, e0 - s0), rows = (r.ql - i0) * G;  // queries i0.. see entry e0
    float sum = 0.f;
    for (int h = 0; h < c.Hkv && rows > 0; ++h) {
      const T* pk = static_cast<const T*>(c.pool) + page * c.page_elems + ((long long)c.layer * 2 * c.Hkv + h) * 64 * HD;
      __syncthreads();
      for (int i = tid; i < 64 * HD; i += 256) sK[(i / HD) * KS + i % HD] = to_f32(pk[i]);
      for (int r0 = 0; r0 < rows; r0 += QR) {
        const int nr = min(QR, rows - r0);
        __syncthreads();
        for (int i = tid; i < nr * HD; i += 256) {
          const int q = i0 + (r0 + i / HD) / G, g = (r0 + i / HD) % G;
          sQ[i] = to_f32(static_cast<const T*>(a.q)[(long long)(r.t0 + q) * a.qs + (long long)(h * G + g) * HD + i % HD]) * a.scale;
        }
        if (tid < nr) {
          const int q = i0 + (r0 + tid) / G, g = (r0 + tid) % G;
          s_lse[tid] = a.lse[(long long)(r.t0 + q) * c.Hq + h * G + g] * LOG2E;
          s_see[tid] = s0 + q;
        }
        __syncthreads();
        for (int i = part; i < nr; i += 4) {
          float s = 0.f;
#pragma unroll 8
          for (int d = 0; d < HD; d += 4) {
            const float4 q = *reinterpret_cast<const float4*>(sQ + i * HD + d), k = *reinterpret_cast<const float4*>(sK + key * KS + d);
            s += q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
          }
          if (e0 + key <= s_see[i]) sum += exp2f(s - s_lse[i]);
        }
      }
    }
    __syncthreads();
    s_sum[part][key] = sum;
    __syncthreads();
    if (tid < 64 && e0 + tid < r.len) {
      const long long at = (long long)page * 64 + tid;
      w_out[at] = (w_in ? w_in[at] : 0.f) + ((s_sum[0][tid] + s_sum[1][tid]) + (s_sum[2][tid] + s_sum[3][tid]));
    }
  }
  pdl_trigger();
}

// ----------------------------------------------------------------------------
// Launches
// ----------------------------------------------------------------------------
// Which kernel and split a call takes; a function of the arguments and the device alone.
struct ChunkPath {
  int rt;       // rows of a tile
  int ctas;
  size_t part_ml, lse, total;  // scratch offsets (part_o at 0)
};
static int pow2_log(int x) {  // largest l with 2^l <= x
  int l = 0;
  while ((2 << l) <= x) ++l;
  return l;
}
static ChunkPath chunk_path(const ChunkDev& c, int dtype, const tlf_attn_chunk_args& a, int num_sms) {
  ChunkPath p{};
  p.rt = (long long)c.max_chunk * c.G <= 16 ? 16 : 64;
  p.ctas = 2 * num_sms;
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = (o + bytes + 255) / 256 * 256; return at; };
  take((size_t)2 * p.ctas * p.rt * c.hd * 4);
  p.part_ml = take((size_t)2 * p.ctas * p.rt * 8);
  p.lse = take(a.weight_out && !a.lse ? (size_t)c.T * c.Hq * 4 : 0);
  p.total = std::max<size_t>(o, 256);
  return p;
}
size_t chunk_attn_scratch(const ChunkDev& c, int dtype, const tlf_attn_chunk_args& a, int num_sms) {
  return chunk_path(c, dtype, a, num_sms).total;
}

template <typename T, int RT, int HD>
static cudaError_t simt_launch(const ChunkAttn& a, cudaStream_t st) {
  const int smem = SimtShape<RT, HD>::bytes(a.c.n);
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_simt<T, RT, HD>), SimtShape<RT, HD>::bytes(SV_MAX_ROWS)))
    return e;
  return launch_k(k_chunk_simt<T, RT, HD>, dim3(a.ctas), dim3(256), smem, st, a);
}
template <typename T>
static cudaError_t chunk_launch(const ChunkAttn& a, const tlf_attn_chunk_args& args, int num_sms, cudaStream_t st) {
  cudaError_t e = cudaErrorInvalidValue;
  switch (a.c.hd) {
    case 16: e = a.rows == 16 ? simt_launch<T, 16, 16>(a, st) : simt_launch<T, 64, 16>(a, st); break;
    case 32: e = a.rows == 16 ? simt_launch<T, 16, 32>(a, st) : simt_launch<T, 64, 32>(a, st); break;
    case 64: e = a.rows == 16 ? simt_launch<T, 16, 64>(a, st) : simt_launch<T, 64, 64>(a, st); break;
    case 128: e = a.rows == 16 ? simt_launch<T, 16, 128>(a, st) : simt_launch<T, 64, 128>(a, st); break;
  }
  if (e) return e;
  const int base = (a.c.n + 1) * 8;
  if (cudaError_t j = launch_k(k_chunk_join<T>, dim3(a.ctas - 1, (a.rows + 7) / 8), dim3(256), base, st, a)) return j;
  if (!args.weight_out) return cudaSuccess;
  const dim3 grid(4 * num_sms);
  switch (a.c.hd) {
    case 16: return launch_k(k_chunk_weigh<T, 16>, grid, dim3(256), base, st, a, args.weight_in, args.weight_out);
    case 32: return launch_k(k_chunk_weigh<T, 32>, grid, dim3(256), base, st, a, args.weight_in, args.weight_out);
    case 64: return launch_k(k_chunk_weigh<T, 64>, grid, dim3(256), base, st, a, args.weight_in, args.weight_out);
    case 128: {
      if (cudaError_t x = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_weigh<T, 128>), (SV_MAX_ROWS + 1) * 8)) return x;
      return launch_k(k_chunk_weigh<T, 128>, grid, dim3(256), base, st, a, args.weight_in, args.weight_out);
    }
  }
  return cudaErrorInvalidValue;
}

cudaError_t launch_chunk_attn(const ChunkDev& c, int dtype, const tlf_attn_chunk_args& args, void* scratch, int num_sms,
                              cudaStream_t st) {
  const ChunkPath p = chunk_path(c, dtype, args, num_sms);
  char* s = static_cast<char*>(scratch);
  ChunkAttn a{};
  a.c = c;
  a.sp = ChunkSplit{pow2_log(std::max(1, p.rt / c.G)), 6};
  a.q = args.q;
  a.qs = args.q_stride ? args.q_stride : (long long)c.Hq * c.hd;
  a.out = args.out;
  a.os = args.out_stride ? args.out_stride : (long long)c.Hq * c.hd;
  a.lse = args.lse ? args.lse : args.weight_out ? reinterpret_cast<float*>(s + p.lse) : nullptr;
  a.scale = (args.scale != 0.f ? args.scale : 1.f / sqrtf((float)c.hd)) * LOG2E;
  a.ctas = p.ctas;
  a.rows = p.rt;
  a.min_blocks = 1;
  a.part_o = reinterpret_cast<float*>(s);
  a.part_ml = reinterpret_cast<float2*>(s + p.part_ml);
  return dtype == TLF_DTYPE_BF16 ? chunk_launch<bf16>(a, args, num_sms, st) : chunk_launch<float>(a, args, num_sms, st);
}

}  // namespace tlf
