// Attention of chunks of new tokens over paged caches (tlf_attn_chunk).
//
// A work item is a tile of queries of one row with the G query heads of one kv head (MMA or thread row r = query * G + head);
// its keys are the row's cache up to the tile's last query. The items' key blocks are dealt out evenly (k_chunk.cuh). A CTA
// runs an online softmax over its blocks of an item: running maximum m and sum l of 2^(s - m) (scores times log2 e), and
// O = sum 2^(s - m) v, all in float32. An item inside one CTA's share is written out; the parts of a shared one go to the
// scratch, and k_chunk_join adds them: M = max m_c, O = sum 2^(m_c - M) O_c / sum 2^(m_c - M) l_c.
//
// k_chunk_mma    bfloat16, up to 64 query rows a tile: tensor cores through mma.sync.
// k_chunk_simt   float32: tiles in shared memory, products on the CUDA cores.
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
  uint32_t* werr;  // error word of the waits: the caller's, or one in the scratch
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
// Tensor cores, few rows: mma.sync (bfloat16)
// ----------------------------------------------------------------------------
// A kv head's keys meet at most 64 query rows here, so a page's 2 x 64 x hd x rows products take less time than its bytes
// (a tcgen05 tile would be 128 rows of mostly padding and its scores a trip through tensor memory). A producer warp copies
// K and V of each page through a tensor map (128-byte swizzle; 64 at head_dim 32) into a ring; eight warps share it:
//   MT = 1 (up to 16 rows)  two teams of four warps take the pages in turn, each warp 16 of a page's keys,
//   MT = 2, 4 (32, 64 rows) warp w has rows 16 (w mod MT).. and 64 MT / 8 keys of every page.
// A warp keeps q as A fragments, m, l and O of its rows for its keys; scores and probabilities stay in registers (the score
// fragment is the A fragment of the second product). The running maximum is refreshed lazily: O is rescaled only when a row's
// maximum grows by more than 8 in base 2. At an item's end the warps' parts meet in shared memory.
//
// V of keys that no row of the tile sees is zeroed in the fragments (0 times an infinity is not 0). Keys that only some rows
// see can still spoil the others' O with a 0 x infinity: a row whose O is not finite is then done again by chunk_redo, over
// the keys that it sees alone.
template <int HD, int MT>
struct MmaShape {
  static constexpr int RT = 16 * MT, KS = 8 / MT, KW = MT == 4 ? 32 : 16;  // rows, key groups, keys of a warp in a page
  static constexpr int ROW = HD == 32 ? 64 : 128;        // bytes of a swizzled row
  static constexpr int ATOM = 64 * ROW, ATOMS = HD * 2 / ROW, SEG = ATOM * ATOMS, STAGE = 2 * SEG;
  static constexpr int PER_SM = HD == 128 ? 1 : 2;
  static constexpr int NST = HD == 128 ? 5 : HD == 64 ? 5 : 8;
  static constexpr int OS = HD + 8;                      // floats of a merge buffer's row
  static constexpr int OFF_O = NST * STAGE, OFF_ML = OFF_O + 4 * 16 * OS * 4, OFF_BAR = OFF_ML + KS * RT * 8,
                       OFF_INT = OFF_BAR + 2 * NST * 8, OFF_BASE = OFF_INT + (NST + 2 + 64 + 1) / 2 * 8;
  static int bytes(int n) { return OFF_BASE + (n + 1) * 8 + 1024; }
  static constexpr int THREADS = 288;
};

__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t a, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void mma_16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void bar_named(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

__device__ __forceinline__ bool finite4(float4 v) {
  return fabsf(v.x) < INFINITY && fabsf(v.y) < INFINITY && fabsf(v.z) < INFINITY && fabsf(v.w) < INFINITY;
}

// Query row (token, head) over entries e0 .. e1 - 1 of row b alone, by one warp: m (times log2 e), l and O.
template <int HD>
__device__ __noinline__ void chunk_redo(const ChunkAttn& a, int b, int h, long long token, int head, int e0, int e1, float& m,
                                        float& l, float (&o)[(HD + 31) / 32]) {
  constexpr int D = HD / 32;
  const int lane = threadIdx.x & 31;
  const bf16* q = static_cast<const bf16*>(a.q) + token * a.qs + (long long)head * HD;
  float qv[D];
#pragma unroll
  for (int d = 0; d < D; ++d) qv[d] = to_f32(q[lane + 32 * d]), o[d] = 0.f;
  m = -INFINITY;
  l = 0.f;
  for (int e = e0; e < e1; ++e) {
    const int page = a.c.page_table[(size_t)b * a.c.max_pages + e / 64];
    if (page < 0 || page >= a.c.n_pages) continue;
    const bf16* k = static_cast<const bf16*>(a.c.pool) + page * a.c.page_elems + ((long long)a.c.layer * 2 * a.c.Hkv + h) * 64 * HD + (e % 64) * HD;
    const bf16* v = k + (long long)a.c.Hkv * 64 * HD;
    float s = 0.f;
#pragma unroll
    for (int d = 0; d < D; ++d) s += qv[d] * to_f32(k[lane + 32 * d]);
    s = warp_sum(s) * a.scale;
    const float mn = fmaxf(m, s), ref = mn == -INFINITY ? 0.f : mn, cr = exp2f(m - ref), p = exp2f(s - ref);
    m = mn;
    l = l * cr + p;
#pragma unroll
    for (int d = 0; d < D; ++d) o[d] = o[d] * cr + p * to_f32(v[lane + 32 * d]);
  }
}

template <int HD, int MT>
__global__ void __launch_bounds__(288, MmaShape<HD, MT>::PER_SM) k_chunk_mma(ChunkAttn a,
                                                                             const __grid_constant__ CUtensorMap pool_map) {
  using Sh = MmaShape<HD, MT>;
  constexpr int NST = Sh::NST, KS = Sh::KS, KW = Sh::KW, NT = KW / 8, OS = Sh::OS;
  extern __shared__ uint8_t smem_raw[];
  __shared__ long long s_red[33];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* s_o = reinterpret_cast<float*>(sm + Sh::OFF_O);
  float2* s_ml = reinterpret_cast<float2*>(sm + Sh::OFF_ML);
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + Sh::OFF_BAR);
  volatile int* s_skip = reinterpret_cast<volatile int*>(sm + Sh::OFF_INT);  // [NST] the stage holds nothing to see
  volatile int* abort_flag = s_skip + NST;
  volatile int* s_any = s_skip + NST + 1;
  volatile int* s_bad = s_skip + NST + 2;  // [RT]
  long long* s_base = reinterpret_cast<long long*>(sm + Sh::OFF_BASE);
  auto full = [&](int st) { return smem_u32(&bars[st]); };
  auto empty = [&](int st) { return smem_u32(&bars[NST + st]); };
  const ChunkDev& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 8);
    }
    *abort_flag = 0;
    *s_any = 0;
    fence_barrier_init();
    prefetch_tensormap(&pool_map);
  }
  if (tid < Sh::RT) s_bad[tid] = 0;
  pdl_wait();
  chunk_plan(c, a.sp, s_base, s_red);
  const long long all = s_base[c.n], per = chunk_share(a, all);
  long long pos = blockIdx.x * per;
  const long long end = pos + per < all ? pos + per : all;
  const int G = c.G, qt = 1 << a.sp.qt_log;
  // a bounded wait; once one has run out, the others are skipped and everybody winds down
  auto wait = [&](uint32_t b, uint32_t parity) {
    if (*abort_flag) return false;
    if (mbar_wait(b, parity, a.werr)) return true;
    *abort_flag = 1;
    return false;
  };
  unsigned seq = 0;  // pages that this CTA's ring has taken

  if (warp == 8) {
    while (pos < end) {
      const ChunkItem it = chunk_item(c, a.sp, s_base, pos);
      const int kb0 = (int)(pos - it.first), kb1 = (int)(end - it.first < it.nb ? end - it.first : it.nb);
      const int rowK = (c.layer * 2 * c.Hkv + it.h) * 64, rowV = rowK + c.Hkv * 64;
      for (int g0 = kb0; g0 < kb1; g0 += 32) {
        int mine = -1;
        if (g0 + lane < kb1 && (g0 + lane) * 64 < it.len)
          mine = chunk_page(c.page_table, c.max_pages, c.n_pages, it.b, g0 + lane, c.err);
        for (int i = 0; i < min(32, kb1 - g0); ++i, ++seq) {
          const int page = __shfl_sync(0xffffffffu, mine, i), st = seq % NST;
          if (lane == 0) {
            const bool ok = seq < NST || wait(empty(st), (seq / NST - 1) & 1u);
            if (ok) {
              s_skip[st] = page < 0;
              if (page < 0) {
                mbar_arrive(full(st));
              } else {
                mbar_arrive_expect_tx(full(st), Sh::STAGE);
                const uint32_t dst = smem_u32(sm + st * Sh::STAGE);
#pragma unroll
                for (int x = 0; x < Sh::ATOMS; ++x) {
                  tma_load_3d(dst + x * Sh::ATOM, &pool_map, x * (Sh::ROW / 2), rowK, page, full(st));
                  tma_load_3d(dst + Sh::SEG + x * Sh::ATOM, &pool_map, x * (Sh::ROW / 2), rowV, page, full(st));
                }
              }
            }
          }
          __syncwarp();
        }
      }
      pos = it.first + kb1;
    }
    if (*abort_flag) drain_copies();
    pdl_trigger();
    return;
  }

  const int mt = warp % MT, grp = warp / MT, slice = MT == 1 ? grp & 3 : grp;
  const bool q_even = (reinterpret_cast<uintptr_t>(a.q) % 4 == 0) && a.qs % 2 == 0;
  // shared-memory offset of this lane's row of a fragment load: matrix i = lane / 8 has rows 8 (i / 2).. of keys and the
  // (i % 2)-th chunk of 8 dims (K), or rows 8 (i % 2).. and the (i / 2)-th chunk (V)
  const int kk = slice * KW + (lane >> 4) * 8 + (lane & 7), kc = (lane >> 3) & 1;
  const int vk = slice * KW + ((lane >> 3) & 1) * 8 + (lane & 7), vc = lane >> 4;
  constexpr int CH = Sh::ROW / 16;  // 16-byte chunks of a row
  auto swz = [](int key) { return HD == 32 ? (key >> 1) & 3 : key & 7; };
  while (pos < end) {
    const ChunkItem it = chunk_item(c, a.sp, s_base, pos);
    const int kb0 = (int)(pos - it.first), kb1 = (int)(end - it.first < it.nb ? end - it.first : it.nb);
    const int nq = min(qt, it.ql - it.t * qt), rows = nq * G;
    const int token0 = it.t0 + it.t * qt, see0 = it.s0 + it.t * qt, see_last = see0 + nq - 1;
    const int r0 = mt * 16 + (lane >> 2), r1 = r0 + 8;
    // rows past the tile's see what its first query sees, with q = 0; nobody reads them
    const int sees[2] = {see0 + (r0 < rows ? r0 / G : 0), see0 + (r1 < rows ? r1 / G : 0)};
    uint32_t qf[HD / 16][4];
    {
      const bf16* base = static_cast<const bf16*>(a.q) + (long long)(it.h * G) * HD + (lane & 3) * 2;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = x ? r1 : r0;
        const bf16* row = base + (token0 + r / G) * a.qs + (r % G) * HD;
#pragma unroll
        for (int k = 0; k < HD / 8; ++k) {
          uint32_t v = 0;
          if (r < rows) {
            if (q_even) {
              v = *reinterpret_cast<const uint32_t*>(row + k * 8);
            } else {
              v = (uint32_t)__bfloat16_as_ushort(row[k * 8]) | (uint32_t)__bfloat16_as_ushort(row[k * 8 + 1]) << 16;
            }
          }
          qf[k / 2][(k & 1) * 2 + x] = v;
        }
      }
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[HD / 8][4];
#pragma unroll
    for (int i = 0; i < HD / 8; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.f;

    for (int kb = kb0; kb < kb1; ++kb, ++seq) {
      // every warp waits for and releases every page, the other team's too: a stage may not be filled twice while a warp has
      // yet to look at its barrier, whose parity would then be the one before
      const int st = seq % NST;
      const bool ok = __all_sync(0xffffffffu, wait(full(st), (seq / NST) & 1u));
      const bool mine = MT > 1 || (int)(seq & 1u) == grp >> 2;
      const int key0 = kb * 64 + slice * KW;
      if (ok && mine && key0 <= see_last && !s_skip[st]) {
        const uint32_t sk = smem_u32(sm + st * Sh::STAGE), sv = sk + Sh::SEG;
        float s[NT][4];
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
#pragma unroll
          for (int g = 0; g < KW / 16; ++g) {
            uint32_t b[4];
            const int key = kk + g * 16, ch = 2 * k + kc;
            ldsm4(sk + (ch / CH) * Sh::ATOM + key * Sh::ROW + (((ch % CH) ^ swz(key)) << 4), b);
            mma_16816(s[2 * g], qf[k], b[0], b[1]);
            mma_16816(s[2 * g + 1], qf[k], b[2], b[3]);
          }
        const bool tail = key0 + KW - 1 > see0;
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] *= a.scale;
            if (tail && key0 + i * 8 + (lane & 3) * 2 + (j & 1) > sees[j >> 1]) s[i][j] = -INFINITY;
            mx[j >> 1] = fmaxf(mx[j >> 1], s[i][j]);
          }
        float cr[2] = {1.f, 1.f};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 1));
          mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 2));
          if (mx[x] > m[x] + 8.f) {
            cr[x] = ex2_fast(m[x] - mx[x]);
            m[x] = mx[x];
            l[x] *= cr[x];
          }
        }
        if (__any_sync(0xffffffffu, cr[0] != 1.f || cr[1] != 1.f)) {
#pragma unroll
          for (int i = 0; i < HD / 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] *= cr[j >> 1];
        }
        const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
        uint32_t p[KW / 16][4];
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float p0 = ex2_fast(s[i][2 * x] - ref[x]), p1 = ex2_fast(s[i][2 * x + 1] - ref[x]);
            l[x] += p0 + p1;
            p[i / 2][(i & 1) * 2 + x] = pack_bf16(p0, p1);
          }
        const bool cut = key0 + KW - 1 > see_last;
#pragma unroll
        for (int g = 0; g < KW / 16; ++g) {
          uint32_t keep[2] = {0xffffffffu, 0xffffffffu};
          if (cut) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int key = key0 + g * 16 + x * 8 + (lane & 3) * 2;
              keep[x] = (key <= see_last ? 0xffffu : 0u) | (key + 1 <= see_last ? 0xffff0000u : 0u);
            }
          }
#pragma unroll
          for (int d = 0; d < HD / 16; ++d) {
            uint32_t b[4];
            const int key = vk + g * 16, ch = 2 * d + vc;
            ldsm4_t(sv + (ch / CH) * Sh::ATOM + key * Sh::ROW + (((ch % CH) ^ swz(key)) << 4), b);
            if (cut) b[0] &= keep[0], b[1] &= keep[1], b[2] &= keep[0], b[3] &= keep[1];
            mma_16816(o[2 * d], p[g], b[0], b[1]);
            mma_16816(o[2 * d + 1], p[g], b[2], b[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }

    // the warps' parts: each to the item's maximum, the upper half of the key groups added to the lower, then all
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
      l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
      if ((lane & 3) == 0) s_ml[grp * Sh::RT + (x ? r1 : r0)] = make_float2(m[x], l[x]);
    }
    bar_named(1, 256);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float mm = -INFINITY;
#pragma unroll
      for (int g = 0; g < KS; ++g) mm = fmaxf(mm, s_ml[g * Sh::RT + (x ? r1 : r0)].x);
      const float f = ex2_fast(m[x] - (mm == -INFINITY ? 0.f : mm));
#pragma unroll
      for (int i = 0; i < HD / 8; ++i) o[i][2 * x] *= f, o[i][2 * x + 1] *= f;
    }
    float* buf = s_o + ((grp % (KS / 2)) * MT + mt) * 16 * OS + (lane >> 2) * OS + (lane & 3) * 2;
    auto put = [&] {
#pragma unroll
      for (int i = 0; i < HD / 8; ++i) {
        *reinterpret_cast<float2*>(buf + i * 8) = make_float2(o[i][0], o[i][1]);
        *reinterpret_cast<float2*>(buf + 8 * OS + i * 8) = make_float2(o[i][2], o[i][3]);
      }
    };
    if (grp >= KS / 2) put();
    bar_named(1, 256);
    if (grp < KS / 2) {
#pragma unroll
      for (int i = 0; i < HD / 8; ++i) {
        const float2 u = *reinterpret_cast<const float2*>(buf + i * 8), v = *reinterpret_cast<const float2*>(buf + 8 * OS + i * 8);
        o[i][0] += u.x, o[i][1] += u.y, o[i][2] += v.x, o[i][3] += v.y;
      }
      put();
    }
    bar_named(1, 256);
    const bool whole = kb0 == 0 && kb1 == it.nb;
    const size_t part = (size_t)(2 * blockIdx.x + (kb0 == 0)) * a.rows;
    auto row_ml = [&](int r) {
      float mm = -INFINITY, ll = 0.f;
#pragma unroll
      for (int g = 0; g < KS; ++g) mm = fmaxf(mm, s_ml[g * Sh::RT + r].x);
#pragma unroll
      for (int g = 0; g < KS; ++g) {
        const float2 ml = s_ml[g * Sh::RT + r];
        ll += ml.y * ex2_fast(ml.x - (mm == -INFINITY ? 0.f : mm));
      }
      return make_float2(mm, ll);
    };
    for (int i = tid; i < rows * (HD / 4); i += 256) {
      const int r = i / (HD / 4), d = (i % (HD / 4)) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int g = 0; g < KS / 2; ++g) {
        const float4 u = *reinterpret_cast<const float4*>(s_o + ((g * MT + r / 16) * 16 + r % 16) * OS + d);
        v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
      }
      if (nq > 1 && !finite4(v)) {
        s_bad[r] = 1;
        *s_any = 1;
      }
      const float2 ml = row_ml(r);
      if (whole) {
        const long long token = token0 + r / G;
        const int head = it.h * G + r % G;
        const float inv = ml.y != 0.f ? 1.f / ml.y : 0.f;
        bf16* out = static_cast<bf16*>(a.out) + token * a.os + (long long)head * HD + d;
        const uint32_t lo = pack_bf16(v.x * inv, v.y * inv), hi = pack_bf16(v.z * inv, v.w * inv);
        if (reinterpret_cast<uintptr_t>(out) % 8 == 0) {
          *reinterpret_cast<uint2*>(out) = make_uint2(lo, hi);
        } else {
          const uint32_t w[2] = {lo, hi};
#pragma unroll
          for (int e = 0; e < 4; ++e) out[e] = __ushort_as_bfloat16((unsigned short)(w[e / 2] >> (16 * (e & 1))));
        }
        if (d == 0 && a.lse) a.lse[token * c.Hq + head] = ml.y != 0.f ? (ml.x + log2f(ml.y)) * LN2 : -INFINITY;
      } else {
        *reinterpret_cast<float4*>(a.part_o + (part + r) * HD + d) = v;
        if (d == 0) a.part_ml[part + r] = ml;
      }
    }
    bar_named(1, 256);
    if (nq > 1 && *s_any) {
      for (int r = warp; r < rows; r += 8) {
        if (!s_bad[r]) continue;
        const long long token = token0 + r / G;
        const int head = it.h * G + r % G;
        float mm, ll, oo[HD / 32];
        chunk_redo<HD>(a, it.b, it.h, token, head, kb0 * 64, min(kb1 * 64, see0 + r / G + 1), mm, ll, oo);
        const float inv = !whole ? 1.f : ll != 0.f ? 1.f / ll : 0.f;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) {
          if (whole) static_cast<bf16*>(a.out)[token * a.os + (long long)head * HD + lane + 32 * d] = from_f32<bf16>(oo[d] * inv);
          else a.part_o[(part + r) * HD + lane + 32 * d] = oo[d];
        }
        if (lane == 0) {
          if (!whole) a.part_ml[part + r] = make_float2(mm, ll);
          else if (a.lse) a.lse[token * c.Hq + head] = ll != 0.f ? (mm + log2f(ll)) * LN2 : -INFINITY;
        }
      }
      bar_named(1, 256);
      if (tid < Sh::RT) s_bad[tid] = 0;
      if (tid == 0) *s_any = 0;
      bar_named(1, 256);
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
  size_t part_ml, lse, werr, total;  // scratch offsets (part_o at 0)
};
static int pow2_log(int x) {  // largest l with 2^l <= x
  int l = 0;
  while ((2 << l) <= x) ++l;
  return l;
}
static ChunkPath chunk_path(const ChunkDev& c, int dtype, const tlf_attn_chunk_args& a, int num_sms) {
  ChunkPath p{};
  const long long rows = (long long)c.max_chunk * c.G;  // of the longest chunk
  if (dtype == TLF_DTYPE_F32) {
    p.rt = rows <= 16 ? 16 : 64;
    p.ctas = 2 * num_sms;
  } else {
    p.rt = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
    p.ctas = (c.hd == 128 ? 1 : 2) * num_sms;
  }
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = (o + bytes + 255) / 256 * 256; return at; };
  take((size_t)2 * p.ctas * p.rt * c.hd * 4);
  p.part_ml = take((size_t)2 * p.ctas * p.rt * 8);
  p.lse = take(a.weight_out && !a.lse ? (size_t)c.T * c.Hq * 4 : 0);
  p.werr = take(4);
  p.total = o;
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
// 3-D map over the pool: {head_dim, rows of a page, pages}, boxes of 64 rows of one 128-byte (head_dim 32: 64-byte) column.
static bool pool_map(CUtensorMap* m, const ChunkDev& c) {
  const auto fn = tensor_map_encoder();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)c.hd, (cuuint64_t)c.J * 2 * c.Hkv * 64, (cuuint64_t)c.n_pages};
  cuuint64_t strides[2] = {(cuuint64_t)c.hd * 2, (cuuint64_t)c.page_elems * 2};
  cuuint32_t box[3] = {c.hd == 32 ? 32u : 64u, 64, 1}, es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, c.pool, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            c.hd == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <int HD, int MT>
static cudaError_t mma_launch(const ChunkAttn& a, cudaStream_t st) {
  CUtensorMap map;
  if (!pool_map(&map, a.c)) return cudaErrorInvalidValue;
  using Sh = MmaShape<HD, MT>;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_mma<HD, MT>), Sh::bytes(SV_MAX_ROWS))) return e;
  return launch_k(k_chunk_mma<HD, MT>, dim3(a.ctas), dim3(Sh::THREADS), Sh::bytes(a.c.n), st, a, map);
}
template <int HD>
static cudaError_t mma_rows(const ChunkAttn& a, cudaStream_t st) {
  return a.rows == 16 ? mma_launch<HD, 1>(a, st) : a.rows == 32 ? mma_launch<HD, 2>(a, st) : mma_launch<HD, 4>(a, st);
}
template <int HD>
static cudaError_t simt_rows(const ChunkAttn& a, cudaStream_t st) {
  return a.rows == 16 ? simt_launch<float, 16, HD>(a, st) : simt_launch<float, 64, HD>(a, st);
}
template <typename T>
static cudaError_t chunk_launch(const ChunkAttn& a, const tlf_attn_chunk_args& args, int num_sms, cudaStream_t st) {
  cudaError_t e;
  if (std::is_same<T, bf16>::value)
    e = a.c.hd == 32 ? mma_rows<32>(a, st) : a.c.hd == 64 ? mma_rows<64>(a, st) : mma_rows<128>(a, st);
  else
    e = a.c.hd == 16 ? simt_rows<16>(a, st) : a.c.hd == 32 ? simt_rows<32>(a, st) : a.c.hd == 64 ? simt_rows<64>(a, st) : simt_rows<128>(a, st);
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
  a.werr = c.err ? c.err : reinterpret_cast<uint32_t*>(s + p.werr);
  a.part_o = reinterpret_cast<float*>(s);
  a.part_ml = reinterpret_cast<float2*>(s + p.part_ml);
  return dtype == TLF_DTYPE_BF16 ? chunk_launch<bf16>(a, args, num_sms, st) : chunk_launch<float>(a, args, num_sms, st);
}

}  // namespace tlf
