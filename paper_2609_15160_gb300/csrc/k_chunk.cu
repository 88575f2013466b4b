// Attention of chunks of new tokens over paged caches (tlf_attn_chunk), under a window (tlf_attn_window), in 4 bits.
//
// A work item is a tile of queries of one row with the G query heads of one kv head (MMA or thread row r = query * G + head);
// its keys are the row's cache up to the tile's last query. The items' key blocks are dealt out evenly (k_chunk.cuh). A CTA
// runs an online softmax over its blocks of an item: running maximum m and sum l of 2^(s - m) (scores times log2 e), and
// O = sum 2^(s - m) v, all in float32. An item inside one CTA's share is written out; the parts of a shared one go to the
// scratch, and k_chunk_join adds them: M = max m_c, O = sum 2^(m_c - M) O_c / sum 2^(m_c - M) l_c.
//
// k_chunk_pair   bfloat16, more than 16 or 32 query rows an item: tcgen05 on pairs of 128-row tiles.
// k_chunk_mma    bfloat16, fewer rows, and what the tiles of the other do not fit: tensor cores through mma.sync.
// k_chunk_simt   float32: tiles in shared memory, products on the CUDA cores.
// With weights, exp(s - lse) of every entry added up over the queries that see it:
// k_weigh_tc            more than 16 rows: S^T again on tcgen05, a thread a key;
// k_chunk_weigh_scores  from the scores that k_chunk_mma leaves;
// k_chunk_weigh         the rest, on the CUDA cores.
#include <algorithm>

#include "k_chunk4.cuh"
#include "k_chunk_dev.cuh"
#include "k_kv4.cuh"

namespace tlf {

// ----------------------------------------------------------------------------
// Joining the parts of shared items
// ----------------------------------------------------------------------------
// A warp takes a row at a time, VW dims a lane (hd = 32 VW, or 16 with VW = 1), and every eight-th row of a CTA's. It reads the
// notes rather than plan again, which took 3 us.
template <typename T, int VW>
__global__ void __launch_bounds__(256) k_chunk_join(ChunkAttn a) {
  pdl_trigger();
  pdl_wait();
  const int4 note = a.join[blockIdx.x + 1];
  const int parts = note.w;
  if (parts == 0) return;
  const int c0 = blockIdx.x, G = a.c.G, rows = note.z, lane = threadIdx.x & 31, hd = a.c.hd;
  const bool mine = lane * VW < hd;
  auto slot = [&](int i, int row) { return (size_t)(i == 0 ? 2 * c0 + 1 : 2 * (c0 + i)) * a.rows + row; };
  auto get = [&](int i, int row, float (&v)[VW]) {
    const float* p = a.part_o + slot(i, row) * hd + lane * VW;
    if (VW == 4) *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(p);
    else if (VW == 2) *reinterpret_cast<float2*>(v) = *reinterpret_cast<const float2*>(p);
    else v[0] = *p;
  };
  auto put = [&](int row, float m, float l, const float (&o)[VW]) {
    const int token = note.x + row / G, head = note.y * G + row % G;
    T* out = static_cast<T*>(a.out) + token * a.os + (long long)head * hd + lane * VW;
    const float inv = l != 0.f ? 1.f / l : 0.f;
    if (mine)
#pragma unroll
      for (int k = 0; k < VW; ++k) out[k] = from_f32<T>(o[k] * inv);
    if (lane == 0 && a.lse) a.lse[(long long)token * a.c.Hq + head] = l != 0.f ? (m + log2f(l)) * LN2 : -INFINITY;
  };
  const int first = blockIdx.y * 8 + (threadIdx.x >> 5), step = gridDim.y * 8;
  if (parts == 2) {  // the usual case: U rows in flight, statistics and sums together
    constexpr int U = 4;
    for (int r0 = first; r0 < rows; r0 += U * step) {
      float2 x[U], y[U];
      float u[U][VW], v[U][VW];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int row = r0 + k * step;
        if (row >= rows) break;
        x[k] = a.part_ml[slot(0, row)];
        y[k] = a.part_ml[slot(1, row)];
        if (mine) {
          get(0, row, u[k]);
          get(1, row, v[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int row = r0 + k * step;
        if (row >= rows) break;
        const float m = fmaxf(x[k].x, y[k].x), ref = m == -INFINITY ? 0.f : m, wx = exp2f(x[k].x - ref), wy = exp2f(y[k].x - ref);
        float o[VW];
#pragma unroll
        for (int d = 0; d < VW; ++d) o[d] = (wx != 0.f ? wx * u[k][d] : 0.f) + (wy != 0.f ? wy * v[k][d] : 0.f);
        put(row, m, wx * x[k].y + wy * y[k].y, o);
      }
    }
    return;
  }
  for (int row = first; row < rows; row += step) {
    float m = -INFINITY, l = 0.f, o[VW];
#pragma unroll
    for (int k = 0; k < VW; ++k) o[k] = 0.f;
    for (int i = lane; i < parts; i += 32) m = fmaxf(m, a.part_ml[slot(i, row)].x);
    m = warp_max(m);
    const float ref = m == -INFINITY ? 0.f : m;
    for (int i0 = 0; i0 < parts; i0 += 32) {
      float w = 0.f;
      if (i0 + lane < parts) {
        const float2 ml = a.part_ml[slot(i0 + lane, row)];
        w = exp2f(ml.x - ref);
        l += w * ml.y;
      }
      constexpr int U = 4;
      for (int i = 0; i < min(32, parts - i0); i += U) {
        float v[U][VW];
#pragma unroll
        for (int k = 0; k < U; ++k)
          if (mine && i0 + i + k < parts) get(i0 + i + k, row, v[k]);
#pragma unroll
        for (int k = 0; k < U; ++k) {
          const float wi = __shfl_sync(0xffffffffu, w, i + k);
          if (mine && i0 + i + k < parts && wi != 0.f)
#pragma unroll
            for (int d = 0; d < VW; ++d) o[d] += wi * v[k][d];
        }
      }
    }
    put(row, m, warp_sum(l), o);
  }
}

// The parts of k_chunk_pair: a warp has 8 rows and half the dims, a lane one row and every fourth 16 bytes of it.
template <int HD>
__global__ void __launch_bounds__(256) k_pair_join(ChunkAttn a) {  // grid y = 8
  pdl_trigger();
  pdl_wait();
  const int4 note = a.join[blockIdx.x + 1];
  const int parts = note.w, c0 = blockIdx.x, G = a.c.G, lane = threadIdx.x & 31, quarter = lane >> 3;
  const int unit = blockIdx.y * 8 + (threadIdx.x >> 5), row = (unit & 31) * 8 + (lane & 7), d0 = (unit >> 5) * (HD / 2) + quarter * 4;
  if (parts == 0 || (unit & 31) * 8 >= note.z) return;
  constexpr int V = HD / 32;  // 16-byte pieces of a lane
  auto slot = [&](int i) { return i == 0 ? 2 * c0 + 1 : 2 * (c0 + i); };
  auto stat = [&](int i) { return a.part_ml[(size_t)slot(i) * PAIR_ROWS + row]; };
  auto get = [&](int i, float4 (&v)[V]) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = *reinterpret_cast<const float4*>(a.part_o + pair_part(slot(i), row, d0 + 16 * k, HD));
  };
  float4 o[V], v[V];
  const float2 x = stat(0), y = stat(1);
  get(0, o);
  get(1, v);
  float m = fmaxf(x.x, y.x);
  for (int i = 2 + quarter; i < parts; i += 4) m = fmaxf(m, stat(i).x);
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
  m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
  const float ref = m == -INFINITY ? 0.f : m, wx = exp2f(x.x - ref), wy = exp2f(y.x - ref);
  auto scaled = [](float w, float4 u) { return w != 0.f ? make_float4(w * u.x, w * u.y, w * u.z, w * u.w) : make_float4(0.f, 0.f, 0.f, 0.f); };
  auto add = [](float4& s, float4 u) { s.x += u.x, s.y += u.y, s.z += u.z, s.w += u.w; };
  float l = wx * x.y + wy * y.y;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    o[k] = scaled(wx, o[k]);
    add(o[k], scaled(wy, v[k]));
  }
#pragma unroll 4
  for (int i = 2; i < parts; ++i) {
    const float2 ml = stat(i);
    get(i, v);
    const float w = exp2f(ml.x - ref);
    l += w * ml.y;
#pragma unroll
    for (int k = 0; k < V; ++k) add(o[k], scaled(w, v[k]));
  }
  if (row >= note.z) return;
  const int token = note.x + row / G, head = note.y * G + row % G;
  const float inv = l != 0.f ? 1.f / l : 0.f;
  bf16* out = static_cast<bf16*>(a.out) + token * a.os + (long long)head * HD + d0;
  const bool wide = reinterpret_cast<uintptr_t>(a.out) % 8 == 0 && a.os % 4 == 0;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    if (wide) {
      *reinterpret_cast<uint2*>(out + 16 * k) = make_uint2(pack_bf16(o[k].x * inv, o[k].y * inv), pack_bf16(o[k].z * inv, o[k].w * inv));
    } else {
      const float e[4] = {o[k].x, o[k].y, o[k].z, o[k].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) out[16 * k + j] = from_f32<bf16>(e[j] * inv);
    }
  }
  if (d0 == 0 && a.lse) a.lse[(long long)token * a.c.Hq + head] = l != 0.f ? (m + log2f(l)) * LN2 : -INFINITY;
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
// row's statistics and probabilities never leave its half warp. Bound by launch and first loads on the models it serves
// (4 rows of up to 5 tokens over up to 60 entries, 4 heads x 16: 8 us with the join, in a CUDA graph).
template <typename T, int RT, int HD, int MODE>
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
  const auto sp = split_of<MODE>(a);
  chunk_plan(c, sp, s_base, s_red);
  pdl_trigger();
  const long long all = s_base[c.n], per = chunk_share(a, all);
  long long pos = blockIdx.x * per;
  const long long end = pos + per < all ? pos + per : all;
  const int tid = threadIdx.x, x = tid & 15, y = tid >> 4, G = c.G, qt = 1 << a.sp.qt_log;
  if (pos >= end && tid == 0) join_note(a, nullptr, per);
  for (bool first = true; pos < end; first = false) {
    const ChunkItem it = chunk_item(c, sp, s_base, pos);
    if (first && tid == 0) join_note(a, &it, per);
    if (pos < it.first) pos = it.first;
    if (pos >= end) break;
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
    int sinks = 0;
    if constexpr (MODE != KEYS_ALL) sinks = sp.sinks();
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
    for (int i = kb0; i < kb1; ++i) {
      const int kb = block_at<MODE>(i, sinks, it.skip);
      const int page = kb * 64 < it.len ? chunk_page(c.page_table, c.max_pages, c.n_pages, it.b, kb, c.err) : -1;
      if (page < 0) continue;  // nothing to see there
      __syncthreads();
      constexpr int VEC = MODE == KEYS_4BIT ? 8 : Vec16<T>::N;
      for (int i = tid * VEC; i < 64 * HD; i += 256 * VEC) {
        float kk[VEC], vv[VEC];
        if constexpr (MODE == KEYS_4BIT) {
          using F = Kv4<HD>;
          const uint8_t* pk = static_cast<const uint8_t*>(c.pool) + page * c.page_elems + ((long long)c.layer * 2 * c.Hkv + it.h) * F::BLOCK;
          const uint8_t* pv = pk + (long long)c.Hkv * F::BLOCK;
          const int pair = F::CODES + ((i / HD) * F::NG + i % HD / F::GS) * 4;
          kv4_values(*reinterpret_cast<const uint32_t*>(pk + i / 2), kv4_pair(*reinterpret_cast<const uint32_t*>(pk + pair)), kk);
          kv4_values(*reinterpret_cast<const uint32_t*>(pv + i / 2), kv4_pair(*reinterpret_cast<const uint32_t*>(pv + pair)), vv);
        } else {
          const T* pk = static_cast<const T*>(c.pool) + page * c.page_elems + ((long long)c.layer * 2 * c.Hkv + it.h) * 64 * HD;
          Vec16<T>::load(pk + i, kk);
          Vec16<T>::load(pk + (long long)c.Hkv * 64 * HD + i, vv);
        }
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
        // but for those from past..low: hidden by the window and not among the first
        const int past = MODE == KEYS_ALL ? 64 : a.first - kb * 64, low = MODE == KEYS_ALL ? -1 : hidden_to(see[i], a.window) - kb * 64;
        auto hidden = [&](int key) { return key > vis || (MODE != KEYS_ALL && key >= past && key <= low); };
        mixed |= vis < 63 || (MODE != KEYS_ALL && low >= 0 && past < 64);
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (hidden(x + 16 * j)) s[i][j] = -INFINITY;
          mx = fmaxf(mx, s[i][j]);
        }
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : mn, cr = exp2f(m[i] - ref);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = hidden(x + 16 * j) ? 0.f : exp2f(s[i][j] - ref);
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
          const int past = a.first - kb * 64, low = hidden_to(see[i], a.window) - kb * 64;
          for (int key = 0; key <= vis; ++key) {
            if (MODE != KEYS_ALL && key >= past && key <= low) continue;
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
}

// ----------------------------------------------------------------------------
// Tensor cores, few rows: mma.sync (bfloat16)
// ----------------------------------------------------------------------------
// A kv head's keys meet few query rows here (up to 64 where k_chunk_pair's tiles do not fit the heads or q), so a page's 2 x 64 x
// hd x rows products take about as long as its bytes or less, and a tcgen05 tile would be 128 rows of mostly padding. A producer warp copies
// K and V of each page through a tensor map (128-byte swizzle; 64 at head_dim 32) into a ring; eight warps share it:
//   MT = 1 (up to 16 rows)  two teams of four warps take the pages in turn, each warp 16 of a page's keys,
//   MT = 2, 4 (32, 64 rows) warp w has rows 16 (w mod MT).. and 64 MT / 8 keys of every page.
// A warp keeps q as A fragments, m, l and O of its rows for its keys; scores and probabilities stay in registers (the score
// fragment is the A fragment of the second product). The running maximum is refreshed lazily: O is rescaled only when a row's
// maximum grows by more than 8 in base 2. At an item's end the warps' parts meet in shared memory.
//
// P is rounded to bf16, the type of the second product's operands (as in k_chunk_pair; l adds up P before the rounding).
//
// 0 times an infinity is not 0: V of keys that no row of the tile sees is zeroed in the fragments, and so are elements that are
// not finite of keys that only some rows see. Those rows get them from chunk_left_out at the item's end.
//
// Bound by HBM: 16 single tokens over 32k entries, 16 / 8 heads x 128: 311 us with the join, 6.8 TB/s (0.99 of the copy rate);
// 32 over up to 8192 entries, 16 heads x 64: 105 us, 5.7 TB/s, the rest of it ramp, items' ends and the join.
struct MmaSeg {  // a CTA's part of an item: blocks kb0 .. kb1 - 1 of nb
  long long first;  // the item's first block in the flat order
  int b, h, token0, see0, nq, kb0, kb1, nb;
  static constexpr int RING = 16;
};
template <int HD, int MT>
struct MmaShape {
  static constexpr int RT = 16 * MT, KS = 8 / MT, KW = MT == 4 ? 32 : 16;  // rows, key groups, keys of a warp in a page
  static constexpr int ROW = HD == 32 ? 64 : 128;        // bytes of a swizzled row
  static constexpr int ATOM = 64 * ROW, ATOMS = HD * 2 / ROW, SEG = ATOM * ATOMS, STAGE = 2 * SEG;
  static constexpr int PER_SM = HD == 128 ? 1 : 2;
  static constexpr int NST = HD == 128 ? 5 : HD == 64 ? 5 : 8;
  static constexpr int OS = HD + 8;                      // floats of a merge buffer's row
  static constexpr int OFF_O = NST * STAGE, OFF_ML = OFF_O + 4 * 16 * OS * 4, OFF_BAR = OFF_ML + KS * RT * 8,
                       OFF_INT = OFF_BAR + 2 * NST * 8, OFF_SEG = OFF_INT + (NST + 2 + 1) / 2 * 8,
                       OFF_BASE = OFF_SEG + MmaSeg::RING * (int)sizeof(MmaSeg);
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
// 0xffff for each half that is an infinity or NaN of bfloat16.
__device__ __forceinline__ uint32_t bf16x2_not_finite(uint32_t v) { return __vcmpeq2(v & 0x7f807f80u, 0x7f807f80u); }

// Entries e .. e1 - 1 of row b, new tokens that some queries of a tile see and others do not: adds to x the elements of V that are
// not finite, which the tile's products left out. A query that sees the entries has p > 0 for each of them, so that its sums plus
// x are what the formula gives: infinities and NaN. By one warp; a lane has dims lane * HD / 32 .. Later queries see what earlier
// ones do: a warp goes over its rows in order and goes on with x.
template <int HD>
__device__ __noinline__ void chunk_left_out(const ChunkAttn& a, int b, int h, int& e, int e1, float (&x)[HD / 32]) {
  constexpr int D = HD / 32, U = 8;  // in flight
  const bf16* pv = static_cast<const bf16*>(a.c.pool) + ((long long)(a.c.layer * 2 + 1) * a.c.Hkv + h) * 64 * HD + (threadIdx.x & 31) * D;
  for (; e < e1; e = min(e + U, e1)) {
    float f[U][D];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int page = e + u < e1 ? a.c.page_table[(size_t)b * a.c.max_pages + (e + u) / 64] : -1;
      const bool there = page >= 0 && page < a.c.n_pages;
#pragma unroll
      for (int d = 0; d < D; ++d) f[u][d] = there ? to_f32(pv[page * a.c.page_elems + ((e + u) % 64) * HD + d]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int d = 0; d < D; ++d)
        if (!(fabsf(f[u][d]) < INFINITY)) x[d] += f[u][d];
  }
}

// The same under a window, for one row of a tile: a query at entry `see` of a tile with queries see0 .. see_last, in the item's blocks
// kb0 .. kb1 - 1. Left out were the entries from `first` on that the last query no longer sees, and the new tokens'. What one row
// sees does not hold what another one does: x starts from zero.
template <int HD>
__device__ __noinline__ void window_left_out(const ChunkAttn& a, int b, int h, int see, int see0, int see_last, int kb0, int kb1, int sinks,
                                             int skip, float (&x)[HD / 32]) {
  const int low = hidden_to(see, a.window) + 1;
  auto scan = [&](int lo, int hi) {  // entries lo .. hi of the blocks
    int e = max(lo, kb0 * 64);
    chunk_left_out<HD>(a, b, h, e, min(hi, min(kb1, sinks) * 64 - 1) + 1, x);
    e = max(lo, (max(kb0, sinks) + skip) * 64);
    if (kb1 > sinks) chunk_left_out<HD>(a, b, h, e, min(hi, (kb1 + skip) * 64 - 1) + 1, x);
  };
  scan(max(a.first, low), min(see0, hidden_to(see_last, a.window)));
  scan(see0 + 1, min(see, a.first - 1));
  scan(max(see0 + 1, max(a.first, low)), see);
}

template <int HD, int MT, int MODE>
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
  volatile int* s_any = s_skip + NST + 1;  // something was left out of the item's products
  MmaSeg* s_seg = reinterpret_cast<MmaSeg*>(sm + Sh::OFF_SEG);
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
  pdl_wait();
  const auto sp = split_of<MODE>(a);
  int sinks = 0;
  if constexpr (MODE != KEYS_ALL) sinks = sp.sinks();
  chunk_plan(c, sp, s_base, s_red);
  pdl_trigger();
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
    if (pos >= end && lane == 0) join_note(a, nullptr, per);
    for (unsigned segs = 0; pos < end; ++segs) {
      const ChunkItem it = chunk_item(c, sp, s_base, pos);
      if (segs == 0 && lane == 0) join_note(a, &it, per);
      if (pos < it.first) pos = it.first;
      if (pos >= end) {
        if (segs == 0 && lane == 0) {
          s_seg[0].nb = 0;
          mbar_arrive(full(0));
        }
        break;
      }
      const int kb0 = (int)(pos - it.first), kb1 = (int)(end - it.first < it.nb ? end - it.first : it.nb);
      // the consumers find the item here when they see its first page
      if (lane == 0) s_seg[segs % MmaSeg::RING] = MmaSeg{it.first, it.b, it.h, it.t0 + it.t * qt, it.s0 + it.t * qt, min(qt, it.ql - it.t * qt), kb0, kb1, it.nb};
      const int rowK = (c.layer * 2 * c.Hkv + it.h) * 64, rowV = rowK + c.Hkv * 64;
      for (int g0 = kb0; g0 < kb1; g0 += 32) {
        int mine = -1;
        const int at = block_at<MODE>(g0 + lane, sinks, it.skip);
        if (g0 + lane < kb1 && at * 64 < it.len) mine = chunk_page(c.page_table, c.max_pages, c.n_pages, it.b, at, c.err);
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
  bool go = pos < end;
  for (unsigned segs = 0; go; ++segs) {
    // the item is written before its first page's barrier is armed; the ring of pages keeps the producer less than RING ahead.
    // The warps leave together or not at all: they meet at barriers below, which know no time limit
    if (bar_any(1, 256, !wait(full(seq % NST), (seq / NST) & 1u))) break;
    const MmaSeg it = s_seg[segs % MmaSeg::RING];
    if (it.nb == 0) break;  // this share is all pad
    const int kb0 = it.kb0, kb1 = it.kb1, nq = it.nq, rows = nq * G, token0 = it.token0, see0 = it.see0, see_last = see0 + nq - 1;
    const int r0 = mt * 16 + (lane >> 2), r1 = r0 + 8;
    // rows past the tile's see what its first query sees, with q = 0; nobody reads them
    const int sees[2] = {see0 + (r0 < rows ? r0 / G : 0), see0 + (r1 < rows ? r1 / G : 0)};
    // under a window: the entries from `first` up to hid are hidden, from all queries up to gone_to
    int skip = 0, hid[2] = {-1, -1}, gone_to = -1, edge_to = -1;
    if constexpr (MODE != KEYS_ALL) {
      skip = sp.skip_at(see0);
      hid[0] = hidden_to(sees[0], a.window);
      hid[1] = hidden_to(sees[1], a.window);
      gone_to = hidden_to(see0, a.window);
      edge_to = hidden_to(see_last, a.window);
    }
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
      const int key0 = block_at<MODE>(kb, sinks, skip) * 64 + slice * KW;
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
        const bool tail = key0 + KW - 1 > see0 || (MODE != KEYS_ALL && key0 <= edge_to && key0 + KW - 1 >= a.first);
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] *= a.scale;
            const int key = key0 + i * 8 + (lane & 3) * 2 + (j & 1);
            if (tail && (key > sees[j >> 1] || (MODE != KEYS_ALL && key >= a.first && key <= hid[j >> 1]))) s[i][j] = -INFINITY;
            mx[j >> 1] = fmaxf(mx[j >> 1], s[i][j]);
          }
        if (a.scores) {
          const long long width = (long long)c.max_pages * 64;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int r = x ? r1 : r0;
            if (r >= rows) continue;
            float* to = a.scores + ((long long)(token0 + r / G) * c.Hq + it.h * G + r % G) * width + key0 + (lane & 3) * 2;
#pragma unroll
            for (int i = 0; i < NT; ++i) *reinterpret_cast<float2*>(to + i * 8) = make_float2(s[i][2 * x], s[i][2 * x + 1]);
          }
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
        auto products = [&](auto masked) {
#pragma unroll
          for (int g = 0; g < KW / 16; ++g) {
            uint32_t keep[2], look[2];  // keys that some row sees; and some do not
            if constexpr (masked) {
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const int key = key0 + g * 16 + x * 8 + (lane & 3) * 2;
                auto seen = [&](int k) { return k <= see_last && (MODE == KEYS_ALL || k < a.first || k > gone_to); };
                auto mixed = [&](int k) { return k > see0 || (MODE != KEYS_ALL && k >= a.first && k <= edge_to); };
                keep[x] = (seen(key) ? 0xffffu : 0u) | (seen(key + 1) ? 0xffff0000u : 0u);
                look[x] = keep[x] & ((mixed(key) ? 0xffffu : 0u) | (mixed(key + 1) ? 0xffff0000u : 0u));
              }
            }
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) {
              uint32_t b[4];
              const int key = vk + g * 16, ch = 2 * d + vc;
              ldsm4_t(sv + (ch / CH) * Sh::ATOM + key * Sh::ROW + (((ch % CH) ^ swz(key)) << 4), b);
              if constexpr (masked) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  b[x] &= keep[x & 1];
                  const uint32_t out = bf16x2_not_finite(b[x]) & look[x & 1];
                  b[x] &= ~out;
                  if (out) *s_any = 1;
                }
              }
              mma_16816(o[2 * d], p[g], b[0], b[1]);
              mma_16816(o[2 * d + 1], p[g], b[2], b[3]);
            }
          }
        };
        if (tail) products(std::true_type{});
        else products(std::false_type{});
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
    if (nq > 1 && *s_any) {  // (written before the barriers above)
      bar_named(1, 256);     // the rows are written
      float x[HD / 32] = {};
      int e = max(kb0 * 64, see0 + 1);
      for (int r = warp; r < rows; r += 8) {
        if constexpr (MODE == KEYS_ALL) {
          chunk_left_out<HD>(a, it.b, it.h, e, min(kb1 * 64, see0 + r / G + 1), x);
        } else {
#pragma unroll
          for (int d = 0; d < HD / 32; ++d) x[d] = 0.f;
          window_left_out<HD>(a, it.b, it.h, see0 + r / G, see0, see_last, kb0, kb1, sinks, skip, x);
        }
        bf16* out = static_cast<bf16*>(a.out) + (token0 + r / G) * a.os + (long long)(it.h * G + r % G) * HD + lane * (HD / 32);
        float* po = a.part_o + (part + r) * HD + lane * (HD / 32);
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) {
          if (x[d] == 0.f) continue;
          if (whole) out[d] = from_f32<bf16>(to_f32(out[d]) + x[d]);
          else po[d] += x[d];
        }
      }
      bar_named(1, 256);
      if (tid == 0) *s_any = 0;
      bar_named(1, 256);
    }
    // the next item lies behind its pad
    go = kb1 == it.nb && it.first + it.nb + a.sp.pad < end;
  }
}

// ----------------------------------------------------------------------------
// Tensor cores, many rows: tcgen05 (bfloat16, head_dim 64 and 128)
// ----------------------------------------------------------------------------
// One CTA an SM. An item is two tiles of 128 MMA rows (row = query * G + head) that share every block of 64 keys (a page):
//   warps 0-3, 4-7  softmax of tile 0 and 1, one thread a row: S from tensor memory, mask, running maximum (refreshed lazily)
//                   and sum in float32, P in bf16 back to tensor memory, where it is the A operand of P V; at the end O out;
//   warp 8          producer: q of both tiles, then K and V of every block, through tensor maps;
//   warps 9, 10     issue S = Q K^T and O += P V (V taken as an MN-major operand) of tile 0 and 1: at a block of 64 keys one
//                   thread for both was slower than the tensor cores (2.0k to 2.5k cycles a block);
//   warp 11         makes V fit for the products, as below.
// P = 0 does not cancel an infinity: in blocks with keys that some of the item's queries do not see, warp 11 zeroes V of keys
// behind the last query and elements that are not finite of the new tokens' V before the products read them. The rows that see
// such a token get its infinities and NaN from chunk_left_out at the item's end.
// Tensor memory: O of both tiles (head_dim columns each) and two S buffers of 64 columns a tile; P overwrites its S. One
// thread's MMAs run in order, so S of block i + 2 is issued right behind the P V of block i that reads the buffer, and the
// softmax of block i + 1 finds its S ready when it is done with block i. With blocks of 128 keys there is room for one S a tile
// only: a tile's chain S, softmax, P V was then 4.8k cycles a block, 2.0k of them MMAs (4 x 2048 tokens over up to 10240
// entries, 16 / 8 heads x 128: 485 us, 343 so at first).
//
// P is rounded to bf16 because the second product takes 16-bit operands of one type: with P in two bf16 terms it would be two
// products. l adds up P before the rounding. Against 64 bits the output is then off by 2.3e-3 where it is off by 1.7e-3 with P in
// float32, most of which is the rounding of the output itself.
//
// What bounds it: the softmax warps' chain from S to P. A block of 64 keys and two tiles takes 1410 cycles at head_dim 128 and 1340
// at 64, of which the tensor pipe works 990 and 510; the exponentials (32 a cycle and SM) are 512, and nearly half of the issue
// slots are taken. Products and sums of two floats at a time took 10 us off 362: the issue slots count. Exponentials by polynomials
// beside the unit's made it slower. Warp 11 instead of the softmax warps for V (134.5 us there, 132 so and with no look at V at all:
// 4 x 1000 tokens with weights) has 16 keys in flight (four: 139). With the join: 327 us for the case above in single calls (1455
// TFLOP/s, 0.76 of the measured bf16 rate; 371 to 386 in a long loop, where the clock falls), 284 us with 16 heads x 64 (838), 195 us
// for 8192 causal tokens (1405).
//
// Under a window (MODE) the same on a band: 4 x 2048 tokens, window 1024, 16 / 8 heads x 128: 89 us (730 TFLOP/s): an
// item has 20 blocks, so that its ends, which the loop does not hide, weigh more than in a whole cache.
constexpr int PAIR_THREADS = 384;

template <int HD>
struct PairShape {
  static constexpr int ATOMS = HD / 64, QCOL = 128 * 128, Q_BYTES = ATOMS * QCOL;  // a tile of 128 rows of q
  static constexpr int COL = 64 * 128, T_BYTES = ATOMS * COL;                      // 64 rows of K or V
  static constexpr int NST = HD == 128 ? 4 : 8;  // of the K ring and of the V ring
  static constexpr int OFF_K = 2 * Q_BYTES, OFF_V = OFF_K + NST * T_BYTES, OFF_BAR = OFF_V + NST * T_BYTES;
  static constexpr int NBAR = 5 * NST + 2 + 4 + 4 + 4 + 1 + 2 * PairSeg::RING;
  static constexpr int FLAGS = 16;  // more than the blocks that the producer can be ahead of the softmax
  static constexpr int OFF_INT = OFF_BAR + NBAR * 8, OFF_SEG = OFF_INT + (FLAGS + 4 + PairSeg::RING) * 4;
  static constexpr int OFF_BASE = OFF_SEG + PairSeg::RING * (int)sizeof(PairSeg);
  static int bytes(int n) { return std::max(OFF_BASE + (n + 1) * 8 + 1024, tmem_min_smem(512)); }
  static constexpr uint32_t OCOL = 256;
};

template <int HD, int MODE>
__global__ void __launch_bounds__(PAIR_THREADS, 1) k_chunk_pair(ChunkAttn a, int g_log, const __grid_constant__ CUtensorMap q_map,
                                                                const __grid_constant__ CUtensorMap pool_map) {
  using Sh = PairShape<HD>;
  constexpr int NST = Sh::NST;
  extern __shared__ uint8_t smem_raw[];
  __shared__ long long s_red[33];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + Sh::OFF_BAR);
  volatile int* s_flag = reinterpret_cast<volatile int*>(sm + Sh::OFF_INT);  // the block's page is not there
  volatile int* abort_flag = s_flag + Sh::FLAGS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + Sh::OFF_INT) + Sh::FLAGS + 1;
  // [RING] the last item (its number in this CTA) that had something left out of its products
  volatile unsigned* s_left = reinterpret_cast<volatile unsigned*>(sm + Sh::OFF_INT) + Sh::FLAGS + 4;
  PairSeg* s_seg = reinterpret_cast<PairSeg*>(sm + Sh::OFF_SEG);
  long long* s_base = reinterpret_cast<long long*>(sm + Sh::OFF_BASE);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  // block b of this CTA: its place in the rings, and the use's parity
  auto k_full = [&](unsigned b) { return bar(b % NST); };
  auto k_empty = [&](unsigned b) { return bar(NST + b % NST); };
  auto v_full = [&](unsigned b) { return bar(2 * NST + b % NST); };
  auto v_empty = [&](unsigned b) { return bar(3 * NST + b % NST); };
  auto q_full = [&](int x) { return bar(4 * NST + x); };
  // block n of tile x: S written, P written, P V done; a barrier for even and one for odd blocks, since up to two phases may pass
  // before the other side looks (S of block n is issued behind the P V of block n - 2: by then that one's barrier is free)
  auto s_full = [&](int x, unsigned n) { return bar(4 * NST + 2 + 2 * x + (n & 1)); };
  auto p_full = [&](int x, unsigned n) { return bar(4 * NST + 6 + 2 * x + (n & 1)); };
  auto o_done = [&](int x, unsigned n) { return bar(4 * NST + 10 + 2 * x + (n & 1)); };
  const uint32_t q_free = bar(4 * NST + 14);
  // V of block b fit for the products, where that needs a look. One barrier a stage: its next phase lies behind both issuers'
  // release of this use, so neither can find two phases gone by, which a parity does not tell from none
  auto v_tail = [&](unsigned b) { return bar(4 * NST + 15 + b % NST); };
  auto seg_full = [&](unsigned i) { return bar(5 * NST + 15 + i % PairSeg::RING); };
  auto seg_empty = [&](unsigned i) { return bar(5 * NST + 15 + PairSeg::RING + i % PairSeg::RING); };
  const ChunkDev& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(k_full(i), 1);
      mbar_init(k_empty(i), 2);
      mbar_init(v_full(i), 1);
      mbar_init(v_empty(i), 3);
      mbar_init(v_tail(i), 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(q_full(x), 1);
      for (unsigned n = 0; n < 2; ++n) {
        mbar_init(s_full(x, n), 1);
        mbar_init(p_full(x, n), 4);
        mbar_init(o_done(x, n), 1);
      }
    }
    mbar_init(q_free, 2);
    for (unsigned i = 0; i < PairSeg::RING; ++i) {
      mbar_init(seg_full(i), 1);
      mbar_init(seg_empty(i), 11);  // the other warps
      s_left[i] = ~0u;
    }
    *abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&q_map);
    prefetch_tensormap(&pool_map);
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  pdl_wait();
  const auto sp = split_of<MODE>(a);
  int sinks = 0;
  if constexpr (MODE != KEYS_ALL) sinks = sp.sinks();
  chunk_plan(c, sp, s_base, s_red);
  tc_fence_before();
  __syncthreads();  // barriers initialised, tensor memory allocated
  tc_fence_after();
  pdl_trigger();  // not before: a dependent CTA on this SM could take the columns that warp 9 still waits for
  const uint32_t tmem = *tmem_slot;
  const long long all = s_base[c.n], per = chunk_share(a, all);
  long long pos = blockIdx.x * per;
  const long long end = pos + per < all ? pos + per : all;
  const int qt_log = a.sp.qt_log, QT = 1 << (qt_log - 1);  // queries of a tile
  // a bounded wait; once any role has given up, the others skip their waits and wind down
  auto wait = [&](uint32_t b, uint32_t parity) {
    if (mbar_try_wait(b, parity & 1u)) return true;
    if (*abort_flag) return false;
    if (mbar_wait(b, parity & 1u, a.werr)) return true;
    *abort_flag = 1;
    return false;
  };
  PairSeg s;
  unsigned segs = 0;  // read or published
  auto skip_of = [&](int see0) {  // of the item whose first query is at entry see0
    if constexpr (MODE == KEYS_ALL) return 0;
    else return sp.skip_at(see0);
  };
  // does block kb of a row hold keys that some of the queries at entries see0 .. see_last see and others do not, or nobody?
  auto partly_seen = [&](int kb, int see0, int see_last) {
    return kb * 64 + 63 > see0 || (MODE != KEYS_ALL && kb * 64 <= hidden_to(see_last, a.window) && kb * 64 + 63 >= a.first);
  };

  if (warp == 8) {
    // ---------------- producer ----------------
    // finds the items and publishes them
    unsigned blk = 0;
    ChunkItem it{};
    for (bool ok = true;;) {
      s.nb = 0;
      if (pos < end) {
        chunk_item_next(c, sp, s_base, pos, it);
        if (segs == 0 && lane == 0) join_note(a, &it, per);
        if (pos < it.first) pos = it.first;
      } else if (segs == 0 && lane == 0) {
        join_note(a, nullptr, per);
      }
      if (pos < end) {
        const int q0 = it.t << qt_log, left = it.ql - q0;
        s = PairSeg{it.b, it.h, it.t0 + q0, it.s0 + q0, {}, {}, (int)(pos - it.first), (int)(end - it.first < it.nb ? end - it.first : it.nb), it.nb, 0};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          s.nq[x] = max(0, min(QT, left - x * QT));
          const int last = s.see0 + x * QT + s.nq[x] - 1;  // entry of the tile's last query
          const int nb = s.nq[x] > 0 ? (last < 0 ? 1 : last / 64 + 1 - it.skip) : 0;
          s.e[x] = max(0, min(s.kb1, nb) - s.kb0);
        }
        pos = it.first + s.kb1;
      }
      if (lane == 0) {
        ok = ok && (segs < PairSeg::RING || wait(seg_empty(segs), segs / PairSeg::RING - 1));
        if (ok) {
          s_seg[segs % PairSeg::RING] = s;
          mbar_arrive(seg_full(segs));
        }
      }
      if (s.nb == 0) break;
      const int E = s.kb1 - s.kb0;
      if (lane == 0) {
        ok = ok && (segs == 0 || wait(q_free, segs - 1));
        for (int x = 0; x < 2; ++x) {
          if (!ok || s.e[x] == 0) continue;
          mbar_arrive_expect_tx(q_full(x), Sh::Q_BYTES);
#pragma unroll
          for (int k = 0; k < Sh::ATOMS; ++k)
            tma_load_3d(smem_u32(sm + x * Sh::Q_BYTES + k * Sh::QCOL), &q_map, k * 64, s.h << g_log, s.token0 + x * QT, q_full(x));
        }
      }
      const int rowK = (c.layer * 2 * c.Hkv + s.h) * 64, rowV = rowK + c.Hkv * 64;
      for (int g0 = 0; g0 < E; g0 += 32) {
        int mine = -1;  // the pages of 32 blocks, one a lane; for one that is not there K is left as it is, V is zeros
        const int at = block_at<MODE>(s.kb0 + g0 + lane, sinks, it.skip);
        if (g0 + lane < E && at * 64 < it.len) mine = chunk_page(c.page_table, c.max_pages, c.n_pages, s.b, at, c.err);
        for (int i = 0; i < min(32, E - g0); ++i, ++blk) {
          const int page = __shfl_sync(0xffffffffu, mine, i);
          if (lane == 0 && ok) {
            ok = blk < NST || wait(k_empty(blk), blk / NST - 1);
            if (ok) {
              s_flag[blk % Sh::FLAGS] = page < 0;
              if (page < 0) {
                mbar_arrive(k_full(blk));
              } else {
                mbar_arrive_expect_tx(k_full(blk), Sh::T_BYTES);
#pragma unroll
                for (int k = 0; k < Sh::ATOMS; ++k)
                  tma_load_3d(smem_u32(sm + Sh::OFF_K + (blk % NST) * Sh::T_BYTES + k * Sh::COL), &pool_map, k * 64, rowK, page, k_full(blk));
              }
              ok = blk < NST || wait(v_empty(blk), blk / NST - 1);
            }
            if (ok && page >= 0) {
              mbar_arrive_expect_tx(v_full(blk), Sh::T_BYTES);
#pragma unroll
              for (int k = 0; k < Sh::ATOMS; ++k)
                tma_load_3d(smem_u32(sm + Sh::OFF_V + (blk % NST) * Sh::T_BYTES + k * Sh::COL), &pool_map, k * 64, rowV, page, v_full(blk));
            }
          }
          __syncwarp();
          if (page < 0 && __shfl_sync(0xffffffffu, (int)ok, 0)) {  // P = 0 does not cancel an infinity
            uint4* v = reinterpret_cast<uint4*>(sm + Sh::OFF_V + (blk % NST) * Sh::T_BYTES);
            for (int k = lane; k < Sh::T_BYTES / 16; k += 32) v[k] = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(v_full(blk));
          }
        }
      }
      ++segs;
    }
  } else if (warp == 11) {
    // ---------------- V of keys that not every query sees ----------------
    // (every block is waited for and released, so that no phase goes by unseen)
    auto wait_w = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, wait(b, parity)); };
    unsigned b = 0;
    for (bool ok = true; ok && wait_w(seg_full(segs), segs / PairSeg::RING); ++segs) {
      s = s_seg[segs % PairSeg::RING];
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(segs));
      if (s.nb == 0) break;
      const int behind = s.see0 + s.nq[0] + s.nq[1];  // no query sees entries from here on
      const int skip = skip_of(s.see0);
      // nor, under a window, those from `first` up to gone_to; those up to edge_to not all queries
      const int gone_to = MODE == KEYS_ALL ? -1 : hidden_to(s.see0, a.window), edge_to = MODE == KEYS_ALL ? -1 : hidden_to(behind - 1, a.window);
      for (int i = s.kb0; i < s.kb1; ++i, ++b) {
        const int kb = block_at<MODE>(i, sinks, skip);
        if (!wait_w(v_full(b), b / NST)) { ok = false; break; }
        if (partly_seen(kb, s.see0, behind - 1)) {
          bool wrote = false;
          uint4* v = reinterpret_cast<uint4*>(sm + Sh::OFF_V + (b % NST) * Sh::T_BYTES) + lane;
          const bool edge = MODE != KEYS_ALL && kb * 64 <= edge_to;
          for (int r0 = edge ? 0 : max(0, s.see0 + 1 - kb * 64) & ~15; r0 < 64; r0 += 16) {  // 16 keys; four of them take the warp's lanes
            uint4 u[4][Sh::ATOMS];
            uint32_t any = 0;  // the sign bits: exponents that are all ones
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int k = 0; k < Sh::ATOMS; ++k) u[i][k] = v[(r0 + 4 * i) * 8 + k * (Sh::COL / 16)];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int k = 0; k < Sh::ATOMS; ++k)
                any |= ((u[i][k].x & 0x7f807f80u) + 0x00800080u) | ((u[i][k].y & 0x7f807f80u) + 0x00800080u) |
                       ((u[i][k].z & 0x7f807f80u) + 0x00800080u) | ((u[i][k].w & 0x7f807f80u) + 0x00800080u);
            if (!(any & 0x80008000u) && kb * 64 + r0 + 15 < behind) continue;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = kb * 64 + r0 + 4 * i + (lane >> 3);
#pragma unroll
              for (int k = 0; k < Sh::ATOMS; ++k) {  // (a row keeps its place in the swizzle)
                const uint4 w = u[i][k], out = make_uint4(bf16x2_not_finite(w.x), bf16x2_not_finite(w.y), bf16x2_not_finite(w.z), bf16x2_not_finite(w.w));
                uint4& at = v[(r0 + 4 * i) * 8 + k * (Sh::COL / 16)];
                const bool hides = MODE != KEYS_ALL && key >= a.first;
                if (key >= behind || (hides && key <= gone_to)) {
                  at = make_uint4(0, 0, 0, 0);
                  wrote = true;
                } else if ((key > s.see0 || (hides && key <= edge_to)) && (out.x | out.y | out.z | out.w)) {
                  at = make_uint4(w.x & ~out.x, w.y & ~out.y, w.z & ~out.z, w.w & ~out.w);
                  s_left[segs % PairSeg::RING] = segs;
                  wrote = true;
                }
              }
            }
          }
          if (wrote) fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(v_tail(b));
        }
        if (lane == 0) mbar_arrive(v_empty(b));
      }
    }
  } else if (warp >= 9) {
    // ---------------- MMA issuers, one a tile ----------------
    if (elect_one()) {
      constexpr uint32_t IDS = idesc_bf16_f32(128, 64), IDO = idesc_bf16_f32_bmn(128, HD);
      constexpr uint64_t QCOL_E = Sh::QCOL >> 4, T_E = Sh::T_BYTES >> 4, COL_E = Sh::COL >> 4, V16_E = 2048 >> 4;
      const int x = warp - 9;
      const uint64_t qd = smem_desc_sw128(smem_u32(sm + x * Sh::Q_BYTES)), dk = smem_desc_sw128(smem_u32(sm + Sh::OFF_K));
      const uint64_t dv = smem_desc_sw128_mn(smem_u32(sm + Sh::OFF_V), Sh::COL);
      const uint32_t t_s = tmem + 128u * x, t_o = tmem + Sh::OCOL + (uint32_t)(HD * x);
      unsigned blk = 0, tails = 0, qn = 0, n = 0;  // tails: a bit a stage, v_tail's parity; n: blocks of the tile whose P V has been issued
      auto issue_s = [&](unsigned b, unsigned n) {
        const uint64_t kd = dk + (uint64_t)(b % NST) * T_E;
#pragma unroll
        for (int kc = 0; kc < Sh::ATOMS; ++kc)
#pragma unroll
          for (int k = 0; k < 4; ++k)  // K = 16 an MMA: +32 bytes (encoded +2) inside the atom column
            tc_mma_f16(t_s + 64u * (n & 1), qd + kc * QCOL_E + 2 * k, kd + kc * COL_E + 2 * k, IDS, (kc | k) ? 1u : 0u);
        tc_commit(s_full(x, n));
      };
      bool ok = true;
      auto next = [&] {
        if (!wait(seg_full(segs), segs / PairSeg::RING)) return false;
        s = s_seg[segs % PairSeg::RING];
        mbar_arrive(seg_empty(segs));
        ++segs;
        return s.nb > 0;
      };
      while (ok && next()) {
        const int E = s.kb1 - s.kb0, e = x ? s.e[1] : s.e[0], skip = skip_of(s.see0), see_last = s.see0 + s.nq[0] + s.nq[1] - 1;
        ok = e == 0 || wait(q_full(x), qn++);
        for (int i = 0; i < min(2, E) && ok; ++i) {  // S of the first two blocks
          ok = wait(k_full(blk + i), (blk + i) / NST);
          if (!ok) break;
          tc_fence_after();
          if (i < e) issue_s(blk + i, n + i);
          tc_commit(k_empty(blk + i));
        }
        if (ok && E <= 2) tc_commit(q_free);
        for (int i = 0; i < E && ok; ++i) {
          const unsigned b = blk + i;
          const bool more = i + 2 < E, tail = partly_seen(block_at<MODE>(s.kb0 + i, sinks, skip), s.see0, see_last);
          // (what this tile does not use it waits for and releases all the same, in step with the other)
          ok = wait(v_full(b), b / NST) && (!tail || wait(v_tail(b), tails >> b % NST)) &&
               (!more || wait(k_full(b + 2), (b + 2) / NST)) && (i >= e || wait(p_full(x, n), n >> 1));
          if (!ok) break;
          if (tail) tails ^= 1u << b % NST;
          if (i < e) {
            tc_fence_after();
            const uint64_t vd = dv + (uint64_t)(b % NST) * T_E;
#pragma unroll
            for (int k = 0; k < 4; ++k)  // K = 16 keys an MMA: 8 columns of P, +2048 bytes (16 rows) of V
              mma_ts(t_o, t_s + 64u * (n & 1) + 8u * k, vd + V16_E * k, IDO, i > 0 || k > 0 ? 1u : 0u);
            tc_commit(o_done(x, n));
            if (i + 2 < e) issue_s(b + 2, n + 2);
            ++n;
          }
          tc_commit(v_empty(b));
          if (more) tc_commit(k_empty(b + 2));
          if (i + 3 == E) tc_commit(q_free);
        }
        blk += E;
        }
    }
    __syncwarp();
  } else {
    // ---------------- softmax: thread = MMA row = TMEM lane ----------------
    const int x = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_off = (uint32_t)(quad * 32) << 16;
    const uint32_t t_s = tmem + lane_off + 128u * (uint32_t)x;
    const uint32_t t_o = tmem + lane_off + Sh::OCOL + (uint32_t)(HD * x);
    const int qi = row >> g_log, g = row & ((1 << g_log) - 1);
    unsigned n = 0, blk = 0;  // blocks of this tile, and of the CTA
    bool ok = true;
    // waits taken by the whole warp: the TMEM accesses after them are warp-collective
    auto wait_w = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, wait(b, parity)); };
    auto next = [&] {
      if (!wait_w(seg_full(segs), segs / PairSeg::RING)) return false;
      s = s_seg[segs % PairSeg::RING];
      ++segs;
      return s.nb > 0;
    };
    while (ok && next()) {
      const bool row_ok = qi < s.nq[x];
      const int see = row_ok ? s.see0 + x * QT + qi : -1;  // a row past the tile's queries sees nothing
      const int see0 = s.see0 + x * QT;                    // of the tile's first query
      const int skip = skip_of(s.see0), see_last = see0 + s.nq[x] - 1, hid = MODE == KEYS_ALL ? -1 : hidden_to(see, a.window);
      float m_run = -INFINITY, l_run = 0.f, scale = a.scale;  // m in units of the raw scores; scale: smaller where m is large
      for (int i = 0; i < s.e[x]; ++i, ++n) {
        if (!wait_w(s_full(x, n), n >> 1)) { ok = false; break; }
        tc_fence_after();
        const int key0 = block_at<MODE>(s.kb0 + i, sinks, skip) * 64;
        const uint32_t t_sn = t_s + 64u * (n & 1);
        uint32_t su[64];
        tmem_ld_32_issue(t_sn, su);
        tmem_ld_32_issue(t_sn + 32, su + 32);
        const bool gone = s_flag[(blk + i) % Sh::FLAGS] != 0;
        tmem_ld_wait();
        if constexpr (MODE == KEYS_ALL) {
          if (key0 + 63 > see0 || gone || !__all_sync(0xffffffffu, row_ok)) {
            const int vis = gone ? -1 : see - key0;  // columns 0..vis are visible
#pragma unroll
            for (int k = 0; k < 64; ++k)
              if (k > vis) su[k] = 0xff800000u;  // -inf
          }
        } else if (partly_seen(key0 / 64, see0, see_last) || gone) {
          // columns 0..see - key0 are visible, but for first - key0..hid - key0 (elsewhere a row past the tile's queries may take what
          // its q gives: nobody reads it)
          const uint64_t m = gone ? 0 : low_bits(see - key0 + 1) & (low_bits(a.first - key0) | ~low_bits(hid - key0 + 1));
          const uint32_t bits[2] = {(uint32_t)m, (uint32_t)(m >> 32)};
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (!(bits[k / 32] & (1u << (k % 32)))) su[k] = 0xff800000u;  // -inf
        }
        float pm4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int k = 0; k < 64; ++k) pm4[k & 3] = fmaxf(pm4[k & 3], __uint_as_float(su[k]));
        const float pm = fmaxf(fmaxf(pm4[0], pm4[1]), fmaxf(pm4[2], pm4[3]));
        // O is rescaled only when a row's maximum grows by more than 8 in base 2, after the P V before has landed (the first
        // visible key: by infinity, at any scale; -inf - -inf, none so far, is not a number)
        const bool grow = (pm - m_run) * scale > 8.f;
        if (__any_sync(0xffffffffu, grow)) {
          const float cr = grow ? exp2f((m_run - pm) * scale) : 1.f;  // 0 when m_run was -inf
          if (i > 0) {
            if (!wait_w(o_done(x, n - 1), (n - 1) >> 1)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int c0 = 0; c0 < HD; c0 += 16) {
              float o[16];
              tmem_ld_16(t_o + (uint32_t)c0, o);
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] *= cr;
              tmem_st_16(t_o + (uint32_t)c0, o);
            }
          }
          if (grow) {
            l_run *= cr;
            m_run = pm;
            // s scale - m scale, rounded once, keeps what rounding m scale left, half a step. A score that it matters for, of 2^28, has
            // no neighbour in float32 that is not 16 away, so that a smaller scale leaves the same keys with the probability.
            scale = fminf(a.scale, 0x1p28f / fabsf(pm));
          }
        }
        const float mref = m_run == -INFINITY ? 0.f : m_run * scale;  // no visible key so far: any finite value
        const uint64_t scale2 = f2_pack(scale, scale), mref2 = f2_pack(-mref, -mref);
        uint64_t ps[2] = {0, 0};  // (two sums each)
#pragma unroll
        for (int c0 = 0; c0 < 64; c0 += 32) {
          uint32_t pk[16];
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            const float2 e = f2_unpack(f2_fma(f2_pack(__uint_as_float(su[c0 + k]), __uint_as_float(su[c0 + k + 1])), scale2, mref2));
            const float p0 = ex2_fast(e.x), p1 = ex2_fast(e.y);
            ps[k / 2 & 1] = f2_add(ps[k / 2 & 1], f2_pack(p0, p1));
            pk[k / 2] = pack_bf16(p0, p1);
          }
          tmem_put_16(t_sn + (uint32_t)(c0 / 2), pk);
        }
        const float2 sum = f2_unpack(f2_add(ps[0], ps[1]));
        l_run += sum.x + sum.y;
        tmem_st_wait_done();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(x, n));
      }
      // the last P V, then the row out: O / l, or its part
      const bool whole = s.kb0 == 0 && s.kb1 == s.nb;
      const long long token = s.token0 + x * QT + qi;
      const int head = (s.h << g_log) + g;
      const int slot = 2 * blockIdx.x + (s.kb0 == 0), prow = x * 128 + row;  // of the part
      bf16* orow = static_cast<bf16*>(a.out) + token * a.os + (long long)head * HD;
      const bool wide = reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && a.os % 8 == 0;
      if (ok && s.e[x] > 0) {
        if (!wait_w(o_done(x, n - 1), (n - 1) >> 1)) break;
        tc_fence_after();
        const float inv = whole ? (l_run != 0.f ? 1.f / l_run : 0.f) : 1.f;
#pragma unroll
        for (int c0 = 0; c0 < HD; c0 += 32) {
          float o[32];
          tmem_ld_32(t_o + (uint32_t)c0, o);
          if (!row_ok) continue;
          if (!whole) {
#pragma unroll
            for (int k = 0; k < 32; k += 4)
              *reinterpret_cast<float4*>(a.part_o + pair_part(slot, prow, c0 + k, HD)) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
          } else if (wide) {
#pragma unroll
            for (int k = 0; k < 32; k += 8)
              *reinterpret_cast<uint4*>(orow + c0 + k) =
                  make_uint4(pack_bf16(o[k] * inv, o[k + 1] * inv), pack_bf16(o[k + 2] * inv, o[k + 3] * inv),
                             pack_bf16(o[k + 4] * inv, o[k + 5] * inv), pack_bf16(o[k + 6] * inv, o[k + 7] * inv));
          } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) orow[c0 + k] = from_f32<bf16>(o[k] * inv);
          }
        }
        tc_fence_before();
      } else if (row_ok && !whole) {  // the tile has no block here: an empty part
        for (int k = 0; k < HD; ++k) a.part_o[pair_part(slot, prow, k, HD)] = 0.f;
      }
      if (row_ok) {
        if (!whole) a.part_ml[(size_t)slot * PAIR_ROWS + prow] = make_float2(m_run == -INFINITY ? -INFINITY : m_run * a.scale, l_run);
        else if (a.lse) a.lse[token * c.Hq + head] = l_run != 0.f ? (m_run * a.scale + log2f(l_run)) * LN2 : -INFINITY;
      }
      if (ok && s_left[(segs - 1) % PairSeg::RING] == segs - 1) {  // (written before the last P V that it concerns)
        __syncwarp();  // the rows are written
        float left[HD / 32] = {};
        int e = max(s.kb0 * 64, s.see0 + 1);
        for (int i = 0; i < 32; ++i) {
          const int see_r = __shfl_sync(0xffffffffu, see, i), head_r = __shfl_sync(0xffffffffu, head, i), prow_r = __shfl_sync(0xffffffffu, prow, i);
          const long long token_r = __shfl_sync(0xffffffffu, token, i);
          if (see_r < 0) continue;
          if constexpr (MODE == KEYS_ALL) {
            chunk_left_out<HD>(a, s.b, s.h, e, min(s.kb1 * 64, see_r + 1), left);
          } else {
#pragma unroll
            for (int k = 0; k < HD / 32; ++k) left[k] = 0.f;
            window_left_out<HD>(a, s.b, s.h, see_r, s.see0, s.see0 + s.nq[0] + s.nq[1] - 1, s.kb0, s.kb1, sinks, skip, left);
          }
          bf16* out = static_cast<bf16*>(a.out) + token_r * a.os + (long long)head_r * HD + lane * (HD / 32);
#pragma unroll
          for (int k = 0; k < HD / 32; ++k) {
            if (left[k] == 0.f) continue;
            if (whole) out[k] = from_f32<bf16>(to_f32(out[k]) + left[k]);
            else a.part_o[pair_part(slot, prow_r, lane * (HD / 32) + k, HD)] += left[k];
          }
        }
        __syncwarp();
      }
      blk += s.kb1 - s.kb0;
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(segs - 1));  // only now: s_left's word was this item's until here
    }
  }
  if (*abort_flag) drain_copies();
  tc_fence_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

// ----------------------------------------------------------------------------
// Weights
// ----------------------------------------------------------------------------
// base[b] = items (`entries` entries each) of the rows before b; returns how many there are. By the whole block.
__device__ __forceinline__ long long weigh_items(const ChunkDev& c, int entries, long long* base, long long* red) {
  long long carry = 0;
  for (int b0 = 0; b0 < c.n; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    const long long items = b < c.n ? (chunk_row(c, b).len + entries - 1) / entries : 0;
    long long total;
    const long long at = carry + block_scan(items, red, &total);
    if (b < c.n) base[b] = at;
    carry += total;
  }
  if (threadIdx.x == 0) base[c.n] = carry;
  __syncthreads();
  return carry;
}
__device__ __forceinline__ int item_row(const long long* base, int n, long long item) {  // largest b with base[b] <= item
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (base[mid] <= item) lo = mid;
    else hi = mid;
  }
  return lo;
}

// An item is a page of a row, with all heads and all queries that see one of its entries; one writer an entry, and a fixed
// order of the sums. Four threads a key, each with every fourth query row.
template <typename T, int HD>
__global__ void __launch_bounds__(256) k_chunk_weigh(ChunkAttn a, const float* w_in, float* w_out) {
  constexpr int KS = HD + 4, QR = HD == 128 ? 16 : 32;
  extern __shared__ long long s_base[];
  __shared__ long long s_red[33];
  __shared__ __align__(16) float sK[64 * KS];
  __shared__ __align__(16) float sQ[QR * HD];
  __shared__ float s_lse[QR];
  __shared__ int s_see[QR];
  __shared__ float s_sum[4][64];
  const ChunkDev& c = a.c;
  const int tid = threadIdx.x, key = tid & 63, part = tid >> 6, G = c.G;
  const long long items = weigh_items(c, 64, s_base, s_red);
  pdl_wait();
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int lo = item_row(s_base, c.n, item);
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

// The same from the scores that k_chunk_mma left: an item is 256 entries of a row; 64 threads x 4 entries, four groups of
// threads that take every fourth (query, head). Reads 4 bytes a (query, head, entry) instead of K again: 32 single tokens over
// up to 8192 entries, 16 heads x 64: 8 us.
__global__ void __launch_bounds__(256) k_chunk_weigh_scores(ChunkAttn a, const float* w_in, float* w_out) {
  extern __shared__ long long s_base[];
  __shared__ long long s_red[33];
  __shared__ float4 s_sum[4][64];
  const ChunkDev& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, part = tid >> 6;
  const long long items = weigh_items(c, 256, s_base, s_red);  // (of lengths alone: beside the kernels before)
  pdl_wait();
  const long long width = (long long)c.max_pages * 64;
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int b = item_row(s_base, c.n, item);
    const ChunkRow r = chunk_row(c, b);
    const int e = (int)(item - s_base[b]) * 256 + lane * 4, s0 = r.len - r.ql;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (e < r.len) {
      // query i sees entries up to s0 + i
      const int i0 = max(0, e - s0), n = (r.ql - i0) * c.Hq;
      for (int j = part; j < n; j += 4) {
        const long long at = (long long)(r.t0 + i0) * c.Hq + j;
        const float l = a.lse[at] * LOG2E;
        const float4 s = *reinterpret_cast<const float4*>(a.scores + at * width + e);
        const int see = s0 + i0 + j / c.Hq - e;
        sum.x += exp2f(s.x - l);
        if (see >= 1) sum.y += exp2f(s.y - l);
        if (see >= 2) sum.z += exp2f(s.z - l);
        if (see >= 3) sum.w += exp2f(s.w - l);
      }
    }
    __syncthreads();
    s_sum[part][lane] = sum;
    __syncthreads();
    if (part == 0 && e < r.len) {
      const int page = chunk_page(c.page_table, c.max_pages, c.n_pages, b, e / 64, c.err);
      if (page < 0) continue;
      const float4 x = s_sum[1][lane], y = s_sum[2][lane], z = s_sum[3][lane];
      const float add[4] = {(sum.x + x.x) + (y.x + z.x), (sum.y + x.y) + (y.y + z.y), (sum.z + x.z) + (y.z + z.z), (sum.w + x.w) + (y.w + z.w)};
      const long long at = (long long)page * 64 + e % 64;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (e + k < r.len) w_out[at + k] = (w_in ? w_in[at + k] : 0.f) + add[k];
    }
  }
  pdl_trigger();
}

// ----------------------------------------------------------------------------
// Weights on tcgen05 (bfloat16, head_dim 64 and 128, many rows)
// ----------------------------------------------------------------------------
// S^T = K Q^T with the keys as MMA rows: a thread owns one key (TMEM lane) and adds exp(s - lse) over the columns, which are
// query rows, so sums need no exchange between threads and no atomics. lse comes off inside the product: 16 more columns beside
// head_dim, ones in K and -lse / scale in q, in three bfloat16 that hold 24 bits (read from shared memory by every thread it
// took the port that the MMAs read their operands through). A CTA goes over its units of the flat order (row, block
// of 256 keys, head, tile of 128 query rows); K of a (block, head) stays in shared memory while the tiles of q stream through.
//   warps 0-15      two sets of eight take turns at the units; warps 0-3 and 4-7 of a set have keys 0-127 and 128-255 of the
//                   block: S from tensor memory, sums, and at the block's end the sum of both sets out;
//   warp 16         producer (tensor maps);
//   warps 17, 18    issue S^T of keys 0-127 and 128-255 into one of two TMEM buffers each;
//   warp 19         the tile's lse into the columns beside q.
// A block inside one CTA's share is written out; parts of a shared one meet in k_weigh_join, in the CTAs' order.
// Bound by the MMAs, 1150 cycles a unit of about 1600 with the softmax warps' latencies and the start: 4 x 1000 tokens over up
// to 5000 entries, 16 / 8 heads x 128: 45 us behind 83 us of attention (65 with lse from shared memory and eight softmax warps).
constexpr int WEIGH_THREADS = 640;
struct WeighTc {
  WeighSplit sp;
  const float* w_in;
  float* w_out;
  float* part;  // [2 ctas][256]
};
template <int HD>
struct WeighShape {
  static constexpr int ATOMS = HD / 64, COL = 128 * 128, T_BYTES = ATOMS * COL;
  static constexpr int NQ = HD == 128 ? 2 : 6, NL = 4;  // tiles of q and of lse on the way
  static constexpr int X_BYTES = 128 * 32;              // 128 rows of the 16 columns beside head_dim
  static constexpr int OFF_Q = 4 * T_BYTES;  // K: two buffers of two tiles
  static constexpr int OFF_X = OFF_Q + NQ * T_BYTES, OFF_SUM = OFF_X + (1 + NL) * X_BYTES, OFF_BAR = OFF_SUM + 2 * 256 * 4;
  static constexpr int NBAR = 4 + 2 * NQ + 4 + 2 * NL, OFF_INT = OFF_BAR + NBAR * 8, OFF_BASE = OFF_INT + 16;
  static int bytes(int n) { return std::max(OFF_BASE + (n + 1) * 8 + 1024, tmem_min_smem(512)); }
};
// Descriptor of a K-major tile of 16 columns: rows of 32 bytes, swizzled in atoms of 8 rows (the halves of rows 4-7 change places).
__device__ __forceinline__ uint64_t smem_desc_sw32(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)1u << 16 | (uint64_t)(256u >> 4) << 32 | (uint64_t)1u << 46 | (uint64_t)6u << 61;
}

__device__ __forceinline__ long long weigh_plan(const ChunkDev& c, const WeighSplit& sp, long long* base, long long* red) {
  long long carry = 0;
  for (int b0 = 0; b0 < c.n; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    long long u = 0;
    if (b < c.n) {
      const ChunkRow r = chunk_row(c, b);
      u = sp.before(r.len - r.ql, r.ql, sp.blocks(r.len - r.ql, r.ql)) * c.Hkv;
    }
    long long total;
    const long long at = carry + block_scan(u, red, &total);
    if (b < c.n) base[b] = at;
    carry += total;
  }
  if (threadIdx.x == 0) base[c.n] = carry;
  __syncthreads();
  return carry;
}
struct WeighBlock {
  int b, kb, t0, s0, ql, len, first, vis;  // row, block; the row's tokens and entries; the block's first tile, tiles
  long long begin;                         // its first unit in the flat order; it has vis * Hkv
};
__device__ __forceinline__ WeighBlock weigh_block(const ChunkDev& c, const WeighSplit& sp, const long long* base, long long pos) {
  WeighBlock w;
  w.b = item_row(base, c.n, pos);
  const ChunkRow r = chunk_row(c, w.b);
  w.t0 = r.t0;
  w.ql = r.ql;
  w.len = r.len;
  w.s0 = r.len - r.ql;
  w.kb = sp.block_of(w.s0, w.ql, c.Hkv, pos - base[w.b]);
  w.first = sp.first(w.s0, w.kb);
  w.vis = sp.tiles(w.ql) - w.first;
  w.begin = base[w.b] + sp.before(w.s0, w.ql, w.kb) * c.Hkv;
  return w;
}

template <int HD>
__global__ void __launch_bounds__(WEIGH_THREADS, 1) k_weigh_tc(ChunkAttn a, WeighTc wt, int g_log, const __grid_constant__ CUtensorMap q_map,
                                                               const __grid_constant__ CUtensorMap pool_map) {
  using Sh = WeighShape<HD>;
  constexpr int NQ = Sh::NQ, NL = Sh::NL;
  extern __shared__ uint8_t smem_raw[];
  __shared__ long long s_red[33];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + Sh::OFF_BAR);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + Sh::OFF_INT);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + Sh::OFF_INT) + 1;
  long long* s_base = reinterpret_cast<long long*>(sm + Sh::OFF_BASE);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  auto k_full = [&](unsigned i) { return bar(i & 1); };
  auto k_empty = [&](unsigned i) { return bar(2 + (i & 1)); };
  auto q_full = [&](unsigned i) { return bar(4 + i % NQ); };
  auto q_empty = [&](unsigned i) { return bar(4 + NQ + i % NQ); };
  auto s_full = [&](unsigned i) { return bar(4 + 2 * NQ + (i & 1)); };
  auto s_read = [&](unsigned i) { return bar(4 + 2 * NQ + 2 + (i & 1)); };
  auto l_full = [&](unsigned i) { return bar(4 + 2 * NQ + 4 + i % NL); };
  auto l_empty = [&](unsigned i) { return bar(4 + 2 * NQ + 4 + NL + i % NL); };
  const ChunkDev& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (unsigned i = 0; i < NQ; ++i) {
      mbar_init(q_full(i), 1);
      mbar_init(q_empty(i), 2);
    }
    for (unsigned i = 0; i < 2; ++i) {
      mbar_init(k_full(i), 1);
      mbar_init(k_empty(i), 2);
      mbar_init(s_full(i), 2);
      mbar_init(s_read(i), 8);
    }
    for (unsigned i = 0; i < NL; ++i) {
      mbar_init(l_full(i), 1);
      mbar_init(l_empty(i), 2);
    }
    *abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&q_map);
    prefetch_tensormap(&pool_map);
  }
  if (warp == 17) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  for (int i = tid; i < (1 + NL) * 256; i += WEIGH_THREADS) {  // the keys' ones, and zeros
    const int r = i >> 1 & 127, half = i & 1;
    *reinterpret_cast<uint4*>(sm + Sh::OFF_X + (i >> 8) * Sh::X_BYTES + r * 32 + (half ^ (r >> 2 & 1)) * 16) =
        i < 256 && half == 0 ? make_uint4(0x3f803f80u, 0x3f80u, 0u, 0u) : make_uint4(0u, 0u, 0u, 0u);
  }
  fence_proxy_async_smem();
  // The plan, K and q are read without waiting for the kernels before, which write none of it; only the lse are theirs, so only
  // warp 19 waits, and what this grid writes comes after an lse.
  const long long all = weigh_plan(c, wt.sp, s_base, s_red), per = chunk_share(a, all);
  long long pos = blockIdx.x * per;
  const long long end = pos + per < all ? pos + per : all;
  __shared__ WeighBlock s_first;
  if (tid == 0 && pos < end) s_first = weigh_block(c, wt.sp, s_base, pos);
  tc_fence_before();
  __syncthreads();  // barriers initialised, tensor memory allocated
  tc_fence_after();
  pdl_trigger();
  const uint32_t tmem = *tmem_slot;
  WeighBlock w = s_first;
  const int QT = 1 << wt.sp.qt_log;
  auto wait = [&](uint32_t b, uint32_t parity) {
    if (mbar_try_wait(b, parity & 1u)) return true;
    if (*abort_flag) return false;
    if (mbar_wait(b, parity & 1u, a.werr)) return true;
    *abort_flag = 1;
    return false;
  };
  // f(block, head, tile, unit's number in this CTA, first unit of its K here, last one) for this CTA's units; false ends it
  auto each = [&](auto&& f, auto&& block_end) {
    for (unsigned n = 0; pos < end;) {
      if (n > 0) w = weigh_block(c, wt.sp, s_base, pos);
      const long long stop = w.begin + (long long)w.vis * c.Hkv < end ? w.begin + (long long)w.vis * c.Hkv : end, start = pos;
      int h = (int)((pos - w.begin) / w.vis), t = (int)((pos - w.begin) % w.vis);
      for (bool k_new = true; pos < stop; ++pos, ++n) {
        const bool k_last = t + 1 == w.vis || pos + 1 == stop;
        if (!f(w, h, w.first + t, n, k_new, k_last)) return;
        k_new = k_last;
        if (++t == w.vis) t = 0, ++h;
      }
      if (!block_end(w, start, stop)) return;
    }
  };
  auto no_end = [](const WeighBlock&, long long, long long) { return true; };

  if (warp == 16) {
    unsigned kl = 0;
    each([&](const WeighBlock& w, int h, int t, unsigned n, bool k_new, bool) {
      bool ok = true;
      if (k_new) {
        const int p = min(w.kb * 4 + (lane & 3), (w.len - 1) / 64);
        int mine = chunk_page(c.page_table, c.max_pages, c.n_pages, w.b, p, lane < 4 ? c.err : nullptr);
        mine = max(mine, 0);  // reported; what it adds goes nowhere
        int pg[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) pg[i] = __shfl_sync(0xffffffffu, mine, i);
        if (lane == 0 && (kl < 2 || (ok = wait(k_empty(kl), kl / 2 - 1)))) {
          mbar_arrive_expect_tx(k_full(kl), 2 * Sh::T_BYTES);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < Sh::ATOMS; ++k)
              tma_load_3d(smem_u32(sm + ((kl & 1) * 2 + i / 2) * Sh::T_BYTES + k * Sh::COL + (i & 1) * (Sh::COL / 2)), &pool_map, k * 64,
                          (c.layer * 2 * c.Hkv + h) * 64, pg[i], k_full(kl));
        }
        ++kl;
      }
      if (lane == 0 && ok && (n < NQ || (ok = wait(q_empty(n), n / NQ - 1)))) {
        mbar_arrive_expect_tx(q_full(n), Sh::T_BYTES);
#pragma unroll
        for (int k = 0; k < Sh::ATOMS; ++k)
          tma_load_3d(smem_u32(sm + Sh::OFF_Q + (n % NQ) * Sh::T_BYTES + k * Sh::COL), &q_map, k * 64, h << g_log, w.t0 + t * QT, q_full(n));
      }
      return (bool)__all_sync(0xffffffffu, ok);
    }, no_end);
  } else if (warp == 17 || warp == 18) {
    if (elect_one()) {
      const int x = warp - 17;
      constexpr uint32_t IDS = idesc_bf16_f32(128, 128);
      constexpr uint64_t T_E = Sh::T_BYTES >> 4, COL_E = Sh::COL >> 4;
      const uint64_t dk = smem_desc_sw128(smem_u32(sm)), dq = smem_desc_sw128(smem_u32(sm + Sh::OFF_Q));
      const uint64_t d_one = smem_desc_sw32(smem_u32(sm + Sh::OFF_X)), d_lse = smem_desc_sw32(smem_u32(sm + Sh::OFF_X + Sh::X_BYTES));
      unsigned kl = 0;
      each([&](const WeighBlock&, int, int, unsigned n, bool k_new, bool k_last) {
        if (k_new && !wait(k_full(kl), kl / 2)) return false;
        if (!wait(q_full(n), n / NQ) || (n >= 2 && !wait(s_read(n), n / 2 - 1))) return false;
        tc_fence_after();
#pragma unroll
        for (int kc = 0; kc < Sh::ATOMS; ++kc)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            tc_mma_f16(tmem + (n & 1) * 256 + 128u * x, dk + ((kl & 1) * 2 + x) * T_E + kc * COL_E + 2 * k,
                       dq + (n % NQ) * T_E + kc * COL_E + 2 * k, IDS, (kc | k) ? 1u : 0u);
        tc_commit(q_empty(n));
        if (k_last) {
          tc_commit(k_empty(kl));
          ++kl;
        }
        if (!wait(l_full(n), n / NL)) return false;
        tc_fence_after();
        tc_mma_f16(tmem + (n & 1) * 256 + 128u * x, d_one, d_lse + (n % NL) * (uint64_t)(Sh::X_BYTES >> 4), IDS, 1u);
        tc_commit(l_empty(n));
        tc_commit(s_full(n));
        return true;
      }, no_end);
    }
    __syncwarp();
  } else if (warp == 19) {
    pdl_wait();
    const float by = -LOG2E / a.scale;
    float ahead[4];  // the next unit's, on their way
    auto put = [&](unsigned n, const float (&v)[4]) {
      if (n >= NL && !__all_sync(0xffffffffu, wait(l_empty(n), n / NL - 1))) return false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = v[i] * by, hi = __bfloat162float(__float2bfloat16(x)), r1 = x - hi, mid = __bfloat162float(__float2bfloat16(r1));
        const bool fin = fabsf(hi) < INFINITY;  // else hi alone
        const int j = lane + 32 * i;
        *reinterpret_cast<uint4*>(sm + Sh::OFF_X + (1 + n % NL) * Sh::X_BYTES + j * 32 + (j >> 2 & 1) * 16) =
            make_uint4(pack_bf16(hi, fin ? mid : 0.f), pack_bf16(fin ? r1 - mid : 0.f, 0.f), 0u, 0u);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(l_full(n));
      return true;
    };
    unsigned got = 0;
    each([&](const WeighBlock& w, int h, int t, unsigned n, bool, bool) {
      const int cols = min(QT, w.ql - t * QT) << g_log;
      float l[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = lane + 32 * i;
        l[i] = j < cols ? a.lse[(long long)(w.t0 + t * QT + (j >> g_log)) * c.Hq + (h << g_log) + (j & ((1 << g_log) - 1))] : 0.f;
      }
      if (n > 0 && !put(n - 1, ahead)) return false;
#pragma unroll
      for (int i = 0; i < 4; ++i) ahead[i] = l[i];
      got = n + 1;
      return true;
    }, no_end);
    if (got > 0 && pos >= end) put(got - 1, ahead);
  } else {
    const int set = warp >> 3, x = warp >> 2 & 1, row = (warp & 3) * 32 + lane;
    const uint32_t t_s = tmem + ((uint32_t)((warp & 3) * 32) << 16) + 128u * (uint32_t)x;
    const float scale = a.scale;
    float sum = 0.f;
    unsigned ends = 0;
    // a failed wait does not end the loop: all sixteen warps meet at the blocks' ends
    each([&](const WeighBlock& w, int, int t, unsigned n, bool, bool) {
      if ((n & 1) != set || !__all_sync(0xffffffffu, wait(s_full(n), n / 2))) return true;
      tc_fence_after();
      const int key = w.kb * 256 + x * 128 + row, cols = min(QT, w.ql - t * QT) << g_log;
      // query i of the row sees the key when s0 + i >= key: columns from lo on
      const int lo = min(max(key - w.s0 - t * QT, 0), cols >> g_log) << g_log;
      const uint64_t scale2 = f2_pack(scale, scale);
      uint64_t p4[2] = {0, 0};  // (two sums each)
#pragma unroll 1
      for (int c0 = 0; c0 < cols; c0 += 32) {
        uint32_t su[32];
        tmem_ld_32_issue(t_s + (n & 1) * 256 + (uint32_t)c0, su);
        tmem_ld_wait();
        if (c0 + 32 >= cols) {  // S is in registers: the buffer is free
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(s_read(n));
        }
        if (cols >= c0 + 32 && __all_sync(0xffffffffu, lo <= c0)) {
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float2 e = f2_unpack(f2_fma(f2_pack(__uint_as_float(su[j]), __uint_as_float(su[j + 1])), scale2, 0));
            p4[j / 2 & 1] = f2_add(p4[j / 2 & 1], f2_pack(ex2_fast(e.x), ex2_fast(e.y)));
          }
        } else if (!__all_sync(0xffffffffu, lo >= c0 + 32)) {
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float p = ex2_fast(__uint_as_float(su[j]) * scale), r = ex2_fast(__uint_as_float(su[j + 1]) * scale);
            p4[j / 2 & 1] = f2_add(p4[j / 2 & 1], f2_pack((unsigned)(c0 + j - lo) < (unsigned)(cols - lo) ? p : 0.f,
                                                          (unsigned)(c0 + j + 1 - lo) < (unsigned)(cols - lo) ? r : 0.f));
          }
        }
      }
      const float2 added = f2_unpack(f2_add(p4[0], p4[1]));
      sum += added.x + added.y;
      return true;
    }, [&](const WeighBlock& w, long long start, long long stop) {
      // the other set's sums, through one of two buffers in turn: one is written again only after the barrier in between
      float* other = reinterpret_cast<float*>(sm + Sh::OFF_SUM) + (ends++ & 1) * 256 + x * 128 + row;
      if (set == 1) *other = sum;
      bar_named(1, 512);
      if (set == 0) {
        sum += *other;
        const int key = w.kb * 256 + x * 128 + row;
        if (start != w.begin || stop != w.begin + (long long)w.vis * c.Hkv) {
          wt.part[(2 * blockIdx.x + (start == w.begin)) * 256 + x * 128 + row] = sum;
        } else if (key < w.len) {
          const int page = chunk_page(c.page_table, c.max_pages, c.n_pages, w.b, key / 64, nullptr);
          const long long at = (long long)page * 64 + key % 64;
          if (page >= 0) wt.w_out[at] = (wt.w_in ? wt.w_in[at] : 0.f) + sum;
        }
      }
      sum = 0.f;
      return true;
    });
  }
  if (*abort_flag) drain_copies();
  tc_fence_before();
  __syncthreads();
  if (warp == 17) tmem_dealloc(tmem, 512);
}

// Blocks that k_weigh_tc's CTAs share: the first CTA whose share starts inside one adds its parts (grid x < ctas - 1). The
// other CTAs of the grid copy the weights of rows without new tokens.
__global__ void __launch_bounds__(256) k_weigh_join(ChunkAttn a, WeighTc wt, int per_row) {
  extern __shared__ long long s_base[];
  __shared__ long long s_red[33];
  const ChunkDev& c = a.c;
  if ((int)blockIdx.x >= a.ctas - 1) {
    const int i = blockIdx.x - (a.ctas - 1), b = i / per_row;
    pdl_wait();
    const ChunkRow r = chunk_row(c, b);
    if (r.ql > 0) return;
    for (int e = (i % per_row) * 256 + threadIdx.x; e < r.len; e += per_row * 256) {
      const int page = chunk_page(c.page_table, c.max_pages, c.n_pages, b, e / 64, c.err);
      const long long at = (long long)page * 64 + e % 64;
      if (page >= 0) wt.w_out[at] = wt.w_in ? wt.w_in[at] : 0.f;
    }
    return;
  }
  const long long all = weigh_plan(c, wt.sp, s_base, s_red), per = chunk_share(a, all), pos = (blockIdx.x + 1) * per;
  __shared__ WeighBlock s_w;
  if (threadIdx.x == 0) {
    s_w.begin = pos;
    if (pos < all) s_w = weigh_block(c, wt.sp, s_base, pos);
  }
  __syncthreads();
  const WeighBlock w = s_w;
  pdl_wait();  // (as in k_chunk_join)
  if (pos >= all || w.begin == pos || w.begin / per != blockIdx.x) return;
  const int c0 = blockIdx.x, c1 = (int)((w.begin + (long long)w.vis * c.Hkv - 1) / per), key = w.kb * 256 + threadIdx.x;
  float sum = wt.part[(2 * c0 + 1) * 256 + threadIdx.x];
  for (int i = c0 + 1; i <= c1; ++i) sum += wt.part[2 * i * 256 + threadIdx.x];
  if (key >= w.len) return;
  const int page = chunk_page(c.page_table, c.max_pages, c.n_pages, w.b, key / 64, c.err);
  const long long at = (long long)page * 64 + key % 64;
  if (page >= 0) wt.w_out[at] = (wt.w_in ? wt.w_in[at] : 0.f) + sum;
}

// ----------------------------------------------------------------------------
// Launches
// ----------------------------------------------------------------------------
// Which kernel and split a call takes; a function of the arguments and the device alone.
//
// What an item counts beside its blocks (microseconds at 0 / 4 blocks of k_chunk_pair: 8192 causal tokens, 16 / 8 heads x 128,
// 225 / 194, 4 x 1000 over 4000 entries 87 / 81; at 0 / 10 pages of k_chunk_mma with head_dim 64: 32 single tokens over up to
// 8192 entries 119 / 105, 32 rows of up to 16 tokens 128 / 107; at 2 / 6 pages with head_dim 128: 100 single tokens over up to
// 500 entries 45 / 40). Without, CTAs with many short items finished up to a third later than the others.
constexpr int PAD_PAIR = 4, PAD_MMA128 = 6, PAD_MMA = 10, PAD_SIMT = 2, PAD_Q4 = 6;
struct ChunkPath {
  bool pair;    // k_chunk_pair
  int rt;       // rows of an item
  int ctas;
  int pad;      // blocks that an item counts beside its own
  bool weigh_tc;  // the weights from k_weigh_tc
  long long scores;  // bytes of the scores that k_chunk_mma leaves for the weights
  size_t part_ml, join, lse, werr, weigh, scores_at, total;  // scratch offsets (part_o at 0)
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
    p.pad = PAD_SIMT;
  } else {
    // tcgen05: tiles of 128 rows of whole groups of heads, q through a tensor map
    const bool tc = c.hd >= 64 && (c.G & (c.G - 1)) == 0 && reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_stride % 8 == 0;
    // k_weigh_tc divides lse by the scale; out of this range the weights come from the scores, or from the CUDA cores
    const float scale = a.scale > 0.f ? a.scale : 1.f;
    const bool weigh_fits = !a.weight_out || (scale >= 0x1p-64f && scale <= 0x1p64f);
    // k_chunk_pair also where its tiles are mostly padding: k_chunk_mma's products cost it more from 17 rows on at head_dim 128
    // (32 rows of 16 / 32 tokens over up to 8192 entries, 16 / 8 heads: 109 / 112 us against 115 / 179; 8 tokens, 16 rows: 108
    // against 101), from 33 on at 64 (32 rows of 48 / 64 tokens, 16 heads: 179 / 177 against 183 / 187, 4 rows of 64 over up to
    // 1000: 16 against 24; 32 rows of 17 / 32 tokens: 178 / 177 against 132 / 134)
    p.pair = tc && weigh_fits && rows > (c.hd == 128 ? 16 : 32);
    // weights: the scores that k_chunk_mma has at hand, 4 bytes a (query, head, entry) written and read instead of K again, up to
    // 16 rows (32 rows of 8 tokens over up to 8192 entries, 16 / 8 heads x 128: 142 us so, 155 with k_weigh_tc; of 16 tokens with
    // 16 heads x 64 170 both ways, and twice the bytes at 32) and up to a bound on the scratch, which the host can only size by
    // the longest row. With few entries the sums over the queries of a block of 256 entries are a chain that nothing hides: there
    // k_weigh_tc from 9 rows on (4 rows of 16 tokens over up to 1000 entries, 16 heads x 64: 40 us from the scores, 23 so; one of
    // 8 over 8000, 16 / 8 heads x 128: 33 / 27). S^T on the CUDA cores where the tiles do not fit.
    // (the largest arguments pass 2^63 here and below)
    const bool fit = (double)c.T * c.Hq * c.max_pages * 256 <= (256 << 20), few = (long long)c.n * ((c.max_pages + 3) / 4) < num_sms;
    p.weigh_tc = a.weight_out && tc && weigh_fits && (rows > 16 || !fit || (few && rows > 8));
    p.scores = a.weight_out && !p.weigh_tc && fit ? (long long)c.T * c.Hq * c.max_pages * 256 : 0;
    p.rt = p.pair ? PAIR_ROWS : rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
    p.ctas = (c.hd == 128 || p.pair ? 1 : 2) * num_sms;
    p.pad = p.pair ? PAD_PAIR : c.hd == 128 ? PAD_MMA128 : PAD_MMA;
  }
  // no more CTAs than there can be blocks
  const int qt_log = pow2_log(std::max(1, p.rt / c.G));
  p.ctas = (int)std::min<double>(p.ctas, std::max(1.0, ((double)(c.T >> qt_log) + c.n) * c.Hkv * ((double)c.max_pages + p.pad)));
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = (o + bytes + 255) / 256 * 256; return at; };
  take((size_t)2 * p.ctas * p.rt * c.hd * 4);
  p.part_ml = take((size_t)2 * p.ctas * p.rt * 8);
  p.join = take((size_t)p.ctas * 16);
  p.lse = take(a.weight_out && !a.lse ? (size_t)c.T * c.Hq * 4 : 0);
  p.werr = take(4);
  p.weigh = take(p.weigh_tc ? (size_t)2 * num_sms * 256 * 4 : 0);
  p.scores_at = take((size_t)p.scores);
  p.total = o;
  return p;
}
size_t chunk_attn_scratch(const ChunkDev& c, int dtype, const tlf_attn_chunk_args& a, int num_sms) {
  return chunk_path(c, dtype, a, num_sms).total;
}

template <typename T, int RT, int HD, int MODE>
static cudaError_t simt_launch(const ChunkAttn& a, cudaStream_t st) {
  const int smem = SimtShape<RT, HD>::bytes(a.c.n);
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_simt<T, RT, HD, MODE>), SimtShape<RT, HD>::bytes(SV_MAX_ROWS)))
    return e;
  return launch_k(k_chunk_simt<T, RT, HD, MODE>, dim3(a.ctas), dim3(256), smem, st, a);
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
bool chunk_q_map(CUtensorMap* m, const ChunkAttn& a) {
  const auto fn = tensor_map_encoder();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)a.c.hd, (cuuint64_t)a.c.Hq, (cuuint64_t)a.c.T};
  cuuint64_t strides[2] = {(cuuint64_t)a.c.hd * 2, (cuuint64_t)a.qs * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)a.c.G, (cuuint32_t)(128 / a.c.G)}, es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.q), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <int HD, int MODE>
static cudaError_t pair_launch(const ChunkAttn& a, cudaStream_t st) {
  CUtensorMap qm, pm;
  if (!chunk_q_map(&qm, a) || !pool_map(&pm, a.c)) return cudaErrorInvalidValue;
  using Sh = PairShape<HD>;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_pair<HD, MODE>), Sh::bytes(SV_MAX_ROWS))) return e;
  return launch_k(k_chunk_pair<HD, MODE>, dim3(a.ctas), dim3(PAIR_THREADS), Sh::bytes(a.c.n), st, a, pow2_log(a.c.G), qm, pm);
}
template <int HD>
static cudaError_t weigh_launch(ChunkAttn a, const tlf_attn_chunk_args& args, float* part, int num_sms, cudaStream_t st) {
  a.ctas = num_sms;
  CUtensorMap qm, pm;
  if (!chunk_q_map(&qm, a) || !pool_map(&pm, a.c)) return cudaErrorInvalidValue;
  using Sh = WeighShape<HD>;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_weigh_tc<HD>), Sh::bytes(SV_MAX_ROWS))) return e;
  const WeighTc w{WeighSplit{7 - pow2_log(a.c.G), 8}, args.weight_in, args.weight_out, part};
  if (cudaError_t e = launch_k(k_weigh_tc<HD>, dim3(a.ctas), dim3(WEIGH_THREADS), Sh::bytes(a.c.n), st, a, w, pow2_log(a.c.G), qm, pm))
    return e;
  const int per_row = std::max(1, std::min(8, 1024 / a.c.n));
  return launch_k(k_weigh_join, dim3(a.ctas - 1 + per_row * a.c.n), dim3(256), (a.c.n + 1) * 8, st, a, w, per_row);
}
template <int HD, int MT, int MODE>
static cudaError_t mma_launch(const ChunkAttn& a, cudaStream_t st) {
  CUtensorMap map;
  if (!pool_map(&map, a.c)) return cudaErrorInvalidValue;
  using Sh = MmaShape<HD, MT>;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_mma<HD, MT, MODE>), Sh::bytes(SV_MAX_ROWS))) return e;
  return launch_k(k_chunk_mma<HD, MT, MODE>, dim3(a.ctas), dim3(Sh::THREADS), Sh::bytes(a.c.n), st, a, map);
}
template <int HD, int MODE>
static cudaError_t mma_rows(const ChunkAttn& a, cudaStream_t st) {
  if constexpr (HD >= 64)
    if (a.rows == 256) return pair_launch<HD, MODE>(a, st);
  return a.rows == 16 ? mma_launch<HD, 1, MODE>(a, st) : a.rows == 32 ? mma_launch<HD, 2, MODE>(a, st) : mma_launch<HD, 4, MODE>(a, st);
}
template <int MODE>
static cudaError_t bf16_launch(const ChunkAttn& a, cudaStream_t st) {
  return a.c.hd == 32 ? mma_rows<32, MODE>(a, st) : a.c.hd == 64 ? mma_rows<64, MODE>(a, st) : mma_rows<128, MODE>(a, st);
}
template <typename T, int MODE>
static cudaError_t simt_rows(const ChunkAttn& a, cudaStream_t st) {
  if constexpr (std::is_same<T, float>::value)
    if (a.c.hd == 16) return a.rows == 16 ? simt_launch<T, 16, 16, MODE>(a, st) : simt_launch<T, 64, 16, MODE>(a, st);
  switch (a.c.hd) {
    case 32: return a.rows == 16 ? simt_launch<T, 16, 32, MODE>(a, st) : simt_launch<T, 64, 32, MODE>(a, st);
    case 64: return a.rows == 16 ? simt_launch<T, 16, 64, MODE>(a, st) : simt_launch<T, 64, 64, MODE>(a, st);
    case 128: return a.rows == 16 ? simt_launch<T, 16, 128, MODE>(a, st) : simt_launch<T, 64, 128, MODE>(a, st);
  }
  return cudaErrorInvalidValue;
}
template <typename T>
static cudaError_t join_launch(const ChunkAttn& a, cudaStream_t st) {  // of T
  const dim3 jg(a.ctas - 1, std::max(1, a.rows / 32));
  if (a.ctas <= 1) return cudaSuccess;
  return a.rows == PAIR_ROWS ? (a.c.hd == 128 ? launch_k(k_pair_join<128>, jg, dim3(256), 0, st, a) : launch_k(k_pair_join<64>, jg, dim3(256), 0, st, a))
         : a.c.hd == 128 ? launch_k(k_chunk_join<T, 4>, jg, dim3(256), 0, st, a)
         : a.c.hd == 64 ? launch_k(k_chunk_join<T, 2>, jg, dim3(256), 0, st, a)
                         : launch_k(k_chunk_join<T, 1>, jg, dim3(256), 0, st, a);
}
template <typename T>
static cudaError_t chunk_launch(const ChunkAttn& a, const tlf_attn_chunk_args& args, float* weigh, int num_sms, cudaStream_t st) {
  cudaError_t e;
  if (std::is_same<T, bf16>::value)
    e = bf16_launch<KEYS_ALL>(a, st);
  else
    e = simt_rows<T, KEYS_ALL>(a, st);
  if (e) return e;
  const int base = (a.c.n + 1) * 8;
  if ((e = join_launch<T>(a, st))) return e;
  if (!args.weight_out) return cudaSuccess;
  const dim3 grid(4 * num_sms);
  if constexpr (std::is_same<T, bf16>::value)
    if (weigh) return a.c.hd == 64 ? weigh_launch<64>(a, args, weigh, num_sms, st) : weigh_launch<128>(a, args, weigh, num_sms, st);
  if (a.scores) return launch_k(k_chunk_weigh_scores, dim3(8 * num_sms), dim3(256), base, st, a, args.weight_in, args.weight_out);
  switch (a.c.hd) {
    case 16:
      if constexpr (std::is_same<T, float>::value)
        return launch_k(k_chunk_weigh<T, 16>, grid, dim3(256), base, st, a, args.weight_in, args.weight_out);
      break;
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
  a.sp = ChunkSplit{pow2_log(std::max(1, p.rt / c.G)), 6, p.pad};
  a.q = args.q;
  a.qs = args.q_stride ? args.q_stride : (long long)c.Hq * c.hd;
  a.out = args.out;
  a.os = args.out_stride ? args.out_stride : (long long)c.Hq * c.hd;
  a.lse = args.lse ? args.lse : args.weight_out ? reinterpret_cast<float*>(s + p.lse) : nullptr;
  a.scale = (args.scale != 0.f ? args.scale : 1.f / sqrtf((float)c.hd)) * LOG2E;
  a.ctas = p.ctas;
  a.rows = p.rt;
  a.scores = p.scores ? reinterpret_cast<float*>(s + p.scores_at) : nullptr;
  a.werr = c.err ? c.err : reinterpret_cast<uint32_t*>(s + p.werr);
  a.part_o = reinterpret_cast<float*>(s);
  a.part_ml = reinterpret_cast<float2*>(s + p.part_ml);
  a.join = reinterpret_cast<int4*>(s + p.join);
  a.window = 0x7fffffff;
  float* weigh = p.weigh_tc ? reinterpret_cast<float*>(s + p.weigh) : nullptr;
  return dtype == TLF_DTYPE_BF16 ? chunk_launch<bf16>(a, args, weigh, num_sms, st) : chunk_launch<float>(a, args, weigh, num_sms, st);
}

static tlf_attn_chunk_args plain_args(const tlf_attn_window_args& a) {
  return tlf_attn_chunk_args{a.q, a.q_stride, a.out, a.out_stride, a.lse, nullptr, nullptr, a.scale, 0};
}

// tlf_attn_window. A window of 0 over a cache in the dtype is tlf_attn_chunk's case, and its kernels'.
struct WindowPath {
  int rt, ctas, pad;  // as in ChunkPath
  bool four;          // k_chunk4.cu's kernels
  size_t part_ml, join, werr, total;
};
static WindowPath window_path(const ChunkDev& c, int dtype, const tlf_attn_window_args& a, int num_sms) {
  WindowPath p{};
  const long long rows = (long long)c.max_chunk * c.G;
  if (dtype == TLF_DTYPE_BF16 && a.kv_format == TLF_KV_PLAIN) {  // as without a window
    const ChunkPath whole = chunk_path(c, dtype, plain_args(a), num_sms);
    p.rt = whole.rt;
    p.ctas = whole.ctas;
    p.pad = whole.pad;
  } else if (dtype == TLF_DTYPE_BF16 && c.hd >= 64 && (c.G & (c.G - 1)) == 0 && (rows > (c.hd == 128 ? 16 : 48) || (c.G > 16 && rows > 0)) &&
             reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_stride % 8 == 0) {
    // tcgen05 where tiles of 16 rows, each with the cache again, take longer. 32 rows over up to 8192 entries, 16 / 8 heads x 128, of
    // 8 / 12 / 16 / 32 tokens: 146 / 147 / 145 / 146 us, in tiles of 16 rows 85 / 145 / 148 / 282; 16 heads x 64, of 16 / 32 / 48 / 64
    // tokens: 207 / 208 / 208 / 210, in tiles 78 / 140 / 204 / 267; under a window of 1024, 4 rows of 40 / 64 tokens: 22.1 / 22.5 and
    // 21.3 / 23.8. The tiles of 128 rows hold whole groups of a power of two heads alone: other groups of up to 16 are in tiles of 16
    // rows at any length (4 x 2048 tokens over up to 10240 entries, 24 / 8 and 28 / 4 heads x 128: 5.8 ms, 16 / 8 heads 0.45), larger
    // ones on the CUDA cores (64 single tokens over up to 4096 entries, 24 / 1 heads x 128: 395 us, 32 / 1 heads 39).
    p.four = true;
    p.rt = PAIR_ROWS;
    p.ctas = num_sms;
    p.pad = PAD_PAIR;
  } else if (dtype == TLF_DTYPE_BF16 && c.G <= 16) {
    p.four = true;
    p.rt = rows <= 8 ? 8 : 16;
    p.ctas = chunk4_per_sm(c.hd, p.rt) * num_sms;
    p.pad = PAD_Q4;
  } else {
    p.rt = rows <= 16 ? 16 : 64;
    p.ctas = 2 * num_sms;
    p.pad = PAD_SIMT;
  }
  const int qt_log = pow2_log(std::max(1, p.rt / c.G));
  p.ctas = (int)std::min<double>(p.ctas, std::max(1.0, ((double)(c.T >> qt_log) + c.n) * c.Hkv * ((double)c.max_pages + p.pad)));
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = (o + bytes + 255) / 256 * 256; return at; };
  take((size_t)2 * p.ctas * p.rt * c.hd * 4);
  p.part_ml = take((size_t)2 * p.ctas * p.rt * 8);
  p.join = take((size_t)p.ctas * 16);
  p.werr = take(4);
  p.total = o;
  return p;
}
size_t window_attn_scratch(const ChunkDev& c, int dtype, const tlf_attn_window_args& a, int num_sms) {
  if (a.window == 0 && a.kv_format == TLF_KV_PLAIN) return chunk_attn_scratch(c, dtype, plain_args(a), num_sms);
  return window_path(c, dtype, a, num_sms).total;
}
template <typename T>
static cudaError_t window_launch(const ChunkAttn& a, int kv_format, bool four, cudaStream_t st) {
  cudaError_t e;
  if (std::is_same<T, bf16>::value && kv_format == TLF_KV_4BIT && four) e = launch_chunk4(a, st);
  else if (kv_format == TLF_KV_4BIT) e = simt_rows<T, KEYS_4BIT>(a, st);
  else if constexpr (std::is_same<T, bf16>::value) e = bf16_launch<KEYS_WINDOW>(a, st);
  else e = simt_rows<T, KEYS_WINDOW>(a, st);
  if (e) return e;
  return join_launch<T>(a, st);
}
cudaError_t launch_window_attn(const ChunkDev& c, int dtype, const tlf_attn_window_args& args, void* scratch, int num_sms,
                               cudaStream_t st) {
  if (args.window == 0 && args.kv_format == TLF_KV_PLAIN) return launch_chunk_attn(c, dtype, plain_args(args), scratch, num_sms, st);
  const WindowPath p = window_path(c, dtype, args, num_sms);
  char* s = static_cast<char*>(scratch);
  ChunkAttn a{};
  a.c = c;
  a.sp = ChunkSplit{pow2_log(std::max(1, p.rt / c.G)), 6, p.pad};
  a.q = args.q;
  a.qs = args.q_stride ? args.q_stride : (long long)c.Hq * c.hd;
  a.out = args.out;
  a.os = args.out_stride ? args.out_stride : (long long)c.Hq * c.hd;
  a.lse = args.lse;
  a.scale = (args.scale != 0.f ? args.scale : 1.f / sqrtf((float)c.hd)) * LOG2E;
  a.ctas = p.ctas;
  a.rows = p.rt;
  a.werr = c.err ? c.err : reinterpret_cast<uint32_t*>(s + p.werr);
  a.part_o = reinterpret_cast<float*>(s);
  a.part_ml = reinterpret_cast<float2*>(s + p.part_ml);
  a.join = reinterpret_cast<int4*>(s + p.join);
  a.window = args.window > 0 ? args.window : 0x7fffffff;
  a.first = args.window > 0 ? args.n_first : 0;
  return dtype == TLF_DTYPE_BF16 ? window_launch<bf16>(a, args.kv_format, p.four, st) : window_launch<float>(a, args.kv_format, p.four, st);
}

}  // namespace tlf
