// What the attention kernels of chunks share (k_chunk.cu, k_chunk4.cu): arguments, the plan of a CTA's share, items, notes for the
// join, and wrappers of instructions.
#pragma once

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
  float* scores;   // k_chunk_mma: [T][Hq][max_pages * 64] scores that it leaves for the weights, or NULL
  uint32_t* werr;  // error word of the waits: the caller's, or one in the scratch
  float* part_o;   // [2 ctas][rows][hd]; of k_chunk_pair [2 ctas][hd / 4][rows][4]
  float2* part_ml; // [2 ctas][rows]
  int4* join;      // [ctas] what each CTA leaves to k_chunk_join
  int window, first;  // tlf_attn_window's; 2^31 - 1 and 0 where there is no window
};

// What a kernel's keys are: every entry up to the query's, of a cache in the dtype; those of a window; those of a window, of a
// cache in 4 bits.
enum ChunkKeys { KEYS_ALL = 0, KEYS_WINDOW = 1, KEYS_4BIT = 2 };
template <int MODE>
__device__ __forceinline__ auto split_of(const ChunkAttn& a) {
  if constexpr (MODE == KEYS_ALL) return a.sp;
  else return WindowSplit{a.sp, a.window, a.first};
}
// Number in its row of an item's block i; the last entry of a row that the window hides from a query at entry `see`.
template <int MODE>
__device__ __forceinline__ int block_at(int i, int sinks, int skip) { return MODE == KEYS_ALL || i < sinks ? i : i + skip; }
__device__ __forceinline__ int hidden_to(int see, int window) { return see < window ? -1 : see - window; }

// The n lowest bits of 64 (n may lie outside of 0..64).
__device__ __forceinline__ uint64_t low_bits(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// base[b] = blocks of the rows before b; base[n] = all. By the whole block.
template <class Split>
__device__ __forceinline__ void chunk_plan(const ChunkDev& c, const Split& sp, long long* base, long long* red) {
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
  return all > 0 ? (all + a.ctas - 1) / a.ctas : 1;
}

// The item that holds block `pos` of the flat order.
struct ChunkItem {
  int b, h, t, nb;     // row, kv head, tile, its blocks
  int t0, s0, ql, len; // the row's first new token, old entries, new tokens, entries
  long long first;     // the item's first block in the flat order (may lie behind `pos`, which then is in its pad)
  int skip;            // blocks behind those of the first entries that the window leaves out
};
template <class Split>
__device__ __forceinline__ ChunkItem chunk_item(const ChunkDev& c, const Split& sp, const long long* base, long long pos) {
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
  it.first = base[lo] + it.h * per + sp.before(it.s0, it.ql, it.t) + sp.pad;
  it.skip = 0;
  if constexpr (std::is_same<Split, WindowSplit>::value) it.skip = sp.skip(it.s0, it.t);
  return it;
}

// The same where `it` is the item before, which ends at `pos` (nb = 0: none yet): a row's tiles and heads follow each other in the flat
// order, so that only rows are searched for. (A search is 1.5 us of a warp. 4 x 2048 tokens under a window of 512 in
// k_chunk_pair: 71.0 us with one an item, 67.9 so; where it costs registers, or items are long, it gains nothing.)
template <class Split>
__device__ __forceinline__ void chunk_item_next(const ChunkDev& c, const Split& sp, const long long* base, long long pos, ChunkItem& it) {
  const int tiles = sp.tiles(it.ql);
  if (it.nb == 0 || (it.t + 1 == tiles && it.h + 1 == c.Hkv)) {
    it = chunk_item(c, sp, base, pos);
    return;
  }
  it.first = pos + sp.pad;
  if (++it.t == tiles) {
    it.t = 0;
    ++it.h;
  }
  it.nb = sp.blocks(it.s0, it.ql, it.t);
  if constexpr (std::is_same<Split, WindowSplit>::value) it.skip = sp.skip(it.s0, it.t);
}

// The first CTA whose share starts inside an item notes it: {the tile's first token, kv head, rows, parts}, parts = 0 where there
// is none. CTA c's first item has its part at 2c if it began in an earlier share, the part of an item that goes on past its
// share is at 2c + 1. One thread of every CTA calls this, before any wait; it: what the CTA's share starts with, or NULL.
__device__ __forceinline__ void join_note(const ChunkAttn& a, const ChunkItem* it, long long per) {
  int4 j = make_int4(0, 0, 0, 0);
  const long long pos = blockIdx.x * per;
  if (it && it->first < pos && it->first >= pos - per) {
    const int qt = 1 << a.sp.qt_log, last = (int)((it->first + it->nb - 1) / per);  // the last CTA with a part
    j = make_int4(it->t0 + it->t * qt, it->h, min(qt, it->ql - it->t * qt) * a.c.G, last - (int)blockIdx.x + 2);
  }
  a.join[blockIdx.x] = j;
}

// The parts of the kernels on pairs of 128-row tiles, whose threads have a row each: they leave four dims of all rows side by side, so
// that a warp writes whole lines (row by row, 16 bytes a lane in 32 lines, a part of 256 rows took 4 us).
constexpr int PAIR_ROWS = 256;
__device__ __forceinline__ size_t pair_part(int slot, int row, int d, int hd) {  // of 16 bytes from dim d on
  return (size_t)slot * PAIR_ROWS * hd + ((size_t)(d >> 2) * PAIR_ROWS + row) * 4 + (d & 3);
}

__device__ __forceinline__ void bar_named(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Barrier `id` of `threads` threads; whether any of them has p.
__device__ __forceinline__ bool bar_any(int id, int threads, bool p) {
  int r;
  asm volatile(
      "{\n\t.reg .pred q, s;\n\t"
      "setp.ne.s32 q, %3, 0;\n\t"
      "bar.red.or.pred s, %1, %2, q;\n\t"
      "selp.s32 %0, 1, 0, s;\n\t}"
      : "=r"(r)
      : "r"(id), "r"(threads), "r"((int)p)
      : "memory");
  return r != 0;
}

// D(tmem) (+)= A(tmem) * B(smem desc)
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t at, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(at), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_put_16(uint32_t taddr, const uint32_t* r) {  // completes at the next wait::st
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// One thread of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r != 0;
}
__device__ __forceinline__ void tmem_st_wait_done() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

struct PairSeg {  // a CTA's part of an item: blocks kb0 .. kb1 - 1 of nb, of which tile x has the first e[x]; nb = 0: no more
  int b, h, token0, see0, nq[2], e[2], kb0, kb1, nb, none;
  static constexpr int RING = 4;
};

// Joins the parts of shared items (k_chunk_join, k_pair_join).
cudaError_t launch_chunk_join(const ChunkAttn& a, int dtype, cudaStream_t st);

}  // namespace tlf
