// The work split of the chunk attention (k_chunk.cu), on the host and on the device.
#pragma once

namespace tlf {

// A row's queries are cut into tiles of qt, its cache into blocks of bk entries (both powers of two). Tile t of a row of ql
// new tokens behind s0 = len - ql old entries sees the first nb(t) blocks; an item is a tile of one kv head. All items'
// blocks lie in one flat order (row, head, tile, block), of which every CTA takes an equal share: it streams the same number
// of blocks whatever the lengths, and items that it shares with other CTAs are joined afterwards. nb is at least 1, so that
// queries that see nothing are answered too. An item also costs its CTA something beside its blocks (look-ups, joining the
// warps' parts, writing out): it counts as `pad` more blocks, which lie before its own in the flat order and which nobody
// works on. The sums over tiles are closed forms: no list of items is ever written.
struct ChunkSplit {
  int qt_log, bk_log, pad;

  __host__ __device__ int tiles(int ql) const { return (ql + (1 << qt_log) - 1) >> qt_log; }
  __host__ __device__ int blocks(int s0, int ql, int t) const {
    const long long q = ((long long)t + 1) << qt_log;
    const long long keys = s0 + (q < ql ? q : (long long)ql);
    return keys <= 0 ? 1 : (int)((keys + (1 << bk_log) - 1) >> bk_log);
  }
  // sum over u = 1 .. n of ceil(u / 2^r)
  __host__ __device__ static long long ceil_sum(long long n, int r) {
    const long long q = n >> r, rem = n & ((1LL << r) - 1);
    return ((q * (q + 1) / 2) << r) + rem * (q + 1);
  }
  // blocks of the row's first t tiles (of one head), with what the items count beside; only its last tile may be cut short, so tiles before it are whole
  __host__ __device__ long long before(int s0, int ql, int t) const {
    const int nt = tiles(ql), whole = t < nt ? t : nt - 1;
    if (t <= 0 || nt <= 0) return 0;
    long long sum;
    if (qt_log >= bk_log) {  // nb(i) = max(1, c + (i + 1) m)
      const int ml = qt_log - bk_log;
      const long long m = 1LL << ml, c = -((-(long long)s0) >> bk_log);
      long long k0 = c >= 1 ? 0 : ((1 - c + m - 1) >> ml) - 1;  // tiles with c + (i + 1) m < 1
      if (k0 < 0) k0 = 0;
      if (k0 > whole) k0 = whole;
      sum = k0 + (whole - k0) * c + ((long long)whole * (whole + 1) / 2 - k0 * (k0 + 1) / 2) * m;
    } else {  // nb(i) = max(1, ceil((a + i + 1) / r))
      const int rl = bk_log - qt_log;
      const long long a = -((-(long long)s0) >> qt_log);
      long long k0 = a >= 0 ? 0 : -a;
      if (k0 > whole) k0 = whole;
      sum = k0 + ceil_sum(a + whole > 0 ? a + whole : 0, rl) - ceil_sum(a + k0 > 0 ? a + k0 : 0, rl);
    }
    return (t < nt ? sum : sum + blocks(s0, ql, nt - 1)) + (long long)t * pad;
  }
  // the tile that holds block `at` (counted from the row's first) of the row's head
  __host__ __device__ int tile_of(int s0, int ql, long long at) const {
    int lo = 0, hi = tiles(ql);  // before(lo) <= at < before(hi)
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (before(s0, ql, mid) <= at) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

// The split of the tensor-core weights (k_weigh_tc): a row's cache in blocks of 2^bk_log entries, its queries in tiles of
// 2^qt_log <= 2^bk_log. A unit is one tile that sees something of a block, for one kv head; the flat order is (row, block,
// head, tile), shared out like the above. Tile t sees block kb when its last query sees the block's first entry:
// t >= first(kb), the tile of query kb 2^bk_log - s0.
struct WeighSplit {
  int qt_log, bk_log;

  __host__ __device__ int tiles(int ql) const { return (ql + (1 << qt_log) - 1) >> qt_log; }
  __host__ __device__ int blocks(int s0, int ql) const {  // a row without new tokens has none
    return ql > 0 && s0 + ql > 0 ? (s0 + ql + (1 << bk_log) - 1) >> bk_log : 0;
  }
  __host__ __device__ int first(int s0, int kb) const {
    const long long t = ((long long)kb << (bk_log - qt_log)) + ((-(long long)s0) >> qt_log);
    return t > 0 ? (int)t : 0;
  }
  // units of one head in the row's first n blocks
  __host__ __device__ long long before(int s0, int ql, int n) const {
    const int ml = bk_log - qt_log;
    const long long a = -((-(long long)s0) >> qt_log);         // first(kb) = max(0, kb 2^ml - a)
    long long k0 = a < 0 ? 0 : (a >> ml) + 1;                  // blocks with first = 0
    if (k0 > n) k0 = n;
    return (long long)n * tiles(ql) - ((((long long)n * (n - 1) - k0 * (k0 - 1)) / 2 << ml) - (n - k0) * a);
  }
  // the block that holds unit `at` of the row (all heads)
  __host__ __device__ int block_of(int s0, int ql, int heads, long long at) const {
    int lo = 0, hi = blocks(s0, ql);
    while (hi - lo > 1) {
      const int mid = lo + (hi - lo) / 2;
      if (before(s0, ql, mid) * heads <= at) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

}  // namespace tlf
