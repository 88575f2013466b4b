// Pages of a pool and who holds them: rows that take over the pages of others (tlf_cache_fork), pages in use moved to the front
// (tlf_cache_compact).
//
// Both are a plan and a copy. The plan (one CTA, or a cluster of eight for large pools and many rows) counts the free pages by
// prefix sums over the reference counts, so that the k-th free page has a number without any list that outlives the call: the result
// depends on the inputs alone. The copy runs on the whole GPU: tables, reference counts, and the entries of the pages that the plan
// names.
//
// Small calls are bound by the plan's latency and the host's call (forks of 64 rows over 1000 pages: 9.1 us in a graph; compaction of 16
// rows: 7.5 us), large ones by HBM (a compaction that reads and writes 2.7 GB: 411 us, 6.7 TB/s; the copies of 512 rows forked off 32,
// 388 MB written: 75 us, 5.2 TB/s). A fork's plan has a thread a row, which goes over the slots that the row is to have beside its full
// pages one by one, twice: 64 rows with a reserve of 8192 tokens 89 us, of 32768 283; one row 51 and 179.
#include <algorithm>

#include <cooperative_groups.h>

#include "k_kv4.cuh"

namespace cg = cooperative_groups;

namespace tlf {

constexpr int PG_THREADS = 1024, PG_CLUSTER = 8, PG_WARPS = PG_THREADS / 32;
// Most pages of a plan by one CTA. Batches of pages of 4 KB, one CTA and eight: forks 9.3 and 12.5 us (3.7 K pages), 10.3 and 13.3
// (16 K), 19.2 and 16.3 (60 K), 40.3 and 22.9 (150 K); compactions 10.4 and 12.2 us (4 K), 28.8 and 27.5 (16 K), 237 and 202 (150 K).
constexpr int FORK_ONE_PAGES = 1 << 15, COMPACT_ONE_PAGES = 1 << 13;
constexpr int COPY_THREADS = 256;

// A page's blocks: (layers x K, V x heads) of two parts with `a` and `b` bytes an entry (codes and pairs in 4 bits; b = 0).
struct PageShape {
  int blocks, a, b;
  long long bytes;
  __host__ __device__ long long block_bytes() const { return (long long)SV_PAGE * (a + b); }
};
static PageShape page_shape(int layers, int hkv, int hd, int dtype, int kv_format) {
  PageShape s{};
  s.blocks = layers * 2 * hkv;
  s.a = kv_format == TLF_KV_4BIT ? hd / 2 : hd * (dtype == TLF_DTYPE_BF16 ? 2 : 4);
  s.b = kv_format == TLF_KV_4BIT ? 4 * (hd > 64 ? hd / 64 : 1) : 0;
  s.bytes = s.blocks * s.block_bytes();
  return s;
}

// Sums over the CTAs of the plan: every thread gets the total and, in *before, the sum of the CTAs before its own. s_sum is the CTA's
// word. CS: how many CTAs, a cluster.
template <int CS>
__device__ __forceinline__ void plan_sync() {
  if constexpr (CS > 1) cg::this_cluster().sync();
  else __syncthreads();
}
template <int CS>
__device__ __forceinline__ int plan_scan(int mine, int* s_sum, int* before) {
  if constexpr (CS == 1) {
    *before = 0;
    return mine;
  } else {
    const cg::cluster_group cl = cg::this_cluster();
    const int rank = blockIdx.x % CS;
    if (threadIdx.x == 0) *s_sum = mine;
    cl.sync();
    int total = 0, b = 0;
    for (int i = 0; i < CS; ++i) {
      const int v = *cl.map_shared_rank(s_sum, i);
      total += v;
      if (i < rank) b += v;
    }
    cl.sync();  // nobody writes the word again, or leaves, before all have read it
    *before = b;
    return total;
  }
}

// The pages in runs, one a warp of the plan: p0 .. p1 - 1 is this warp's. f(page, refs) for each, 32 at a time by all lanes (page n_pages
// and refs -1 past the run's end).
struct PageRun {
  long long p0, p1;
};
template <int CS>
__device__ __forceinline__ PageRun page_run(long long n_pages) {
  const long long run = (n_pages + 32LL * PG_WARPS * CS - 1) / (32LL * PG_WARPS * CS) * 32, w = (blockIdx.x % CS) * PG_WARPS + (threadIdx.x >> 5);
  PageRun r;
  r.p0 = w * run < n_pages ? w * run : n_pages;
  r.p1 = r.p0 + run < n_pages ? r.p0 + run : n_pages;
  return r;
}
template <typename Fn>
__device__ __forceinline__ void each_page(const PageRun& r, const int* refs, Fn&& f) {
  constexpr int U = 4;
  for (long long p = r.p0 + (threadIdx.x & 31); p - (threadIdx.x & 31) < r.p1; p += 32 * U) {
    int v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = p + 32 * u < r.p1 ? refs[p + 32 * u] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) f(p + 32 * u, v[u], p + 32 * u < r.p1);
  }
}
__device__ __forceinline__ int lanes_below(unsigned mask) { return __popc(mask & ((1u << (threadIdx.x & 31)) - 1)); }

// ----------------------------------------------------------------------------
// Fork
// ----------------------------------------------------------------------------
struct ForkDev {
  int n_in, n_out, max_pages, reserve, window, first;
  long long n_pages;
  PageShape shape;
  uint8_t* pool;
  const int *table_in, *lens, *parents, *refs;
  int *table_out, *lens_out, *refs_out;
  int* pos;
  float* weight;
  uint32_t* err;
  int *eldest, *children, *len, *cut, *free;  // scratch: [n_in], [n_in], [n_out] of the parent, [n_out] lens_out, [most new pages]
};

struct ForkRow {
  int parent, len, full, need;  // parent -1: none
};
__device__ __forceinline__ ForkRow fork_row(const ForkDev& a, int b, bool report) {
  ForkRow r;
  r.parent = a.parents[b];
  r.len = 0;
  if (r.parent < -1 || r.parent >= a.n_in) {
    if (report) sv_report(a.err, DEVERR_INDEX);
    r.parent = -1;
  }
  if (r.parent >= 0) {
    r.len = a.lens[r.parent];
    if (r.len < 0 || r.len > a.max_pages * SV_PAGE) {
      if (report) sv_report(a.err, DEVERR_INDEX);
      r.len = r.len < 0 ? 0 : a.max_pages * SV_PAGE;
    }
  }
  r.full = r.len / SV_PAGE;
  const long long need = ((long long)r.len + a.reserve + SV_PAGE - 1) / SV_PAGE;
  if (need > a.max_pages && report) sv_report(a.err, DEVERR_INDEX);
  r.need = need > a.max_pages ? a.max_pages : (int)need;
  return r;
}
// The page that a table names, -1 if none.
__device__ __forceinline__ int named(int page, long long n_pages, uint32_t* err) {
  if (page >= 0 && page < n_pages) return page;
  if (page != -1) sv_report(err, DEVERR_INDEX);
  return -1;
}

constexpr int FORK_ONE_ROWS = 4096;  // most old rows of a plan by one CTA, which has their first new rows in shared memory
template <int CS>
__global__ void __launch_bounds__(PG_THREADS) k_fork_plan(ForkDev a) {
  pdl_wait();
  extern __shared__ int s_rows[];  // CS = 1: [2 n_in]
  __shared__ int s_red[33];
  __shared__ int s_sum;
  const int tid = threadIdx.x, lane = tid & 31, rank = blockIdx.x % CS;
  int* eldest = CS == 1 ? s_rows : a.eldest;
  int* children = CS == 1 ? s_rows + a.n_in : a.children;
  for (int r = rank * PG_THREADS + tid; r < a.n_in; r += PG_THREADS * CS) {
    eldest[r] = 0x7fffffff;
    children[r] = 0;
  }
  // new rows in the order of their numbers: a run of them a CTA, a run of those a thread; a thread with one keeps it
  const int rows = (a.n_out + CS - 1) / CS, b0 = min(a.n_out, rank * rows), b1 = min(a.n_out, b0 + rows);
  const int each = (b1 - b0 + PG_THREADS - 1) / PG_THREADS, t0 = min(b1, b0 + tid * each), t1 = min(b1, t0 + each);
  ForkRow first{-1, 0, 0, 0};
  if (t0 < t1) first = fork_row(a, t0, true);
  auto row_of = [&](int b) { return b == t0 ? first : fork_row(a, b, false); };
  // free pages of this warp's run, and the copy of the counts
  const PageRun run = page_run<CS>(a.n_pages);
  int count = 0;
  each_page(run, a.refs, [&](long long p, int v, bool on) {
    count += v == 0;
    if (on && a.refs_out != a.refs) a.refs_out[p] = v;
  });
  count = __reduce_add_sync(0xffffffffu, count);
  int cta_free, free_before;
  int at_free = block_scan(lane == 0 ? count : 0, s_red, &cta_free);  // lane 0: free pages of the CTA's warps before
  const int n_free = plan_scan<CS>(cta_free, &s_sum, &free_before);
  at_free = __shfl_sync(0xffffffffu, at_free, 0) + free_before;
  plan_sync<CS>();  // eldest has been started
  for (int b = t0; b < t1; ++b) {
    const ForkRow r = b == t0 ? first : fork_row(a, b, true);
    a.len[b] = r.len;
    if (r.parent >= 0) {
      atomicMin(&eldest[r.parent], b);
      atomicAdd(&children[r.parent], 1);
    }
  }
  if (CS > 1) __threadfence();
  plan_sync<CS>();
  // does slot s >= full of row b keep the parent's page? *old: that page
  auto keeps = [&](const ForkRow& r, int b, int s, int* old) {
    *old = -1;
    if (r.parent < 0) return false;
    const int page = a.table_in[(size_t)r.parent * a.max_pages + s];
    if (page < 0 || page >= a.n_pages) return false;
    *old = page;
    return (CS == 1 ? eldest[r.parent] : __ldcg(&eldest[r.parent])) == b && a.refs[page] == 1;
  };
  int want = 0, old0 = -1;
  bool keep0 = false;  // of the first row's first slot
  for (int b = t0; b < t1; ++b) {
    const ForkRow r = row_of(b);
    for (int s = r.full; s < r.need; ++s) {
      int old;
      const bool k = keeps(r, b, s, &old);
      want += !k;
      if (b == t0 && s == r.full) keep0 = k, old0 = old;
    }
  }
  int all_mine, row_before;
  int at = block_scan(want, s_red, &all_mine);
  const int total = plan_scan<CS>(all_mine, &s_sum, &row_before);
  at += row_before;
  // the first `total` free pages, in the order of their numbers
  const int taken = min(total, n_free);
  if (at_free < taken)
    each_page(run, a.refs, [&](long long p, int v, bool) {
      const unsigned is = __ballot_sync(0xffffffffu, v == 0);
      const int k = at_free + lanes_below(is);
      if (v == 0 && k < taken) a.free[k] = (int)p;
      at_free += __popc(is);
    });
  __threadfence();
  plan_sync<CS>();
  for (int b = t0; b < t1; ++b) {
    const ForkRow r = row_of(b);
    int cut = r.len;
    for (int s = r.full; s < r.need; ++s) {
      int page = -1, old = old0;
      const bool holds = s == r.full && r.len % SV_PAGE != 0;  // entries of the parent
      if (b == t0 && s == r.full ? keep0 : keeps(r, b, s, &old)) {
        page = old;
      } else {
        if (at < taken) page = __ldcg(&a.free[at]);
        else sv_report(a.err, SVERR_PAGES);
        ++at;
        if (holds && old < 0) {
          sv_report(a.err, DEVERR_INDEX);
          page = -1;
        }
      }
      if (holds && page < 0) cut = r.full * SV_PAGE;
      a.table_out[(size_t)b * a.max_pages + s] = page;
    }
    a.cut[b] = cut;
  }
  if constexpr (CS == 1)
    for (int r = tid; r < a.n_in; r += PG_THREADS) {
      a.eldest[r] = eldest[r];
      a.children[r] = children[r];
    }
  if constexpr (CS > 1) cg::this_cluster().sync();
  pdl_trigger();
}

// Entries 0 .. count - 1 of a page, by the threads that call it with their number and how many they are.
__device__ __forceinline__ void copy_entries(const PageShape& sh, const uint8_t* from, uint8_t* to, int block, int count, int i0, int step) {
  const uint8_t* f = from + block * sh.block_bytes();
  uint8_t* t = to + block * sh.block_bytes();
  auto part = [&](long long off, int bytes) {
    const int wide = bytes / 16;
    constexpr int U = 4;
    for (int i = i0; i < wide; i += U * step) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * step < wide) v[u] = __ldcs(reinterpret_cast<const uint4*>(f + off) + i + u * step);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i + u * step < wide) __stcs(reinterpret_cast<uint4*>(t + off) + i + u * step, v[u]);
    }
    for (int i = wide * 16 + i0 * 4; i < bytes; i += step * 4) *reinterpret_cast<uint32_t*>(t + off + i) = *reinterpret_cast<const uint32_t*>(f + off + i);
  };
  part(0, count * sh.a);
  if (sh.b) part((long long)SV_PAGE * sh.a, count * sh.b);
}

// Work units of eight blocks a row (a warp a block); the first unit of a row also writes its table row, counts its references, and
// so on. What k_fork_plan has put into table_out, slots full .. need - 1, is only read here.
// Units differ (rows without a copy have nearly nothing to do): many small CTAs, four on an SM. 512 rows forked off 32: 75 us the call; with
// three on an SM and 1216 CTAs, as registers would have it, 85, with five (spills) 117.
__global__ void __launch_bounds__(COPY_THREADS, 4) k_fork_apply(ForkDev a, int units) {
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long jobs = (long long)a.n_out * units, all = jobs + a.n_in;
  for (long long job = blockIdx.x; job < all; job += gridDim.x) {
    if (job >= jobs) {  // an old row gives its pages up, less what its new rows take
      const int r = (int)(job - jobs), e = a.eldest[r], n = a.children[r];
      const int len = n > 0 ? a.len[e] : 0, full = len / SV_PAGE;
      const long long need = ((long long)len + a.reserve + SV_PAGE - 1) / SV_PAGE;
      for (int s = tid; s < a.max_pages; s += COPY_THREADS) {
        const int page = named(a.table_in[(size_t)r * a.max_pages + s], a.n_pages, a.err);
        if (page < 0) continue;
        int d = -1;
        if (n > 0) {
          if (s < full) d += (a.window > 0 && 64LL * (s + 1) <= (long long)len - a.window + 1 && 64LL * s >= a.first) ? 0 : n;
          else if (s < need) d += a.table_out[(size_t)e * a.max_pages + s] == page;
        }
        if (d) atomicAdd(&a.refs_out[page], d);
      }
      continue;
    }
    const int b = (int)(job / units), unit = (int)(job % units), len = a.len[b], full = len / SV_PAGE;
    int parent = a.parents[b];
    if (parent >= a.n_in) parent = -1;
    const int* in = a.table_in + (size_t)max(parent, 0) * a.max_pages;
    int* out = a.table_out + (size_t)b * a.max_pages;
    const long long need = ((long long)len + a.reserve + SV_PAGE - 1) / SV_PAGE;
    if (unit == 0) {
      for (int s = tid; s < a.max_pages; s += COPY_THREADS) {
        if (s < full) {
          const bool gone = a.window > 0 && 64LL * (s + 1) <= (long long)len - a.window + 1 && 64LL * s >= a.first;
          const int page = in[s];
          out[s] = gone || page < 0 || page >= a.n_pages ? -1 : page;
        } else if (s >= need) {
          out[s] = -1;
        } else {
          const int page = out[s];
          const bool kept = parent >= 0 && a.eldest[parent] == b && page == in[s];
          if (page >= 0 && !kept) atomicAdd(&a.refs_out[page], 1);
        }
      }
      if (tid == 0) a.lens_out[b] = a.cut[b];
    }
    const int left = len % SV_PAGE;
    if (left == 0 || full >= a.max_pages || parent < 0) continue;
    const int from = in[full], to = out[full];
    if (to < 0 || to == from || from < 0 || from >= a.n_pages) continue;
    const int block = unit * (COPY_THREADS / 32) + warp;
    if (block < a.shape.blocks) copy_entries(a.shape, a.pool + from * a.shape.bytes, a.pool + to * a.shape.bytes, block, left, lane, 32);
    if (unit == 0 && tid < left) {
      if (a.pos) a.pos[(long long)to * SV_PAGE + tid] = a.pos[(long long)from * SV_PAGE + tid];
      if (a.weight) a.weight[(long long)to * SV_PAGE + tid] = a.weight[(long long)from * SV_PAGE + tid];
    }
  }
}

struct ForkScratch {
  size_t eldest, children, len, cut, free, total;
};
static ForkScratch fork_layout(const tlf_fork_args& a) {
  ForkScratch s{};
  size_t o = 0;
  auto take = [&](size_t n) { const size_t at = o; o = (o + n * 4 + 255) / 256 * 256; return at; };
  s.eldest = take(a.n_in);
  s.children = take(a.n_in);
  s.len = take(a.n_out);
  s.cut = take(a.n_out);
  const long long most = ((long long)a.reserve + 2 * SV_PAGE - 2) / SV_PAGE + 1;  // new pages of a row
  s.free = take((size_t)std::min<double>((double)a.n_pages, (double)a.n_out * std::min<long long>(a.max_pages, most)));
  s.total = o;
  return s;
}
size_t fork_scratch(const tlf_fork_args& a) { return fork_layout(a).total; }

cudaError_t launch_fork(const tlf_fork_args& a, void* scratch, int num_sms, cudaStream_t st) {
  const ForkScratch s = fork_layout(a);
  char* m = static_cast<char*>(scratch);
  auto at = [&](size_t o) { return reinterpret_cast<int*>(m + o); };
  const ForkDev d{a.n_in, a.n_out, a.max_pages, a.reserve, a.window, a.n_first, a.n_pages,
                  page_shape(a.n_layers, a.n_kv_heads, a.head_dim, a.dtype, a.kv_format), static_cast<uint8_t*>(a.pool), a.page_table,
                  a.lens, a.parents, a.refs, a.table_out, a.lens_out, a.refs_out, a.entry_pos, a.entry_weight, a.err,
                  at(s.eldest), at(s.children), at(s.len), at(s.cut), at(s.free)};
  const bool one = a.n_in <= FORK_ONE_ROWS && a.n_out <= FORK_ONE_ROWS && a.n_pages <= FORK_ONE_PAGES;
  if (cudaError_t e = one ? launch_k(k_fork_plan<1>, dim3(1), dim3(PG_THREADS), (size_t)a.n_in * 8, st, d)
                          : launch_cluster(k_fork_plan<PG_CLUSTER>, dim3(PG_CLUSTER), dim3(PG_THREADS), PG_CLUSTER, 0, st, d))
    return e;
  const int units = std::max(1, (d.shape.blocks + COPY_THREADS / 32 - 1) / (COPY_THREADS / 32));
  const long long jobs = (long long)a.n_out * units + a.n_in;
  return launch_k(k_fork_apply, dim3((unsigned)std::min<long long>(jobs, 32LL * num_sms)), dim3(COPY_THREADS), 0, st, d, units);
}

// ----------------------------------------------------------------------------
// Compact
// ----------------------------------------------------------------------------
struct CompactDev {
  int n, max_pages;
  long long n_pages;
  PageShape shape;
  uint8_t* pool;
  const int *table_in, *refs;
  int *table_out, *refs_out, *n_live;
  int* pos;
  float* weight;
  uint32_t* err;
  int *hole, *mover, *rank, *count;  // scratch: [n_pages] target and source of the k-th move, [n_pages] k of a page that moves (-1: nobody counts the page), moves
};

template <int CS>
__global__ void __launch_bounds__(PG_THREADS) k_compact_plan(CompactDev a) {
  pdl_wait();
  __shared__ int s_red[33];
  __shared__ int s_sum;
  const int lane = threadIdx.x & 31;
  const PageRun run = page_run<CS>(a.n_pages);
  int count = 0, cta, before;
  each_page(run, a.refs, [&](long long, int v, bool) { count += v > 0; });
  count = __reduce_add_sync(0xffffffffu, count);
  int at = block_scan(lane == 0 ? count : 0, s_red, &cta);  // lane 0: pages in use of the CTA's warps before
  const int live = plan_scan<CS>(cta, &s_sum, &before);
  at = __shfl_sync(0xffffffffu, at, 0) + before;
  // pages in use that stay: those before page `live`, whose run knows how many they are
  int below = -1;
  {
    int n = at;
    if (run.p0 <= live && live < run.p1) {
      each_page(run, a.refs, [&](long long p, int v, bool) { n += __popc(__ballot_sync(0xffffffffu, v > 0 && p < live)); });
      below = n;
    }
  }
  if (live >= a.n_pages) below = live;
  int any;
  below = plan_scan<CS>(block_sum(lane == 0 && below >= 0 && live < a.n_pages ? below : 0, s_red), &s_sum, &any);
  if (live >= a.n_pages) below = live;
  each_page(run, a.refs, [&](long long p, int v, bool on) {
    const unsigned used = __ballot_sync(0xffffffffu, v > 0);
    const int k = at + lanes_below(used);  // pages in use before p
    if (on) {
      if (p < live && v <= 0) a.hole[p - k] = (int)p;
      if (p >= live && v > 0) a.mover[k - below] = (int)p;
      a.rank[p] = v <= 0 ? -1 : p < live ? 0 : k - below;
    }
    at += __popc(used);
  });
  if (blockIdx.x % CS == 0 && threadIdx.x == 0) {
    *a.n_live = live;
    *a.count = live - below;
  }
  pdl_trigger();
}

__global__ void __launch_bounds__(COPY_THREADS) k_compact_apply(CompactDev a, int units) {
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, moves = *a.count, live = *a.n_live;
  const long long threads = (long long)gridDim.x * COPY_THREADS, me = (long long)blockIdx.x * COPY_THREADS + tid;
  const bool same = a.refs_out == a.refs;
  for (long long i = me; i < (long long)a.n * a.max_pages; i += threads) {
    const int page = named(a.table_in[i], a.n_pages, a.err);
    int to = page;
    if (page >= 0) {
      const int k = a.rank[page];  // (refs may be changing)
      if (k < 0) to = -1;
      else if (page >= live) to = a.hole[k];
      if (to < 0) sv_report(a.err, DEVERR_INDEX);
    }
    a.table_out[i] = to;
  }
  if (!same)
    for (long long p = me; p < a.n_pages; p += threads) {
      const int v = a.refs[p];
      if (p < live ? v > 0 : true) a.refs_out[p] = p < live ? v : 0;
    }
  for (long long k = me; k < moves; k += threads) {
    const int from = a.mover[k], to = a.hole[k], v = a.refs[from];
    a.refs_out[to] = v;
    if (same) a.refs_out[from] = 0;
  }
  for (long long job = blockIdx.x; job < (long long)moves * units; job += gridDim.x) {
    const long long k = job / units;
    const int unit = (int)(job % units), from = a.mover[k], to = a.hole[k], block = unit * (COPY_THREADS / 32) + warp;
    if (block < a.shape.blocks) copy_entries(a.shape, a.pool + from * a.shape.bytes, a.pool + to * a.shape.bytes, block, SV_PAGE, lane, 32);
    if (unit == 0 && tid < SV_PAGE) {
      if (a.pos) a.pos[(long long)to * SV_PAGE + tid] = a.pos[(long long)from * SV_PAGE + tid];
      if (a.weight) a.weight[(long long)to * SV_PAGE + tid] = a.weight[(long long)from * SV_PAGE + tid];
    }
  }
}

struct CompactScratch {
  size_t hole, mover, rank, count, total;
};
static CompactScratch compact_layout(const tlf_compact_args& a) {
  CompactScratch s{};
  size_t o = 0;
  auto take = [&](size_t n) { const size_t at = o; o = (o + n * 4 + 255) / 256 * 256; return at; };
  s.hole = take((size_t)a.n_pages);
  s.mover = take((size_t)a.n_pages);
  s.rank = take((size_t)a.n_pages);
  s.count = take(1);
  s.total = o;
  return s;
}
size_t compact_scratch(const tlf_compact_args& a) { return compact_layout(a).total; }

cudaError_t launch_compact(const tlf_compact_args& a, void* scratch, int num_sms, cudaStream_t st) {
  const CompactScratch s = compact_layout(a);
  char* m = static_cast<char*>(scratch);
  auto at = [&](size_t o) { return reinterpret_cast<int*>(m + o); };
  const CompactDev d{a.n, a.max_pages, a.n_pages, page_shape(a.n_layers, a.n_kv_heads, a.head_dim, a.dtype, a.kv_format),
                     static_cast<uint8_t*>(a.pool), a.page_table, a.refs, a.table_out, a.refs_out, a.n_live, a.entry_pos,
                     a.entry_weight, a.err, at(s.hole), at(s.mover), at(s.rank), at(s.count)};
  if (cudaError_t e = a.n_pages <= COMPACT_ONE_PAGES ? launch_k(k_compact_plan<1>, dim3(1), dim3(PG_THREADS), 0, st, d)
                                             : launch_cluster(k_compact_plan<PG_CLUSTER>, dim3(PG_CLUSTER), dim3(PG_THREADS), PG_CLUSTER, 0, st, d))
    return e;
  const int units = std::max(1, (d.shape.blocks + COPY_THREADS / 32 - 1) / (COPY_THREADS / 32));
  return launch_k(k_compact_apply, dim3(8 * num_sms), dim3(COPY_THREADS), 0, st, d, units);
}

}  // namespace tlf
