// Eviction from paged caches by accumulated attention weight (tlf_cache_evict).
//
// k_evict_select: every entry has an ordered 32-bit key (protected: the largest; NaN: the smallest); a radix select over the
// key, 11 bits a level, finds the budget-th largest key; ties are settled by entry index. Entries that stay and lie beyond the
// budget ("movers") are matched, both in order, with the places below it that become free ("holes"): sources and targets are
// then disjoint, so the moves need no order among themselves and each moved entry is read and written once. A row is shared by
// a cluster of up to eight CTAs, each with a run of entries; histograms and counts meet through distributed shared memory.
// k_evict_move copies the movers' keys and values, all layers and heads.
//
// The selection is bound by the latency of its steps (32 rows of 2000 entries, one CTA each: 9 us; 4 rows of 32k, clusters of
// eight: 29 us, one CTA each 98 us), the moves by HBM (25,000 entries of 8 KB: 62 us, 6.7 TB/s).
#include <algorithm>

#include <cooperative_groups.h>

#include "k_serve.cuh"

namespace cg = cooperative_groups;

namespace tlf {

constexpr int EV_THREADS = 1024;
constexpr int EV_CACHED = 40 * 1024;  // most keys that a CTA keeps in shared memory
constexpr int EV_CLUSTER = 8;         // most CTAs that share a row
constexpr int EV_BITS = 11, EV_BINS = 1 << EV_BITS;

struct EvictDev {
  int n, max_pages, budget, n_first, n_recent;
  long long n_pages;
  const int *page_table, *lens, *next_pos, *pos_in;
  int* pos_out;
  const float* w_in;
  float* w_out;
  int* lens_out;
  uint32_t* err;
  int* moves;      // [n] moves of each row
  int2* move;      // [n][budget] (source entry, target entry)
};

__device__ __forceinline__ uint32_t ordered_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 weighs what 0 does
  if (w != w) return 0u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(EV_THREADS) k_evict_select(EvictDev a, int cached, int cs) {
  pdl_wait();
  extern __shared__ uint32_t s_key[];  // [cached] of this CTA's entries, entry i at i + i / 32: a thread reads a run of them
  __shared__ int s_hist[3][EV_BINS];
  __shared__ int s_red[33];
  __shared__ int s_count[2][2];  // of this CTA: ties; holes, movers
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  const cg::cluster_group cl = cg::this_cluster();
  const int b = blockIdx.x / cs, rank = blockIdx.x % cs, tid = threadIdx.x;
  const int* table = a.page_table + (size_t)b * a.max_pages;
  int len = a.lens[b];
  const int next = a.next_pos[b];
  if (len < 0 || len > a.max_pages * SV_PAGE) {
    if (tid == 0) sv_report(a.err, DEVERR_INDEX);
    len = len < 0 ? 0 : a.max_pages * SV_PAGE;
  }
  const int budget = a.budget, kept = min(len, budget);
  const int each = (len + cs - 1) / cs, v0 = min(len, rank * each), v1 = min(len, v0 + each);  // this CTA's entries
  const bool same = a.pos_out == a.pos_in && a.w_out == a.w_in;  // what stays need not be copied
  auto slot = [&](int e) -> long long {  // of an entry in the side tables, -1: no such page
    const int page = table[e / SV_PAGE];
    if (page < 0 || page >= a.n_pages) {
      sv_report(a.err, DEVERR_INDEX);
      return -1;
    }
    return (long long)page * SV_PAGE + e % SV_PAGE;
  };
  auto copy = [&](int from, int to) {
    const long long s = slot(from), d = slot(to);
    if (s < 0 || d < 0) return;
    a.pos_out[d] = a.pos_in[s];
    a.w_out[d] = a.w_in[s];
  };
  auto make_key = [&](int e) -> uint32_t {
    const long long s = slot(e);
    if (s < 0) return 0u;
    const long long p = a.pos_in[s];
    const float w = a.w_in[s];
    return p < a.n_first || p >= (long long)next - a.n_recent ? 0xFFFFFFFFu : ordered_key(w);
  };
  if (len <= budget) {
    if (!same)
      for (int e = v0 + tid; e < v1; e += EV_THREADS) copy(e, e);
    if (tid == 0 && rank == 0) {
      a.lens_out[b] = kept;
      a.moves[b] = 0;
    }
    pdl_trigger();
    return;
  }
  const bool in_smem = each <= cached;
  auto key = [&](int e) { return in_smem ? s_key[(e - v0) + ((e - v0) >> 5)] : make_key(e); };
  for (int i = tid; i < 3 * EV_BINS; i += EV_THREADS) (&s_hist[0][0])[i] = 0;
  if (tid == 0) {
    s_prefix = 0;
    s_need = budget;
  }
  __syncthreads();

  // the budget-th largest key: s_need counts what is still wanted among the keys with the prefix
#pragma unroll
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
    const uint32_t prefix = s_prefix;
    const int need = s_need;
    if (level == 0) {
      for (int e = v0 + tid; e < v1; e += EV_THREADS) {
        const uint32_t k = make_key(e);
        if (in_smem) s_key[(e - v0) + ((e - v0) >> 5)] = k;
        atomicAdd(&s_hist[0][k >> 21], 1);
      }
    } else {
      for (int e = v0 + tid; e < v1; e += EV_THREADS) {
        const uint32_t k = key(e);
        if ((k >> (shift + bits)) == prefix) atomicAdd(&s_hist[level][(k >> shift) & ((1u << bits) - 1u)], 1);
      }
    }
    if (cs > 1) cl.sync();
    else __syncthreads();
    // a thread has two bins, from the largest
    const int hi = EV_BINS - 1 - 2 * tid;
    int c0 = 0, c1 = 0;
    if (cs > 1) {
      for (int r = 0; r < cs; ++r) {
        const int2 h = *reinterpret_cast<const int2*>(cl.map_shared_rank(s_hist[level], r) + hi - 1);
        c0 += h.y;
        c1 += h.x;
      }
    } else {
      c0 = s_hist[level][hi];
      c1 = s_hist[level][hi - 1];
    }
    const int before = block_scan(c0 + c1, s_red, (int*)nullptr);
    if (before < need && before + c0 + c1 >= need) {
      const bool first = before + c0 >= need;
      s_prefix = (prefix << bits) | (uint32_t)(first ? hi : hi - 1);
      s_need = need - before - (first ? 0 : c0);
    }
    __syncthreads();
  }
  const uint32_t kth = s_prefix;
  const int ties = s_need;  // entries with that key that stay: the first ones

  // a thread owns a run of entries; ties, holes and movers are counted in order of entries
  const int run = (each + EV_THREADS - 1) / EV_THREADS, e0 = min(v1, v0 + tid * run), e1 = min(v1, e0 + run);
  auto before_me = [&](int which, int what) {  // sum of a count over the CTAs with entries before this one's
    int n = 0;
    for (int r = 0; r < rank; ++r) n += cl.map_shared_rank(&s_count[0][0], r)[2 * which + what];
    return n;
  };
  int eq = 0, total;
  for (int e = e0; e < e1; ++e) eq += key(e) == kth;
  int rank0 = block_scan(eq, s_red, &total);
  if (cs > 1) {
    if (tid == 0) s_count[0][0] = total;
    cl.sync();
    rank0 += before_me(0, 0);
  }
  int holes = 0, movers = 0, at = rank0;
  for (int e = e0; e < e1; ++e) {
    const uint32_t k = key(e);
    const bool stays = k > kth || (k == kth && at < ties);
    at += k == kth;
    holes += !stays && e < budget;
    movers += stays && e >= budget;
  }
  int n_holes, n_movers;
  int hole = block_scan(holes, s_red, &n_holes), mover = block_scan(movers, s_red, &n_movers);
  if (cs > 1) {
    if (tid == 0) {
      s_count[1][0] = n_holes;
      s_count[1][1] = n_movers;
    }
    cl.sync();
    hole += before_me(1, 0);
    mover += before_me(1, 1);
    n_movers = 0;
    for (int r = 0; r < cs; ++r) n_movers += cl.map_shared_rank(&s_count[0][0], r)[3];
  }
  int2* move = a.move + (size_t)b * budget;
  at = rank0;
  for (int e = e0; e < e1; ++e) {
    const uint32_t k = key(e);
    const bool stays = k > kth || (k == kth && at < ties);
    at += k == kth;
    if (!stays && e < budget) move[hole++].y = e;
    if (stays && e >= budget) move[mover++].x = e;
    if (in_smem) s_key[(e - v0) + ((e - v0) >> 5)] = stays;
    else if (!same && stays && e < budget) copy(e, e);
  }
  if (cs > 1) cl.sync();  // the list of moves is complete
  else __syncthreads();
  if (tid == 0 && rank == 0) {
    a.lens_out[b] = kept;
    a.moves[b] = n_movers;
  }
  // side tables: what keeps its place, and the moved (their sources lie beyond the budget and are not written)
  if (!same && in_smem)
    for (int e = v0 + tid; e < min(v1, budget); e += EV_THREADS)
      if (key(e)) copy(e, e);
  for (int i = rank * EV_THREADS + tid; i < n_movers; i += cs * EV_THREADS) copy(move[i].x, move[i].y);
  pdl_trigger();
}

// A CTA takes one move of a row at a time: 16-byte units of its segments (layer, K or V, head), four a thread in flight.
constexpr int EV_MOVE_THREADS = 128;
__global__ void __launch_bounds__(EV_MOVE_THREADS) k_evict_move(EvictDev a, uint4* pool, int segs, int unit_log) {
  pdl_wait();
  const int b = blockIdx.y, n = a.moves[b], per = segs << unit_log;
  const int* table = a.page_table + (size_t)b * a.max_pages;
  const long long page_units = (long long)per * SV_PAGE;
  for (int m = blockIdx.x; m < n; m += gridDim.x) {
    const int2 mv = a.move[(size_t)b * a.budget + m];
    const int ps = table[mv.x / SV_PAGE], pd = table[mv.y / SV_PAGE];
    if (ps < 0 || ps >= a.n_pages || pd < 0 || pd >= a.n_pages) continue;
    const uint4* from = pool + ps * page_units + ((mv.x % SV_PAGE) << unit_log);
    uint4* to = pool + pd * page_units + ((mv.y % SV_PAGE) << unit_log);
    for (int u0 = threadIdx.x; u0 < per; u0 += 4 * EV_MOVE_THREADS) {
      uint4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int u = u0 + i * EV_MOVE_THREADS;
        if (u < per) v[i] = from[((long long)(u >> unit_log) * SV_PAGE << unit_log) + (u & ((1 << unit_log) - 1))];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int u = u0 + i * EV_MOVE_THREADS;
        if (u < per) to[((long long)(u >> unit_log) * SV_PAGE << unit_log) + (u & ((1 << unit_log) - 1))] = v[i];
      }
    }
  }
  pdl_trigger();
}

// The budget as far as a row can reach it: a caller may give any number for no limit.
static int evict_budget(const tlf_evict_args& a) { return std::min(a.budget, a.max_pages * SV_PAGE); }

size_t evict_scratch(const tlf_evict_args& a) {
  return ((size_t)a.n * 4 + 15) / 16 * 16 + (size_t)a.n * evict_budget(a) * sizeof(int2);
}

cudaError_t launch_evict(const tlf_evict_args& a, void* scratch, int num_sms, cudaStream_t st) {
  EvictDev d{a.n, a.max_pages, evict_budget(a), a.n_first, a.n_recent, a.n_pages, a.page_table, a.lens, a.next_pos, a.pos_in,
             a.pos_out, a.weight_in, a.weight_out, a.lens_out, a.err, static_cast<int*>(scratch),
             reinterpret_cast<int2*>(static_cast<char*>(scratch) + ((size_t)a.n * 4 + 15) / 16 * 16)};
  // CTAs of a row: as many as leave one to an SM
  int cs = 1;
  while (cs < EV_CLUSTER && a.n * cs * 2 <= num_sms && (long long)a.max_pages * SV_PAGE > 4096 * cs) cs *= 2;
  const int cached = (int)std::min<long long>(EV_CACHED, ((long long)a.max_pages * SV_PAGE + cs - 1) / cs);
  const int smem = 4 * (cached + cached / 32 + 1);
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_evict_select), 4 * (EV_CACHED + EV_CACHED / 32 + 1))) return e;
  if (cudaError_t e = launch_cluster(k_evict_select, dim3(a.n * cs), dim3(EV_THREADS), cs, smem, st, d, cached, cs)) return e;
  const int segs = a.n_layers * 2 * a.n_kv_heads, units = a.head_dim * (a.dtype == TLF_DTYPE_BF16 ? 2 : 4) / 16;
  int unit_log = 0;
  while ((1 << unit_log) < units) ++unit_log;
  return launch_k(k_evict_move, dim3(std::max(1, num_sms * 16 / a.n), a.n), dim3(EV_MOVE_THREADS), 0, st, d,
                  static_cast<uint4*>(a.pool), segs, unit_log);
}

}  // namespace tlf
