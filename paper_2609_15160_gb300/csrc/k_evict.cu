// Eviction from paged caches by accumulated attention weight (tlf_cache_evict).
//
// k_evict_select, one CTA a row: every entry has an ordered 32-bit key (protected: the largest; NaN: the smallest); a radix
// select over the key's bytes finds the budget-th largest key; ties are settled by entry index. Entries that stay and lie
// beyond the budget ("movers") are matched, both in order, with the places below it that become free ("holes"): sources and
// targets are then disjoint, so the moves need no order among themselves and each moved entry is read and written once.
// k_evict_move copies the movers' keys and values, all layers and heads.
#include "k_serve.cuh"

namespace tlf {

constexpr int EV_THREADS = 1024;
constexpr int EV_CACHED = 40 * 1024;  // keys that a CTA keeps in shared memory

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
  const uint32_t u = __float_as_uint(w);
  if (w != w) return 0u;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(EV_THREADS) k_evict_select(EvictDev a, int cached) {
  pdl_wait();
  extern __shared__ uint32_t s_key[];  // [cached], entry e at e + e / 32: a thread reads a run of entries
  __shared__ int s_hist[256];
  __shared__ int s_red[33];
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int* table = a.page_table + (size_t)b * a.max_pages;
  int len = a.lens[b];
  if (len < 0 || len > a.max_pages * SV_PAGE) {
    if (tid == 0) sv_report(a.err, DEVERR_INDEX);
    len = len < 0 ? 0 : a.max_pages * SV_PAGE;
  }
  const int next = a.next_pos[b];
  auto slot = [&](int e) -> long long {  // of an entry in the side tables, -1: no such page
    const int page = table[e / SV_PAGE];
    if (page < 0 || page >= a.n_pages) {
      sv_report(a.err, DEVERR_INDEX);
      return -1;
    }
    return (long long)page * SV_PAGE + e % SV_PAGE;
  };
  auto make_key = [&](int e) -> uint32_t {
    const long long s = slot(e);
    if (s < 0) return 0u;
    const long long p = a.pos_in[s];
    if (p < a.n_first || p >= (long long)next - a.n_recent) return 0xFFFFFFFFu;
    return ordered_key(a.w_in[s]);
  };
  const int budget = a.budget, kept = min(len, budget);
  if (tid == 0) {
    a.lens_out[b] = kept;
    if (len <= budget) a.moves[b] = 0;
  }
  if (len <= budget) {
    for (int e = tid; e < len; e += EV_THREADS) {
      const long long s = slot(e);
      if (s < 0) continue;
      a.pos_out[s] = a.pos_in[s];
      a.w_out[s] = a.w_in[s];
    }
    pdl_trigger();
    return;
  }
  const bool in_smem = len <= cached;
  auto key = [&](int e) { return in_smem ? s_key[e + (e >> 5)] : make_key(e); };
  if (in_smem)
    for (int e = tid; e < len; e += EV_THREADS) s_key[e + (e >> 5)] = make_key(e);

  // the budget-th largest key, byte by byte: s_need counts what is still wanted among the keys with the prefix
  if (tid == 0) {
    s_prefix = 0;
    s_need = budget;
  }
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
    const uint32_t prefix = s_prefix;
    const int need = s_need;
    for (int e = tid; e < len; e += EV_THREADS) {
      const uint32_t k = key(e);
      if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&s_hist[(k >> shift) & 255u], 1);
    }
    __syncthreads();
    if (tid < 32) {  // bins 255 - 8 lane - i: from the largest
      int c[8], sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += c[i] = s_hist[255 - 8 * tid - i];
      int before = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, before, o);
        if (tid >= o) before += y;
      }
      before -= sum;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (before < need && before + c[i] >= need) {
          s_prefix = (prefix << 8) | (uint32_t)(255 - 8 * tid - i);
          s_need = need - before;
        }
        before += c[i];
      }
    }
    __syncthreads();
  }
  const uint32_t kth = s_prefix;
  const int ties = s_need;  // entries with that key that stay: the first ones

  // a thread owns a run of entries; ties, holes and movers are counted in order of entries
  const int run = (len + EV_THREADS - 1) / EV_THREADS, e0 = min(len, tid * run), e1 = min(len, e0 + run);
  int eq = 0;
  for (int e = e0; e < e1; ++e) eq += key(e) == kth;
  int rank = block_scan(eq, s_red, (int*)nullptr);
  const int rank0 = rank;
  int holes = 0, movers = 0;
  for (int e = e0; e < e1; ++e) {
    const uint32_t k = key(e);
    const bool stays = k > kth || (k == kth && rank < ties);
    rank += k == kth;
    holes += !stays && e < budget;
    movers += stays && e >= budget;
  }
  int total;
  int hole = block_scan(holes, s_red, (int*)nullptr), mover = block_scan(movers, s_red, &total);
  int2* move = a.move + (size_t)b * budget;
  rank = rank0;
  for (int e = e0; e < e1; ++e) {
    const uint32_t k = key(e);
    const bool stays = k > kth || (k == kth && rank < ties);
    rank += k == kth;
    if (!stays && e < budget) move[hole++].y = e;
    if (stays && e >= budget) move[mover++].x = e;
  }
  if (tid == 0) a.moves[b] = total;
  __syncthreads();
  // side tables: what keeps its place, then the moved (their sources lie beyond the budget and are not written)
  for (int e = tid; e < budget; e += EV_THREADS) {
    const long long s = slot(e);
    if (s < 0) continue;
    a.pos_out[s] = a.pos_in[s];
    a.w_out[s] = a.w_in[s];
  }
  __syncthreads();
  for (int i = tid; i < total; i += EV_THREADS) {
    const int2 m = move[i];
    const long long s = slot(m.x), d = slot(m.y);
    if (s < 0 || d < 0) continue;
    a.pos_out[d] = a.pos_in[s];
    a.w_out[d] = a.w_in[s];
  }
  pdl_trigger();
}

// 16-byte units of the moved entries' segments (layer, K or V, head).
__global__ void __launch_bounds__(256) k_evict_move(EvictDev a, uint4* pool, int segs, int units) {
  pdl_wait();
  const int b = blockIdx.y, n = a.moves[b];
  const int* table = a.page_table + (size_t)b * a.max_pages;
  const long long per = (long long)segs * units, total = per * n, page_units = per * SV_PAGE;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (long long)gridDim.x * blockDim.x) {
    const int m = (int)(i / per), r = (int)(i - m * per), seg = r / units, u = r - seg * units;
    const int2 mv = a.move[(size_t)b * a.budget + m];
    const int ps = table[mv.x / SV_PAGE], pd = table[mv.y / SV_PAGE];
    if (ps < 0 || ps >= a.n_pages || pd < 0 || pd >= a.n_pages) continue;
    const long long in_seg = (long long)seg * SV_PAGE;
    pool[pd * page_units + (in_seg + mv.y % SV_PAGE) * units + u] = pool[ps * page_units + (in_seg + mv.x % SV_PAGE) * units + u];
  }
}

size_t evict_scratch(const tlf_evict_args& a) {
  return ((size_t)a.n * 4 + 15) / 16 * 16 + (size_t)a.n * a.budget * sizeof(int2);
}

cudaError_t launch_evict(const tlf_evict_args& a, void* scratch, int num_sms, cudaStream_t st) {
  EvictDev d{a.n, a.max_pages, a.budget, a.n_first, a.n_recent, a.n_pages, a.page_table, a.lens, a.next_pos, a.pos_in,
             a.pos_out, a.weight_in, a.weight_out, a.lens_out, a.err, static_cast<int*>(scratch),
             reinterpret_cast<int2*>(static_cast<char*>(scratch) + ((size_t)a.n * 4 + 15) / 16 * 16)};
  const int cached = (int)std::min<long long>(EV_CACHED, (long long)a.max_pages * SV_PAGE);
  const int smem = 4 * (cached + cached / 32 + 1);
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_evict_select), smem)) return e;
  if (cudaError_t e = launch_k(k_evict_select, dim3(a.n), dim3(EV_THREADS), smem, st, d, cached)) return e;
  const int segs = a.n_layers * 2 * a.n_kv_heads, units = a.head_dim * (a.dtype == TLF_DTYPE_BF16 ? 2 : 4) / 16;
  return launch_k(k_evict_move, dim3(std::max(1, num_sms * 8 / a.n), a.n), dim3(256), 0, st, d,
                  static_cast<uint4*>(a.pool), segs, units);
}

}  // namespace tlf
