// Sampling from logits with given random numbers (tlf_sample).
//
// With z_i = (l_i - max) / T and w_i = exp(z_i), the kept tokens are a first part of the order by (l, lower index) whatever
// the limits: top-k, top-p and min-p each keep a first part of that order. So a token is kept when its ordered key is above
// a threshold key, or equal to it and early enough among the equal ones. Among the kept, argmax of z_i - log(-log u_i) draws i
// with probability w_i / sum of the kept w: only kept tokens need their random number, and no sum decides between two of them.
//
// Passes over the row (all but the first find it in L2): the maximum; the sum of w; the candidates. Candidates are tokens that
// top-k or top-p can reach; they are few for the usual limits and go to a list in shared memory, where the threshold is found.
//   top-k   tokens from the k-th largest of the threads' own maxima on (to the next 1/16 in z): at least k of them;
//   top-p   tokens from the bin of z on (width 1/16) behind which the rest weighs at most 1 - top_p of the sum at the most;
//           that takes a histogram of the tokens, in the pass of the sum.
// A short list is sorted by counting. A longer one takes a radix select over the keys: by count for top-k, by weight for top-p,
// with weights in 2^-40 fixed point, so the order of the atomics does not matter. When top-p alone leaves too many candidates
// (flat logits), the bins' weights are added up in a pass of their own, which leaves the one bin with the threshold for the
// list; what lies above it takes part in the draw at once. Where that is too much for the list too, the select goes over the
// whole row. A row is split over a cluster of up to eight CTAs while there are SMs left over.
#include <cooperative_groups.h>

#include "k_serve.cuh"

namespace cg = cooperative_groups;

namespace tlf {

constexpr int SM_THREADS = 512;
constexpr int SM_LIST = 6144;
constexpr int SM_SORT = 256;   // longest list that is sorted by counting
constexpr int SM_CLUSTER = 8;  // most CTAs that share a row

struct SampleDev {
  int V;
  const float* logits;
  long long ls;
  const float* noise;
  long long ns;
  const float* temperature;
  const int* top_k;
  const float* top_p;
  const float* min_p;
  int* tokens;
  float* logprobs;
};

typedef unsigned long long u64;

// A token's logit as the operator sees it: NaN and -inf cannot be drawn (-inf), +inf is the largest float.
__device__ __forceinline__ float sample_logit(float l) { return l > -INFINITY ? fminf(l, 3.402823466e38f) : -INFINITY; }
// Ordered key of a logit (-inf: 0x007fffff, the smallest); equal logits, 0 and -0 among them, have equal keys.
constexpr uint32_t SAMPLE_NEVER = 0x007fffffu;
__device__ __forceinline__ uint32_t sample_key(float l) {
  const uint32_t u = __float_as_uint(l + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float sample_unkey(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ u64 sample_mass(float w) { return __float2ull_rn(w * 1099511627776.f); }  // w in 0..1

constexpr int SM_BINS = 512;
constexpr float SM_BIN = 16.f;  // bins per unit of z; the last bin holds the rest
// Bin of a token, rounded to nearest: bin i holds z in -(i + 1/2) / 16 .. -(i - 1/2) / 16.
__device__ __forceinline__ int sample_bin(float z) {
  return (int)(__float_as_uint(fminf(z * -SM_BIN, (float)(SM_BINS - 1)) + 8388608.f) & 0x3ffu);
}

// f(four logits, index of the first) over entries v0 .. v1 - 1 of the row (v0 a multiple of 4), all threads taking part in
// every step; NaN (a token that cannot be drawn) past the end. U loads of a thread are in flight before the first is used.
template <typename F>
__device__ __forceinline__ void sample_pass(const float* row, int v0, int v1, bool wide, F&& f) {
  constexpr int U = 8;
  const float none = __int_as_float(0x7fffffff);
  for (int i0 = v0; i0 < v1; i0 += 4 * U * SM_THREADS) {
    float4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + 4 * (u * SM_THREADS + (int)threadIdx.x);
      if (wide && i + 3 < v1) v[u] = __ldg(reinterpret_cast<const float4*>(row + i));
      else v[u] = make_float4(i < v1 ? row[i] : none, i + 1 < v1 ? row[i + 1] : none, i + 2 < v1 ? row[i + 2] : none, i + 3 < v1 ? row[i + 3] : none);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + 4 * u * SM_THREADS < v1) f(v[u], i0 + 4 * (u * SM_THREADS + (int)threadIdx.x));
  }
}

// A 64-bit sum in shared memory in two words (there is no 64-bit add to shared memory without a loop).
__device__ __forceinline__ void add_mass(u64* at, u64 m) {
  unsigned* w = reinterpret_cast<unsigned*>(at);
  const unsigned lo = (unsigned)m, old = atomicAdd(w, lo), hi = (unsigned)(m >> 32) + (old + lo < old);
  if (hi) atomicAdd(w + 1, hi);
}

struct SampleShared {
  uint32_t key[SM_LIST];
  int idx[SM_LIST];
  u64 mass[SM_BINS];      // of a bin, or of a digit of the select
  unsigned bin[SM_BINS];  // tokens of this CTA's part, or threads' maxima
  unsigned tot[SM_BINS];  // bin of the whole row
  unsigned cnt[256];
  uint32_t skey[SM_SORT];
  int sidx[SM_SORT];
  float redf[33];
  int redi[33];
  u64 redl[33];
  float mx, sum, best[SM_CLUSTER];  // what this CTA found in its part; of all parts (at rank 0)
  int token[SM_CLUSTER];
  int n, pick;
  uint32_t lo, hi, prefix;
  unsigned need, hit;
  u64 above;
};

__global__ void __launch_bounds__(SM_THREADS, 2) k_sample(SampleDev a, int cs) {
  pdl_wait();
  extern __shared__ uint8_t smem_raw[];
  SampleShared& S = *reinterpret_cast<SampleShared*>(smem_raw);
  const cg::cluster_group cl = cg::this_cluster();
  const int b = blockIdx.x / cs, rank = blockIdx.x % cs, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.V;
  const int each = (V + 4 * cs - 1) / (4 * cs) * 4, v0 = min(V, rank * each), v1 = min(V, v0 + each);
  const float* row = a.logits + b * a.ls;
  const float* noise = a.noise + b * a.ns;
  const bool wide = reinterpret_cast<uintptr_t>(row) % 16 == 0;
  constexpr float FMAX = 3.402823466e38f;

  float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  sample_pass(row, v0, v1, wide, [&](float4 v, int) {
    m4[0] = fmaxf(m4[0], v.x);
    m4[1] = fmaxf(m4[1], v.y);
    m4[2] = fmaxf(m4[2], v.z);
    m4[3] = fmaxf(m4[3], v.w);
  });
  const float mine = fminf(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), FMAX);  // this thread's largest
  float mx = warp_max(mine);
  if (lane == 0) S.redf[warp] = mx;
  for (int i = tid; i < SM_BINS; i += SM_THREADS) S.bin[i] = 0;
  if (tid == 0) S.n = 0;
  __syncthreads();
  mx = warp_max(S.redf[lane & (SM_THREADS / 32 - 1)]);
  if (cs > 1) {
    if (tid == 0) S.mx = mx;
    cl.sync();
    for (int r = 0; r < cs; ++r) mx = fmaxf(mx, *cl.map_shared_rank(&S.mx, r));
  }
  if (mx == -INFINITY) {  // nothing can be drawn
    if (cs > 1) cl.sync();
    if (tid == 0 && rank == 0) {
      a.tokens[b] = -1;
      if (a.logprobs) a.logprobs[b] = -INFINITY;
    }
    pdl_trigger();
    return;
  }
  const float temp = a.temperature ? a.temperature[b] : 1.f;
  float min_p = a.min_p ? a.min_p[b] : 0.f;
  const double top_p = a.top_p && a.top_p[b] < 1.f ? (double)a.top_p[b] : 1.0;
  const float T = temp > 0.f ? fmaxf(temp, 1.2e-38f) : 1.f, rT = 1.f / T;
  int k = a.top_k ? a.top_k[b] : 0;
  k = k <= 0 || k > V ? V : k;
  if (!(temp > 0.f) || top_p <= 0.0 || !(min_p <= 1.f)) {  // only the first token
    k = 1;
    min_p = 0.f;
  }
  const bool by_k = k < V, by_p = top_p < 1.0 && k > 1;
  const bool by_max = by_k && k <= SM_THREADS * cs;  // the threads' maxima bound the top-k
  // z as the definition has it, for what decides; times 1 / T for sums and bins (NaN, or 0 x infinity: far below)
  auto z_of = [&](float l) { return (l - mx) / T; };
  auto zq_of = [&](float raw) { return fminf(fmaxf((raw - mx) * rT, -1000.f), 0.f); };
  auto mass_of = [&](uint32_t key) { return sample_mass(expf(z_of(sample_unkey(key)))); };
  // a logit that is not above any token of z >= zc, whatever the roundings
  auto cut_at = [&](float zc) { return fmaxf(mx + zc * T * 1.00001f - 1e-6f * fabsf(mx), -FMAX); };

  if (by_max && mine > -INFINITY) {
    const int bin = sample_bin(zq_of(mine));
    if (bin < SM_BINS - 1) atomicAdd(&S.bin[bin], 1u);
  }
  float sum = 0.f;
  if (a.logprobs || by_p || (by_k && !by_max)) {
    float s4[4] = {0.f, 0.f, 0.f, 0.f};
    const bool bins = !by_max && (by_k || by_p);
    sample_pass(row, v0, v1, wide, [&](float4 v, int) {
      const float z[4] = {zq_of(v.x), zq_of(v.y), zq_of(v.z), zq_of(v.w)};
#pragma unroll
      for (int e = 0; e < 4; ++e) s4[e] += ex2_fast(z[e] * 1.4426950408889634f);
      if (bins) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int bin = sample_bin(z[e]);
          if (bin < SM_BINS - 1) atomicAdd(&S.bin[bin], 1u);
        }
      }
    });
    sum = block_sum((s4[0] + s4[1]) + (s4[2] + s4[3]), S.redf);
  }
  if (cs > 1) {
    if (tid == 0) S.sum = sum;
    cl.sync();
    sum = 0.f;
    for (int r = 0; r < cs; ++r) sum += *cl.map_shared_rank(&S.sum, r);
    for (int i = tid; i < SM_BINS; i += SM_THREADS) {
      unsigned n = 0;
      for (int r = 0; r < cs; ++r) n += cl.map_shared_rank(S.bin, r)[i];
      S.tot[i] = n;
    }
  } else {
    __syncthreads();
    for (int i = tid; i < SM_BINS; i += SM_THREADS) S.tot[i] = S.bin[i];
  }
  __syncthreads();

  // the draw: largest z - log(-log u), ties to the lower index
  float best = -INFINITY;
  int token = V;
  auto race = [&](float l, int idx) {
    const float z = z_of(l);
    if (min_p > 0.f && l != mx && !(expf(z) >= min_p)) return;
    float score = z - logf(-logf(noise[idx]));
    if (!(score == score)) score = -INFINITY;
    if (score > best || (score == best && idx < token)) {
      best = score;
      token = idx;
    }
  };
  // the first bin (from the heaviest tokens on) at which `reached` holds for the values up to it; SM_BINS - 1 if none
  static_assert(SM_BINS == SM_THREADS, "a bin a thread");
  auto first_bin = [&](auto v, auto reached) {
    if (tid == 0) S.pick = SM_BINS - 1;
    decltype(v) before = block_scan(v, reinterpret_cast<decltype(v)*>(S.redl), (decltype(v)*)nullptr);
    if (tid < SM_BINS - 1 && !reached(before) && reached(before + v)) S.pick = tid;
    __syncthreads();
    return S.pick;
  };
  // tokens for which `in` holds into the list, which is rank 0's
  int* n_at = cs > 1 ? cl.map_shared_rank(&S.n, 0) : &S.n;
  uint32_t* key_to = cs > 1 ? cl.map_shared_rank(S.key, 0) : S.key;
  int* idx_to = cs > 1 ? cl.map_shared_rank(S.idx, 0) : S.idx;
  auto put = [&](float raw, int i, bool in) {
    const unsigned who = __ballot_sync(0xffffffffu, in);
    if (!who) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(n_at, __popc(who));
    at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1u));
    if (in && at < SM_LIST) {
      key_to[at] = sample_key(sample_logit(raw));
      idx_to[at] = i;
    }
  };
  auto gather = [&](float cut) {
    sample_pass(row, v0, v1, wide, [&](float4 v, int i) {
      const float e[4] = {v.x, v.y, v.z, v.w};
      if (__any_sync(0xffffffffu, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)) >= cut)) {
#pragma unroll
        for (int x = 0; x < 4; ++x) put(e[x], i + x, e[x] >= cut);
      }
    });
  };

  bool list = false;  // candidates are the list's (else the row's)
  u64 heavier = 0;    // weight of tokens heavier than the list's, which have taken part in the draw already
  const double all_mass = (double)sample_mass(1.f) * (double)sum;
  if (by_k) {
    const int bin = first_bin(tid < SM_BINS - 1 ? S.tot[tid] : 0u, [&](unsigned n) { return n >= (unsigned)k; });
    if (bin < SM_BINS - 1 && (by_max || block_sum(tid <= bin ? (int)S.tot[tid] : 0, S.redi) <= SM_LIST)) {
      gather(cut_at(-(bin + 0.51f) / SM_BIN));
      list = true;
    }
  } else if (by_p) {
    // a token of bin i weighs at most exp(-(i - 1/2) / 16), and all of the last bin together next to nothing
    const float most = S.tot[tid] * ex2_fast(-(tid - 0.51f) * (1.4426950408889634f / SM_BIN));
    const float rest = (float)(1.0 - top_p) * sum * 0.999f, all = block_sum(most, S.redf);
    const int bin = first_bin(most, [&](float m) { return all - m <= rest - 1e-6f * all; });
    if (bin < SM_BINS - 1) {
      if (block_sum(tid <= bin ? (int)S.tot[tid] : 0, S.redi) <= SM_LIST - SM_LIST / 32) {
        gather(cut_at(-(bin + 0.51f) / SM_BIN));
        list = true;
      } else {
        S.mass[tid] = 0;
        __syncthreads();
        sample_pass(row, v0, v1, wide, [&](float4 v, int) {
          const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int at = sample_bin(zq_of(e[x]));
            if (at <= bin) add_mass(&S.mass[at], mass_of(sample_key(sample_logit(e[x]))));
          }
        });
        __syncthreads();
        if (cs > 1) {
          cl.sync();
          u64 m = 0;
          for (int r = 0; r < cs; ++r) m += cl.map_shared_rank(S.mass, r)[tid];
          cl.sync();
          S.mass[tid] = m;
          __syncthreads();
        }
        const u64 target = (u64)ceil(top_p * all_mass);
        const int at = first_bin(tid <= bin ? S.mass[tid] : 0ull, [&](u64 m) { return m >= target; });
        if (at <= bin && S.tot[at] <= SM_LIST) {
          heavier = block_sum(tid < at ? S.mass[tid] : 0ull, S.redl);
          sample_pass(row, v0, v1, wide, [&](float4 v, int i) {
            const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int bin_x = sample_bin(zq_of(e[x]));
              if (bin_x < at) race(sample_logit(e[x]), i + x);
              put(e[x], i + x, bin_x == at);
            }
          });
          list = true;
        }
      }
    }
  } else {  // no limit but min-p
    const float cut = min_p > 0.f ? cut_at(logf(min_p) - 1e-3f) : -FMAX;
    sample_pass(row, v0, v1, wide, [&](float4 v, int i) {
      if (v.x >= cut) race(sample_logit(v.x), i);
      if (v.y >= cut) race(sample_logit(v.y), i + 1);
      if (v.z >= cut) race(sample_logit(v.z), i + 2);
      if (v.w >= cut) race(sample_logit(v.w), i + 3);
    });
  }
  auto race_warp = [&] {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float ob = __shfl_xor_sync(0xffffffffu, best, o);
      const int ot = __shfl_xor_sync(0xffffffffu, token, o);
      if (ob > best || (ob == best && ot < token)) best = ob, token = ot;
    }
  };
  auto race_block = [&] {  // warp 0 has the block's best
    race_warp();
    __syncthreads();
    if (lane == 0) {
      S.redf[warp] = best;
      S.redi[warp] = token;
    }
    __syncthreads();
    if (warp == 0) {
      best = S.redf[lane & (SM_THREADS / 32 - 1)];
      token = S.redi[lane & (SM_THREADS / 32 - 1)];
      race_warp();
    }
  };
  if (cs > 1) {  // what is left is rank 0's: the list, and the others' draws
    race_block();
    if (tid == 0) {
      cl.map_shared_rank(S.best, 0)[rank] = best;
      cl.map_shared_rank(S.token, 0)[rank] = token;
    }
    cl.sync();
    if (rank != 0) {
      pdl_trigger();
      return;
    }
    best = tid < cs ? S.best[tid] : -INFINITY;
    token = tid < cs ? S.token[tid] : V;
  }
  __syncthreads();
  if (list && S.n > SM_LIST) list = false;  // (the cut lets tokens below the bin in, by a rounding)
  const int n = list ? S.n : V;
  if (!list && heavier) {  // taken back: the whole row draws again
    heavier = 0;
    best = -INFINITY;
    token = V;
  }

  if (list && !heavier && n <= SM_SORT) {
    // sorted by (key, lower index): a token's place is the number of tokens before it
    if (tid < n) {
      const uint32_t key = S.key[tid];
      const int idx = S.idx[tid];
      int place = 0;
      for (int i = 0; i < n; ++i) place += S.key[i] > key || (S.key[i] == key && S.idx[i] < idx);
      S.skey[place] = key;
      S.sidx[place] = idx;
    }
    __syncthreads();
    const bool in = tid < n && tid < k;
    const uint32_t key = in ? S.skey[tid] : 0u;
    bool stays = in;
    if (by_p) {
      const u64 m = in ? mass_of(key) : 0;
      u64 total;
      const u64 before = block_scan(m, S.redl, &total);
      stays = in && (tid == 0 || (double)before < top_p * (by_k ? (double)total : all_mass));
    }
    if (stays) race(sample_unkey(key), S.sidx[tid]);
  } else if (by_k || by_p) {
    auto key_at = [&](int i) { return list ? S.key[i] : sample_key(sample_logit(row[i])); };
    // Kept: keys above thr, and the first `ties` of the `equal` tokens with key thr.
    uint32_t thr = SAMPLE_NEVER;
    unsigned ties = 0, equal = 0;
    // Radix select over the candidates' keys above `from`, eight bits of (key - smallest) a level, from the largest digit on: the
    // key at which count or weight reaches what is wanted. By weight, `from` itself stands for `from_ties` tokens. False: not
    // reached, all of them are kept.
    auto walk = [&](bool weigh, unsigned want, u64 target, uint32_t from, unsigned from_ties) {
      if (tid == 0) {
        S.lo = 0xffffffffu;
        S.hi = 0;
        S.prefix = 0;
        S.need = want;
        S.hit = 0;
        S.above = weigh ? heavier : 0;
      }
      __syncthreads();
      uint32_t lo = 0xffffffffu, hi = 0;
      for (int i = tid; i < n; i += SM_THREADS) {
        const uint32_t key = key_at(i);
        if (key <= from && !(from_ties && key == from)) continue;
        lo = min(lo, key);
        hi = max(hi, key);
      }
      lo = __reduce_min_sync(0xffffffffu, lo);
      hi = __reduce_max_sync(0xffffffffu, hi);
      if (lane == 0) {
        atomicMin(&S.lo, lo);
        atomicMax(&S.hi, hi);
      }
      __syncthreads();
      lo = S.lo;
      hi = S.hi;
      if (lo > hi) return false;
      int up = 32 - __clz(hi - lo);  // bits that are not settled yet
      do {
        const int down = up > 8 ? up - 8 : 0, bits = up - down;
        if (tid < 256) {
          S.cnt[tid] = 0;
          S.mass[tid] = 0;
        }
        __syncthreads();
        const uint32_t prefix = S.prefix;
        const unsigned need = S.need;
        const u64 above0 = S.above;
        for (int i = tid; i < n; i += SM_THREADS) {
          const uint32_t key = key_at(i);
          if (key <= from || (u64)(key - lo) >> up != prefix) continue;
          const unsigned digit = (key - lo) >> down & ((1u << bits) - 1u);
          atomicAdd(&S.cnt[digit], 1u);
          if (weigh) add_mass(&S.mass[digit], mass_of(key));
        }
        if (weigh && tid == 0 && from_ties && (u64)(from - lo) >> up == prefix) {
          const unsigned digit = (from - lo) >> down & ((1u << bits) - 1u);
          atomicAdd(&S.cnt[digit], from_ties);
          add_mass(&S.mass[digit], from_ties * mass_of(from));
        }
        __syncthreads();
        if (warp == 0) {  // a lane has eight digits, from the largest
          unsigned c[8], cs8 = 0;
          u64 m[8], ms = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            cs8 += c[i] = S.cnt[255 - 8 * lane - i];
            ms += m[i] = S.mass[255 - 8 * lane - i];
          }
          unsigned cb = cs8;
          u64 mb = ms;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const unsigned cy = __shfl_up_sync(0xffffffffu, cb, o);
            const u64 my = __shfl_up_sync(0xffffffffu, mb, o);
            if (lane >= o) cb += cy, mb += my;
          }
          cb -= cs8;
          u64 at = above0 + (mb - ms);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const bool hit = weigh ? at < target && at + m[i] >= target : cb < need && cb + c[i] >= need;
            if (hit) {
              S.prefix = (prefix << bits) | (unsigned)(255 - 8 * lane - i);
              S.need = need - cb;
              S.above = at;
              S.hit = c[i];
            }
            cb += c[i];
            at += m[i];
          }
        }
        __syncthreads();
        if (!S.hit) return false;
        up = down;
      } while (up > 0);
      if (tid == 0) S.prefix += lo;
      __syncthreads();
      return true;
    };
    if (by_k && walk(false, (unsigned)k, 0, SAMPLE_NEVER, 0)) {
      thr = S.prefix;
      ties = S.need;
      equal = S.hit;
    }
    __syncthreads();
    if (by_p) {
      double target = top_p * all_mass;
      if (by_k) {
        u64 kept = 0;
        for (int i = tid; i < n; i += SM_THREADS) {
          const uint32_t key = key_at(i);
          if (key > thr) kept += mass_of(key);
        }
        kept = block_sum(kept, S.redl) + ties * mass_of(thr);
        target = top_p * (double)kept;
      }
      const uint32_t from = thr;
      const unsigned from_ties = ties, from_equal = equal;
      if (walk(true, 0, (u64)ceil(target), from, from_ties)) {
        thr = S.prefix;
        const double w = (double)mass_of(thr), left = target - (double)S.above;
        ties = (unsigned)fmin((double)S.hit, fmax(1.0, ceil(left / w)));
        equal = thr == from ? from_equal : S.hit;
      }
      __syncthreads();
    }
    // the last index among the equal that stay
    int last = V;
    if (ties < equal) {
      const int run = (V + SM_THREADS - 1) / SM_THREADS, i0 = min(V, tid * run), i1 = min(V, i0 + run);
      int c = 0;
      for (int i = i0; i < i1; ++i) c += sample_key(sample_logit(row[i])) == thr;
      int before = block_scan(c, S.redi, (int*)nullptr);
      if (before < (int)ties && before + c >= (int)ties)
        for (int i = i0; i < i1; ++i)
          if (sample_key(sample_logit(row[i])) == thr && ++before == (int)ties) S.pick = i;
      __syncthreads();
      last = S.pick;
    }
    for (int i = tid; i < n; i += SM_THREADS) {
      const uint32_t key = key_at(i);
      const int idx = list ? S.idx[i] : i;
      if (key > SAMPLE_NEVER && (key > thr || (key == thr && idx <= last))) race(sample_unkey(key), idx);
    }
  }
  race_block();
  if (tid == 0) {
    a.tokens[b] = token;
    if (a.logprobs) a.logprobs[b] = z_of(sample_logit(row[token])) - logf(sum);
  }
  pdl_trigger();
}

cudaError_t launch_sample(const tlf_sample_args& a, int num_sms, cudaStream_t st) {
  SampleDev d{a.vocab, a.logits, a.logits_stride, a.noise, a.noise_stride, a.temperature, a.top_k, a.top_p, a.min_p,
              a.tokens, a.logprobs};
  // rows are split over clusters while that leaves every CTA an SM's half: one row of 32000 takes ... us on one CTA, ... on eight
  int cs = 1;
  while (cs < SM_CLUSTER && (long long)a.n * cs * 2 <= 2 * num_sms && a.vocab > 2048 * cs) cs *= 2;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_sample), sizeof(SampleShared))) return e;
  return launch_cluster(k_sample, dim3(a.n * cs), dim3(SM_THREADS), cs, sizeof(SampleShared), st, d, cs);
}

}  // namespace tlf
