// Sampling from logits with given random numbers (tlf_sample).
//
// With z_i = (l_i - max) / T and w_i = exp(z_i), the kept tokens are a first part of the order by (l, lower index) whatever
// the limits: top-k, top-p and min-p each keep a first part of that order. So a token is kept when its ordered key is above
// a threshold key, or equal to it and early enough among the equal ones. Among the kept, argmax of z_i - log(-log u_i) draws i
// with probability w_i / sum of the kept w: only kept tokens need their random number, and no sum decides between two of them.
//
// Passes over the row (all but the first find it in L2): the maximum; the sum of w; the candidates. Candidates are tokens that
// top-k or top-p can reach; they are few for the usual limits and go to a list in shared memory, where the threshold is found.
//   top-k   tokens from the k-th largest of the threads' own maxima on (to the next 1/32 in z): at least k of them;
//   top-p   a histogram over bins of z of width 1/32 (taken in the pass of the sum) bounds the weight up to every bin from
//           both sides: bins that surely stay, bins that surely do not, and a few between them, where the threshold lies and
//           which alone take part in finding it. The ones that stay go to a list of their own, or, where they are too many,
//           take part in the draw at once.
// A short list is sorted by counting. A longer one takes a radix select over the keys: by count for top-k, by weight for top-p,
// with weights in 2^-40 fixed point, so the order of the atomics does not matter. Where the candidates are too many for the
// list (logits that are nearly all alike), the select goes over the whole row. A row is split over a cluster of up to eight
// CTAs while there are SMs left over. In the draw a token's -log(-log u) is first bounded by -log(1 - u), and only the few that
// could beat the warp's best so far are computed.
//
// Bound by instructions and by the latency of the passes; the bytes' floor is the logits once (256 x 50304: 7.6 us). 256 rows of
// 50304: 17 us greedy, 20 with top-k 50, 42 with top-p 0.95 (nucleus of 1600), 40 with no limit (the random numbers of all
// tokens), 50 with all of these mixed, where the rows with the largest nuclei decide: the median row is done after half of it.
#include <type_traits>

#include <cooperative_groups.h>

#include "k_serve.cuh"

namespace cg = cooperative_groups;

namespace tlf {

constexpr int SM_THREADS = 512;
constexpr int SM_LIST = 4096;   // candidates among which the threshold lies
constexpr int SM_SURE = 12288;  // tokens that stay for sure
constexpr int SM_SORT = 512;   // longest list that is sorted by counting
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

constexpr int SM_BINS = 1024;   // two a thread
constexpr float SM_BIN = 32.f;  // bins per unit of z; the last bin holds the rest
// Bin of a token with z2 = z log2 e, rounded to nearest: bin i holds z in -(i + 1/2) / 32 .. -(i - 1/2) / 32.
__device__ __forceinline__ int sample_bin(float z2) {
  return (int)(__float_as_uint(fminf(z2 * (-SM_BIN * 0.6931471805599453f), (float)(SM_BINS - 1)) + 8388608.f) & 0x7ffu);
}

// f(16 logits, index of the first): the logits are four times four in a row, SM_STEP apart. Entries v0 .. v1 - 1 of the row (v0 a
// multiple of 4), all threads taking part in every step; NaN (a token that cannot be drawn) past the end.
constexpr int SM_STEP = 4 * SM_THREADS;
template <typename F>
__device__ __forceinline__ void sample_pass(const float* row, int v0, int v1, bool wide, F&& f) {
  const float none = __int_as_float(0x7fffffff);
  int i = v0 + 4 * (int)threadIdx.x, left = v1 - v0;
  float e[16];
  if (wide)
    for (; left >= 4 * SM_STEP; left -= 4 * SM_STEP, i += 4 * SM_STEP) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(row + i + u * SM_STEP));
        e[4 * u] = v.x, e[4 * u + 1] = v.y, e[4 * u + 2] = v.z, e[4 * u + 3] = v.w;
      }
      f(e, i);
    }
  for (; left > 0; left -= 4 * SM_STEP, i += 4 * SM_STEP) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = i + u * SM_STEP;
      if (wide && at + 3 < v1) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(row + at));
        e[4 * u] = v.x, e[4 * u + 1] = v.y, e[4 * u + 2] = v.z, e[4 * u + 3] = v.w;
      } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) e[4 * u + x] = at + x < v1 ? row[at + x] : none;
      }
    }
    f(e, i);
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
  int sure[SM_SURE];
  u64 mass[SM_SORT];      // of a digit of the select; of the list, sorted
  alignas(8) unsigned bin[SM_BINS];  // tokens of this CTA's part, or threads' maxima
  unsigned cnt[256];
  uint32_t skey[SM_SORT];
  int sidx[SM_SORT];
  float redf[33];
  int redi[33];
  u64 redl[33];
  float mx, sum, best[SM_CLUSTER];  // what this CTA found in its part; of all parts (at rank 0)
  int token[SM_CLUSTER];
  float heavy[SM_CLUSTER];
  int n, n_sure, pick;
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
  sample_pass(row, v0, v1, wide, [&](const float (&e)[16], int) {
#pragma unroll
    for (int x = 0; x < 16; ++x) m4[x & 3] = fmaxf(m4[x & 3], e[x]);
  });
  const float mine = fminf(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), FMAX);  // this thread's largest
  float mx = warp_max(mine);
  if (lane == 0) S.redf[warp] = mx;
  for (int i = tid; i < SM_BINS; i += SM_THREADS) S.bin[i] = 0;
  if (tid == 0) S.n = S.n_sure = 0;
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
  // z as the definition has it, for what decides; z log2 e by a factor for sums and bins (NaN, or 0 x infinity: far below)
  auto z_of = [&](float l) { return (l - mx) / T; };
  const float r2 = rT * 1.4426950408889634f;
  auto z2_of = [&](float raw) { return fminf(fmaxf((raw - mx) * r2, -1000.f), 0.f); };
  auto mass_of = [&](uint32_t key) { return sample_mass(expf(z_of(sample_unkey(key)))); };
  // a logit that no token of z >= zc is below, whatever the roundings
  auto cut_at = [&](float zc) { return fmaxf(mx + zc * T * 1.00001f - 1e-6f * fabsf(mx), -FMAX); };

  if (by_max && mine > -INFINITY) {
    const int bin = sample_bin(z2_of(mine));
    if (bin < SM_BINS - 1) atomicAdd(&S.bin[bin], 1u);
  }
  float sum = 0.f;
  if (a.logprobs || by_p || (by_k && !by_max)) {
    float s4[4] = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](const float (&e)[16], auto bins) {
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float z2 = z2_of(e[x]);
        s4[x & 3] += ex2_fast(z2);
        if (bins) {
          const int bin = sample_bin(z2);
          if (bin < SM_BINS - 1) atomicAdd(&S.bin[bin], 1u);
        }
      }
    };
    if (!by_max && (by_k || by_p)) sample_pass(row, v0, v1, wide, [&](const float (&e)[16], int) { add(e, std::true_type{}); });
    else sample_pass(row, v0, v1, wide, [&](const float (&e)[16], int) { add(e, std::false_type{}); });
    sum = block_sum((s4[0] + s4[1]) + (s4[2] + s4[3]), S.redf);
  }
  if (cs > 1) {
    if (tid == 0) S.sum = sum;
    cl.sync();
    sum = 0.f;
    for (int r = 0; r < cs; ++r) sum += *cl.map_shared_rank(&S.sum, r);
  }
  // tokens of this thread's two bins in the whole row
  static_assert(SM_BINS == 2 * SM_THREADS && SM_SORT <= SM_THREADS, "two bins a thread");
  const int bin0 = 2 * tid, bin1 = bin0 + 1;
  uint2 tot = make_uint2(0u, 0u);
  if (by_k || by_p) {
    if (cs == 1) __syncthreads();
    for (int r = 0; r < cs; ++r) {
      const uint2 n = *reinterpret_cast<const uint2*>((cs > 1 ? cl.map_shared_rank(S.bin, r) : S.bin) + bin0);
      tot.x += n.x;
      tot.y += n.y;
    }
  }
  const unsigned tot0 = tot.x, tot1 = bin1 < SM_BINS - 1 ? tot.y : 0u;
  __syncthreads();

  // the draw: largest z - log(-log u), ties to the lower index
  float best = -INFINITY;
  int token = V;
  auto race = [&](float l, float u, int idx) {
    const float z = z_of(l);
    if (min_p > 0.f && l != mx && !(expf(z) >= min_p)) return;
    float score = z - logf(-logf(u));
    if (!(score == score)) score = -INFINITY;
    if (score > best || (score == best && idx < token)) {
      best = score;
      token = idx;
    }
  };
  // a token that -log u >= 1 - u lets beat `lim` (what is not a number may)
  float lim = -INFINITY;  // best of the warp
  auto may_win = [&](float raw, float u) { return !((raw - mx) * rT - 0.6931471805599453f * __log2f(1.f - u) + 1e-3f < lim); };
  const bool wide_u = reinterpret_cast<uintptr_t>(noise) % 16 == 0;
  // all tokens from `cut` on take part; returns their weight
  auto race_pass = [&](float cut, auto weigh) {
    float mass = 0.f;
    sample_pass(row, v0, v1, wide, [&](const float (&e)[16], int i) {
      float u[16];
#pragma unroll
      for (int x = 0; x < 16; x += 4) {
        const int at = i + (x / 4) * SM_STEP;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (cut <= -FMAX ? at < V : fmaxf(fmaxf(e[x], e[x + 1]), fmaxf(e[x + 2], e[x + 3])) >= cut) {
          if (wide_u && at + 3 < V) v = __ldg(reinterpret_cast<const float4*>(noise + at));
          else v = make_float4(noise[at], at + 1 < V ? noise[at + 1] : 0.f, at + 2 < V ? noise[at + 2] : 0.f, at + 3 < V ? noise[at + 3] : 0.f);
        }
        u[x] = v.x, u[x + 1] = v.y, u[x + 2] = v.z, u[x + 3] = v.w;
      }
      unsigned may = 0;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        if (e[x] >= cut && may_win(e[x], u[x])) may |= 1u << x;
        if (weigh && e[x] >= cut) mass += ex2_fast(z2_of(e[x]));
      }
      if (__any_sync(0xffffffffu, may != 0)) {
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (may >> x & 1) race(sample_logit(e[x]), u[x], i + (x / 4) * SM_STEP + x % 4);
        lim = warp_max(best);
      }
    });
    return mass;
  };
  // tokens of bins first .. last
  auto tokens_in = [&](int first, int last) {
    return block_sum((bin0 >= first && bin0 <= last ? (int)tot0 : 0) + (bin1 >= first && bin1 <= last ? (int)tot1 : 0), S.redi);
  };
  int* n_at = cs > 1 ? cl.map_shared_rank(&S.n, 0) : &S.n;
  int* sure_at = cs > 1 ? cl.map_shared_rank(&S.n_sure, 0) : &S.n_sure;
  uint32_t* key_to = cs > 1 ? cl.map_shared_rank(S.key, 0) : S.key;
  int* idx_to = cs > 1 ? cl.map_shared_rank(S.idx, 0) : S.idx;
  int* sure_to = cs > 1 ? cl.map_shared_rank(S.sure, 0) : S.sure;
  // tokens from `cut` on into the list; those from `top` on (NaN: none) into the one of the sure, or nowhere
  auto gather = [&](float cut, float top, bool keep) {
    sample_pass(row, v0, v1, wide, [&](const float (&e)[16], int i) {
      unsigned in = 0, high = 0;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        if (e[x] >= cut) in |= 1u << x;
        if (e[x] >= top) high |= 1u << x;
      }
      if (!keep) in &= ~high, high = 0;
      if (!__any_sync(0xffffffffu, in != 0)) return;
      const int mine = __popc(in ^ high) | __popc(high) << 16;
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      int front = 0, back = 0;
      if (lane == 31) {
        if (upto & 0xffff) front = atomicAdd(n_at, upto & 0xffff);
        if (upto >> 16) back = atomicAdd(sure_at, upto >> 16);
      }
      front = __shfl_sync(0xffffffffu, front, 31) + ((upto - mine) & 0xffff);
      back = __shfl_sync(0xffffffffu, back, 31) + ((upto - mine) >> 16);
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        if (!(in >> x & 1)) continue;
        const int idx = i + (x >> 2) * SM_STEP + (x & 3);
        if (high >> x & 1) {
          if (back < SM_SURE) sure_to[back] = idx;
          ++back;
        } else {
          if (front < SM_LIST) {
            key_to[front] = sample_key(sample_logit(e[x]));
            idx_to[front] = idx;
          }
          ++front;
        }
      }
    });
  };

  const float none_f = __int_as_float(0x7fffffff);
  bool list = false;  // candidates are the list's (else the row's)
  float heavy = 0.f;  // weight of the tokens that stay for sure
  const double all_mass = (double)sample_mass(1.f) * (double)sum;
  if (by_k) {
    // the first bin at which the count reaches k
    if (tid == 0) S.pick = SM_BINS - 1;
    const unsigned before = block_scan(tot0 + tot1, reinterpret_cast<unsigned*>(S.redi), (unsigned*)nullptr);
    if (before < (unsigned)k && before + tot0 + tot1 >= (unsigned)k) S.pick = before + tot0 >= (unsigned)k ? bin0 : bin1;
    __syncthreads();
    const int bin = S.pick;
    if (bin < SM_BINS - 1 && (by_max || tokens_in(0, bin) <= SM_LIST)) {
      gather(cut_at(-(bin + 0.51f) / SM_BIN), none_f, false);
      list = true;
    }
  } else if (by_p) {
    // a token of bin i weighs between exp(-(i + 1/2) / 32) and exp(-(i - 1/2) / 32) (and a little: z is rounded), all of the
    // last bin together next to nothing
    auto weight = [&](unsigned n, int bin, float off) { return n * ex2_fast(-(bin + off) * (1.4426950408889634f / SM_BIN)); };
    const float least0 = weight(tot0, bin0, 0.52f), least1 = weight(tot1, bin1, 0.52f);
    const float most0 = weight(tot0, bin0, -0.52f), most1 = weight(tot1, bin1, -0.52f);
    float all_least, all_most;
    const float lower0 = block_scan(least0 + least1, S.redf, &all_least) + least0, lower1 = lower0 + least1;
    const float upper0 = block_scan(most0 + most1, S.redf, &all_most) + most0, upper1 = upper0 + most1;
    const float goal = (float)top_p * sum, rest = (float)(1.0 - top_p) * sum, slip = 1e-5f * sum;
    // bins up to `sure` stay whole; bins from `none` on do not
    auto stays = [&](float lower, float upper) { return upper < goal - slip || all_least - lower > rest + slip; };
    auto open = [&](float lower, float upper) { return !(lower > goal + slip || all_most - upper < rest - slip); };
    const int sure = block_sum((int)stays(lower0, upper0) + (int)(bin1 < SM_BINS - 1 && stays(lower1, upper1)), S.redi) - 1;
    const int none = block_sum((int)open(lower0, upper0) + (int)(bin1 < SM_BINS - 1 && open(lower1, upper1)), S.redi) + 1;
    const int n_sure = tokens_in(0, sure), n_between = tokens_in(sure + 1, none - 1);
    if (none < SM_BINS && n_between <= SM_LIST - SM_LIST / 32) {
      // from `top` on a token is in a sure bin; the rest of those counts as between
      const float cut = cut_at(-(none - 0.49f) / SM_BIN);
      const float top = sure < 0 ? none_f : mx - (sure + 0.49f) / SM_BIN * T * 0.99999f + 1e-6f * fabsf(mx);
      if (n_sure <= SM_SURE) {
        gather(cut, top, true);
      } else {
        heavy = block_sum(race_pass(top, std::true_type{}), S.redf);
        gather(cut, top, false);
      }
      list = true;
    }
  } else {  // no limit but min-p
    race_pass(min_p > 0.f ? cut_at(logf(min_p) - 1e-3f) : -FMAX, std::false_type{});
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
      cl.map_shared_rank(S.heavy, 0)[rank] = heavy;
    }
    cl.sync();
    if (rank != 0) {
      pdl_trigger();
      return;
    }
    best = tid < cs ? S.best[tid] : -INFINITY;
    token = tid < cs ? S.token[tid] : V;
    heavy = 0.f;
    for (int r = 0; r < cs; ++r) heavy += S.heavy[r];
  }
  __syncthreads();
  if (list && S.n > SM_LIST) list = false;  // more tokens at the bound than the bins let expect
  const int n = list ? S.n : V;
  u64 heavier = list ? (u64)(heavy * 1099511627776.f) : 0;
  // list entries that take part: noise of four in flight
  auto race_list = [&](int first, int count, auto stays) {
    for (int i0 = 0; i0 < count; i0 += 4 * SM_THREADS) {
      float u[4];
      bool on[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int i = i0 + x * SM_THREADS + tid;
        on[x] = i < count && stays(S.key[first + i], S.idx[first + i]);
        u[x] = on[x] ? noise[S.idx[first + i]] : 0.f;
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int i = i0 + x * SM_THREADS + tid;
        if (on[x] && may_win(sample_unkey(S.key[first + i]), u[x])) race(sample_unkey(S.key[first + i]), u[x], S.idx[first + i]);
        lim = fmaxf(lim, best);
      }
    }
  };
  if (list && S.n_sure) {  // the tokens that stay for sure
    u64 mass = 0;
    for (int i0 = tid; i0 < S.n_sure; i0 += 4 * SM_THREADS) {
      float l[4], u[4];
      int idx[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int i = i0 + x * SM_THREADS;
        idx[x] = i < S.n_sure ? S.sure[i] : -1;
        l[x] = idx[x] >= 0 ? row[idx[x]] : -INFINITY;
        u[x] = idx[x] >= 0 ? noise[idx[x]] : 0.f;
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (idx[x] < 0) continue;
        mass += sample_mass(ex2_fast(z2_of(l[x])));
        if (may_win(l[x], u[x])) race(sample_logit(l[x]), u[x], idx[x]);
        lim = fmaxf(lim, best);
      }
    }
    heavier += block_sum(mass, S.redl);
  }

  if (list && n <= SM_SORT) {
    // sorted by (key, lower index): a token's place is the number of tokens before it
    if (tid < n) {
      S.mass[tid] = (u64)S.key[tid] << 32 | (uint32_t)~S.idx[tid];
    }
    __syncthreads();
    if (tid < n) {
      const u64 key = S.mass[tid];
      int place = 0;
#pragma unroll 4
      for (int i = 0; i < n; ++i) place += S.mass[i] > key;
      S.skey[place] = S.key[tid];
      S.sidx[place] = S.idx[tid];
    }
    __syncthreads();
    const bool in = tid < n && tid < k;
    const uint32_t key = in ? S.skey[tid] : 0u;
    bool stays = in;
    if (by_p) {
      const u64 m = in ? mass_of(key) : 0;
      u64 total;
      const u64 before = block_scan(m, S.redl, &total);
      stays = in && ((tid == 0 && !heavier) || (double)(heavier + before) < top_p * (by_k ? (double)total : all_mass));
    }
    if (stays) race(sample_unkey(key), noise[S.sidx[tid]], S.sidx[tid]);
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
        ties = (unsigned)fmin((double)S.hit, fmax(heavier ? 0.0 : 1.0, ceil(left / w)));
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
    if (list) {
      race_list(0, n, [&](uint32_t key, int idx) { return key > thr || (key == thr && idx <= last); });
    } else {
      for (int i = tid; i < V; i += SM_THREADS) {
        const uint32_t key = key_at(i);
        if (key > SAMPLE_NEVER && (key > thr || (key == thr && i <= last))) race(sample_unkey(key), noise[i], i);
      }
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
  // rows are split over clusters while there is an SM for every CTA and a part is not too short for its share of the steps that
  // every part has (on 1 / 2 / 4 / 8 CTAs a row, top-p 0.95: one row of 32000 tokens 18.8 / 17.6 / 15.5 / 15.6 us, one of 128000
  // 48.6 / 35.4 / 27.0 / 23.1, 64 of 50304 30.8 / 27.2 / 27.9 / 45.3, 120 of 50304 31.3 / 34.6 / 48.4 / 72.2)
  int cs = 1;
  while (cs < SM_CLUSTER && (long long)a.n * cs * 2 <= num_sms && a.vocab >= 16000 * cs) cs *= 2;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_sample), sizeof(SampleShared))) return e;
  return launch_cluster(k_sample, dim3(a.n * cs), dim3(SM_THREADS), cs, sizeof(SampleShared), st, d, cs);
}

}  // namespace tlf
