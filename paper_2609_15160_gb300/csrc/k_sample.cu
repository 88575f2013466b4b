// Sampling from logits with given random numbers (tlf_sample).
//
// With z_i = (l_i - max) / T and w_i = exp(z_i), the kept tokens are a first part of the order by (l, lower index) whatever
// the limits: top-k, top-p and min-p each keep a first part of that order. So a token is kept when its ordered key is above
// a threshold key, or equal to it and early enough among the equal ones. Among the kept, argmax of z_i - log(-log u_i) draws i
// with probability w_i / sum of the kept w: only kept tokens need their random number, and no sum decides between two of them.
//
// Passes over the row (all but the first find it in L2): the maximum; the sum of w, with a histogram of the tokens over bins
// of z of width 1/16; the candidates. Candidates are the bins that top-k or top-p can reach: by count for top-k, and for top-p
// by the least that the bins' tokens can weigh. They are few for the usual limits and go to a list in shared memory, where a
// radix select over the keys finds the threshold: by count for top-k, by weight for top-p. Weights are then added in 2^-40
// fixed point, so the order of the atomics does not matter. When top-p alone leaves too many candidates (flat logits), the
// bins' weights are added up in a pass of their own, which leaves the one bin with the threshold for the list; what lies above
// it takes part in the draw at once. Where that is too much for the list too, the select goes over the whole row.
#include "k_serve.cuh"

namespace tlf {

constexpr int SM_THREADS = 1024;
constexpr int SM_LIST = 4096;

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

// f(logit, index) over the row, all threads taking part in every step; index -1: nothing.
template <typename F>
__device__ __forceinline__ void sample_pass(const float* row, int V, bool wide, F&& f) {
  if (wide) {
    for (int i0 = 0; i0 < V; i0 += 4 * SM_THREADS) {
      const int i = i0 + 4 * threadIdx.x;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i + 3 < V) v = *reinterpret_cast<const float4*>(row + i);
      else if (i < V) v = make_float4(row[i], i + 1 < V ? row[i + 1] : 0.f, i + 2 < V ? row[i + 2] : 0.f, 0.f);
      f(sample_logit(v.x), i < V ? i : -1);
      f(sample_logit(v.y), i + 1 < V ? i + 1 : -1);
      f(sample_logit(v.z), i + 2 < V ? i + 2 : -1);
      f(sample_logit(v.w), i + 3 < V ? i + 3 : -1);
    }
  } else {
    for (int i0 = 0; i0 < V; i0 += SM_THREADS) {
      const int i = i0 + threadIdx.x;
      f(i < V ? sample_logit(row[i]) : -INFINITY, i < V ? i : -1);
    }
  }
}

__global__ void __launch_bounds__(SM_THREADS) k_sample(SampleDev a) {
  pdl_wait();
  __shared__ uint32_t s_key[SM_LIST];
  __shared__ int s_idx[SM_LIST];
  __shared__ unsigned s_bin[SM_BINS];
  __shared__ u64 s_mass[SM_BINS];  // of a bin, or of a digit of the select
  __shared__ unsigned s_cnt[256];
  __shared__ float s_redf[33];
  __shared__ int s_redi[33];
  __shared__ u64 s_redl[33];
  __shared__ int s_n, s_pick;
  __shared__ uint32_t s_lo, s_hi, s_prefix;
  __shared__ unsigned s_need, s_hit;
  __shared__ u64 s_above;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.V;
  const float* row = a.logits + b * a.ls;
  const float* noise = a.noise + b * a.ns;
  const bool wide = reinterpret_cast<uintptr_t>(row) % 16 == 0;

  float mx = -INFINITY;
  sample_pass(row, V, wide, [&](float l, int i) { mx = fmaxf(mx, i >= 0 ? l : -INFINITY); });
  mx = warp_max(mx);
  if (lane == 0) s_redf[warp] = mx;
  if (tid < SM_BINS) s_bin[tid] = 0;
  if (tid == 0) s_n = 0;
  __syncthreads();
  mx = warp_max(s_redf[lane]);
  if (mx == -INFINITY) {  // nothing can be drawn
    if (tid == 0) {
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
  // z as the definition has it, for what decides; times 1 / T for sums and bins
  auto z_of = [&](float l) { return (l - mx) / T; };
  auto zq_of = [&](float l) { return l > -INFINITY ? fmaxf((l - mx) * rT, -INFINITY) : -INFINITY; };
  auto mass_of = [&](uint32_t key) { return sample_mass(expf(z_of(sample_unkey(key)))); };

  float sum = 0.f;
  if (by_k || by_p) {
    sample_pass(row, V, wide, [&](float l, int i) {
      const float z = i >= 0 ? zq_of(l) : -INFINITY;
      sum += ex2_fast(z * 1.4426950408889634f);
      const int bin = sample_bin(z);
      if (bin < SM_BINS - 1) atomicAdd(&s_bin[bin], 1u);
    });
  } else {
    sample_pass(row, V, wide, [&](float l, int i) { sum += i >= 0 ? ex2_fast(zq_of(l) * 1.4426950408889634f) : 0.f; });
  }
  sum = block_sum(sum, s_redf);

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
  auto first_bin = [&](auto value, auto reached) {
    if (tid == 0) s_pick = SM_BINS - 1;
    auto v = value(tid);  // one bin a thread; threads past the bins add nothing
    decltype(v) before = block_scan(v, reinterpret_cast<decltype(v)*>(s_redl), (decltype(v)*)nullptr);
    if (tid < SM_BINS - 1 && !reached(before) && reached(before + v)) s_pick = tid;
    __syncthreads();
    return s_pick;
  };
  // all tokens of bins first .. last into the list; tokens of bins before `first` take part in the draw
  auto gather = [&](int first, int last) {
    sample_pass(row, V, wide, [&](float l, int i) {
      const int bin = i >= 0 && l > -INFINITY ? sample_bin(zq_of(l)) : SM_BINS;
      if (bin < first) race(l, i);
      const bool in = bin >= first && bin <= last;
      const unsigned who = __ballot_sync(0xffffffffu, in);
      if (who) {
        int at = 0;
        if (lane == 0) at = atomicAdd(&s_n, __popc(who));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1u));
        if (in && at < SM_LIST) {
          s_key[at] = sample_key(l);
          s_idx[at] = i;
        }
      }
    });
    __syncthreads();
  };

  bool list = false;      // candidates are the list's (else the row's)
  u64 heavier = 0;        // weight of tokens heavier than the list's, which have taken part in the draw already
  if (by_k) {
    const int bin = first_bin([&](int i) { return i < SM_BINS - 1 ? s_bin[i] : 0u; }, [&](unsigned n) { return n >= (unsigned)k; });
    if (bin < SM_BINS - 1) {
      gather(0, bin);
      list = s_n <= SM_LIST;
    }
  } else if (by_p) {
    // a token of bin i weighs at least exp(-(i + 1/2) / 16) (and a little: z is rounded)
    const float want = (float)top_p * sum * 1.0001f;
    const int bin = first_bin([&](int i) { return i < SM_BINS - 1 ? s_bin[i] * ex2_fast(-(i + 0.51f) * (1.4426950408889634f / SM_BIN)) : 0.f; },
                              [&](float m) { return m >= want; });
    if (bin < SM_BINS - 1) {
      const int n = block_sum(tid <= bin ? (int)s_bin[tid] : 0, s_redi);
      if (n <= SM_LIST) {
        gather(0, bin);
        list = true;
      } else {
        if (tid < SM_BINS) s_mass[tid] = 0;
        __syncthreads();
        unsigned* mass32 = reinterpret_cast<unsigned*>(s_mass);
        sample_pass(row, V, wide, [&](float l, int i) {
          const int at = i >= 0 && l > -INFINITY ? sample_bin(zq_of(l)) : SM_BINS;
          if (at > bin) return;
          const u64 m = mass_of(sample_key(l));
          const unsigned lo = (unsigned)m, old = atomicAdd(&mass32[2 * at], lo), hi = (unsigned)(m >> 32) + (old + lo < old);
          if (hi) atomicAdd(&mass32[2 * at + 1], hi);
        });
        __syncthreads();
        const double target = top_p * (double)sample_mass(1.f) * (double)sum;
        const int at = first_bin([&](int i) { return i <= bin ? s_mass[i] : 0ull; }, [&](u64 m) { return (double)m >= target; });
        if (at <= bin && s_bin[at] <= SM_LIST) {
          heavier = block_sum(tid < at ? s_mass[tid] : 0ull, s_redl);
          gather(at, at);
          list = true;
        }
      }
    }
  }
  const int n = list ? s_n : V;
  auto key_at = [&](int i) { return list ? s_key[i] : sample_key(sample_logit(row[i])); };

  // Kept: keys above thr, and the first `ties` of the `equal` tokens with key thr.
  uint32_t thr = SAMPLE_NEVER;
  unsigned ties = 0, equal = 0;
  // Radix select over the candidates' keys above `from`, eight bits of (key - smallest) a level, from the largest digit on: the
  // key at which count or weight reaches what is wanted. By weight, `from` itself stands for `from_ties` tokens. False: not
  // reached, all of them are kept.
  auto walk = [&](bool weigh, unsigned want, double target, uint32_t from, unsigned from_ties) {
    if (tid == 0) {
      s_lo = 0xffffffffu;
      s_hi = 0;
      s_prefix = 0;
      s_need = want;
      s_hit = 0;
      s_above = weigh ? heavier : 0;
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
      atomicMin(&s_lo, lo);
      atomicMax(&s_hi, hi);
    }
    __syncthreads();
    lo = s_lo;
    hi = s_hi;
    if (lo > hi) return false;
    int up = 32 - __clz(hi - lo);  // bits that are not settled yet
    do {
      const int down = up > 8 ? up - 8 : 0, bits = up - down;
      if (tid < 256) {
        s_cnt[tid] = 0;
        s_mass[tid] = 0;
      }
      __syncthreads();
      const uint32_t prefix = s_prefix;
      const unsigned need = s_need;
      const u64 above0 = s_above;
      for (int i = tid; i < n; i += SM_THREADS) {
        const uint32_t key = key_at(i);
        if (key <= from || (u64)(key - lo) >> up != prefix) continue;
        const unsigned digit = (key - lo) >> down & ((1u << bits) - 1u);
        atomicAdd(&s_cnt[digit], 1u);
        if (weigh) atomicAdd(&s_mass[digit], mass_of(key));
      }
      if (weigh && tid == 0 && from_ties && (u64)(from - lo) >> up == prefix) {
        const unsigned digit = (from - lo) >> down & ((1u << bits) - 1u);
        atomicAdd(&s_cnt[digit], from_ties);
        atomicAdd(&s_mass[digit], from_ties * mass_of(from));
      }
      __syncthreads();
      if (warp == 0) {  // a lane has eight digits, from the largest
        unsigned c[8], cs = 0;
        u64 m[8], ms = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          cs += c[i] = s_cnt[255 - 8 * lane - i];
          ms += m[i] = s_mass[255 - 8 * lane - i];
        }
        unsigned cb = cs;
        u64 mb = ms;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned cy = __shfl_up_sync(0xffffffffu, cb, o);
          const u64 my = __shfl_up_sync(0xffffffffu, mb, o);
          if (lane >= o) cb += cy, mb += my;
        }
        cb -= cs;
        u64 at = above0 + (mb - ms);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool hit = weigh ? (double)at < target && (double)(at + m[i]) >= target : cb < need && cb + c[i] >= need;
          if (hit) {
            s_prefix = (prefix << bits) | (unsigned)(255 - 8 * lane - i);
            s_need = need - cb;
            s_above = at;
            s_hit = c[i];
          }
          cb += c[i];
          at += m[i];
        }
      }
      __syncthreads();
      if (!s_hit) return false;
      up = down;
    } while (up > 0);
    if (tid == 0) s_prefix += lo;
    __syncthreads();
    return true;
  };
  if (by_k && walk(false, (unsigned)k, 0.0, SAMPLE_NEVER, 0)) {
    thr = s_prefix;
    ties = s_need;
    equal = s_hit;
  }
  __syncthreads();
  if (by_p) {
    double target = top_p * (double)sample_mass(1.f) * (double)sum;
    if (by_k) {
      u64 kept = 0;
      for (int i = tid; i < n; i += SM_THREADS) {
        const uint32_t key = key_at(i);
        if (key > thr) kept += mass_of(key);
      }
      kept = block_sum(kept, s_redl) + ties * mass_of(thr);
      target = top_p * (double)kept;
    }
    const uint32_t from = thr;
    const unsigned from_ties = ties, from_equal = equal;
    if (walk(true, 0, target, from, from_ties)) {
      thr = s_prefix;
      const double w = (double)mass_of(thr), left = target - (double)s_above;
      ties = (unsigned)fmin((double)s_hit, fmax(1.0, ceil(left / w)));
      equal = thr == from ? from_equal : s_hit;
    }
    __syncthreads();
  }
  // the last index among the equal that stay
  int last = V;
  if (ties < equal) {
    const int run = (V + SM_THREADS - 1) / SM_THREADS, i0 = min(V, tid * run), i1 = min(V, i0 + run);
    int c = 0;
    for (int i = i0; i < i1; ++i) c += sample_key(sample_logit(row[i])) == thr;
    int before = block_scan(c, s_redi, (int*)nullptr);
    if (before < (int)ties && before + c >= (int)ties)
      for (int i = i0; i < i1; ++i)
        if (sample_key(sample_logit(row[i])) == thr && ++before == (int)ties) s_n = i;
    __syncthreads();
    last = s_n;
  }

  if (list) {
    for (int i = tid; i < n; i += SM_THREADS) {
      const uint32_t key = s_key[i];
      if (key > thr || (key == thr && s_idx[i] <= last)) race(sample_unkey(key), s_idx[i]);
    }
  } else {
    sample_pass(row, V, wide, [&](float l, int i) {
      const uint32_t key = sample_key(l);
      if (i >= 0 && key > SAMPLE_NEVER && (key > thr || (key == thr && i <= last))) race(l, i);
    });
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float ob = __shfl_xor_sync(0xffffffffu, best, o);
    const int ot = __shfl_xor_sync(0xffffffffu, token, o);
    if (ob > best || (ob == best && ot < token)) best = ob, token = ot;
  }
  if (lane == 0) {
    s_redf[warp] = best;
    s_redi[warp] = token;
  }
  __syncthreads();
  if (warp == 0) {
    best = s_redf[lane];
    token = s_redi[lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float ob = __shfl_xor_sync(0xffffffffu, best, o);
      const int ot = __shfl_xor_sync(0xffffffffu, token, o);
      if (ob > best || (ob == best && ot < token)) best = ob, token = ot;
    }
    if (lane == 0) {
      a.tokens[b] = token;
      if (a.logprobs) a.logprobs[b] = z_of(sample_logit(row[token])) - logf(sum);
    }
  }
  pdl_trigger();
}

cudaError_t launch_sample(const tlf_sample_args& a, int num_sms, cudaStream_t st) {
  (void)num_sms;
  SampleDev d{a.vocab, a.logits, a.logits_stride, a.noise, a.noise_stride, a.temperature, a.top_k, a.top_p, a.min_p,
              a.tokens, a.logprobs};
  return launch_k(k_sample, dim3(a.n), dim3(SM_THREADS), 0, st, d);
}

}  // namespace tlf
