// Sampling from logits with given random numbers (tlf_sample).
//
// With z_i = (l_i - max) / T and w_i = exp(z_i), the kept tokens are a first part of the order by (l, lower index) whatever
// the limits: top-k, top-p and min-p each keep a first part of that order. So a token is kept when its ordered key is above
// a threshold key, or equal to it and early enough among the equal ones. Among the kept, argmax of z_i - log(-log u_i) draws i
// with probability w_i / sum of the kept w: only kept tokens need their random number, and no sum decides between two of them.
//
// Three passes over the row (the second and third find it in L2): maximum; sum of w; candidates. Candidates are a superset of
// the kept tokens that is small for the usual limits: with top-k <= 1024 the tokens not below the k-th largest of the
// threads' maxima, with top-p those that weigh at least (1 - top_p) sum / V (all lighter ones together weigh less than
// 1 - top_p of the sum), with min-p those not below it. The threshold is then a radix select over the candidates' keys: by
// count for top-k, by weight for top-p. Weights are added in 2^-40 fixed point, so the order of the atomics does not matter.
// Where the candidates are too many for the list (flat logits), the same steps run over the whole row.
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

__global__ void __launch_bounds__(SM_THREADS) k_sample(SampleDev a) {
  pdl_wait();
  __shared__ uint32_t s_key[SM_LIST];
  __shared__ int s_idx[SM_LIST];
  __shared__ u64 s_mass[256];
  __shared__ unsigned s_cnt[256];
  __shared__ float s_redf[33];
  __shared__ int s_redi[33];
  __shared__ u64 s_redl[33];
  __shared__ int s_n;
  __shared__ uint32_t s_prefix;
  __shared__ unsigned s_need, s_hit;
  __shared__ u64 s_above;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.V;
  const float* row = a.logits + b * a.ls;

  float mx = -INFINITY;
  for (int i = tid; i < V; i += SM_THREADS) mx = fmaxf(mx, sample_logit(row[i]));
  const float mine = mx;  // this thread's largest
  mx = warp_max(mx);
  if (lane == 0) s_redf[warp] = mx;
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
  const float T = temp > 0.f ? temp : 1.f;
  int k = a.top_k ? a.top_k[b] : 0;
  k = k <= 0 || k > V ? V : k;
  if (!(temp > 0.f) || top_p <= 0.0 || !(min_p <= 1.f)) {  // only the first token
    k = 1;
    min_p = 0.f;
  }
  auto z_of = [&](float l) { return (l - mx) / T; };
  auto w_of = [&](float l) { return l > -INFINITY ? expf(z_of(l)) : 0.f; };

  float sum = 0.f;
  u64 mass = 0;  // of all tokens; needed by top-p without top-k
  for (int i = tid; i < V; i += SM_THREADS) {
    const float w = w_of(sample_logit(row[i]));
    sum += w;
    mass += sample_mass(w);
  }
  sum = block_sum(sum, s_redf);
  mass = block_sum(mass, s_redl);

  // candidates: keys from `cand` on, z from `zc` on
  const bool by_k = k < V, by_p = top_p < 1.0;
  uint32_t cand = SAMPLE_NEVER + 1;
  float zc = -INFINITY;
  bool limited = false;
  if (by_k && k <= SM_THREADS) {
    // k-th largest of the threads' maxima, bit by bit: the largest x with at least k of them at or above it
    const uint32_t own = sample_key(mine);
    uint32_t x = 0;
    for (int bit = 31; bit >= 0; --bit)
      if (__syncthreads_count(own >= (x | 1u << bit)) >= k) x |= 1u << bit;
    cand = max(cand, x);  // fewer than k threads with a token that can be drawn: all tokens
    limited = true;
  } else if (!by_k) {
    // what the lighter tokens weigh together, each rounded up, stays below the part that top-p leaves out
    const double light = by_p ? (1.0 - top_p) * (double)mass / V - 1.0 : 0.0;
    if (light > 0.0) zc = logf((float)(light / 1099511627776.0)) - 1e-3f;
    if (min_p > 0.f) zc = fmaxf(zc, logf(min_p) - 1e-3f);
    limited = zc > -INFINITY;
  }
  bool list = limited;
  if (limited) {
    for (int i0 = 0; i0 < V; i0 += SM_THREADS) {
      const int i = i0 + tid;
      const float l = i < V ? sample_logit(row[i]) : -INFINITY;
      const uint32_t key = sample_key(l);
      const bool is = key >= cand && (zc == -INFINITY || z_of(l) >= zc);
      const unsigned in = __ballot_sync(0xffffffffu, is);
      if (in) {
        int at = 0;
        if (lane == 0) at = atomicAdd(&s_n, __popc(in));
        at = __shfl_sync(0xffffffffu, at, 0) + __popc(in & ((1u << lane) - 1u));
        if (is && at < SM_LIST) {
          s_key[at] = key;
          s_idx[at] = i;
        }
      }
    }
    __syncthreads();
    list = s_n <= SM_LIST;
  }
  const int n = list ? s_n : V;
  auto key_at = [&](int i) { return list ? s_key[i] : sample_key(sample_logit(row[i])); };
  auto mass_of = [&](uint32_t key) { return sample_mass(w_of(sample_unkey(key))); };

  // Kept: keys above thr, and the first `ties` of the `equal` tokens with key thr.
  uint32_t thr = SAMPLE_NEVER;
  unsigned ties = 0, equal = 0;
  // Radix select over keys above `from` (a byte a level, from the largest bin on): the bin in which count or weight reaches
  // what is wanted. By weight, `from` itself stands for `from_ties` tokens. False: not reached, all of them are kept.
  auto walk = [&](bool weigh, unsigned want, double target, uint32_t from, unsigned from_ties) {
    if (tid == 0) {
      s_prefix = 0;
      s_need = want;
      s_hit = 0;
      s_above = 0;
    }
    for (int shift = 24; shift >= 0; shift -= 8) {
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
        if (key <= from || (shift < 24 && (key >> (shift + 8)) != prefix)) continue;
        const unsigned bin = (key >> shift) & 255u;
        atomicAdd(&s_cnt[bin], 1u);
        if (weigh) atomicAdd(&s_mass[bin], mass_of(key));
      }
      if (weigh && tid == 0 && from_ties && (shift == 24 || (from >> (shift + 8)) == prefix)) {
        atomicAdd(&s_cnt[(from >> shift) & 255u], from_ties);
        atomicAdd(&s_mass[(from >> shift) & 255u], from_ties * mass_of(from));
      }
      __syncthreads();
      if (warp == 0) {  // a lane has eight bins, from the largest
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
        mb -= ms;
        u64 above = above0 + mb;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool hit = weigh ? (double)above < target && (double)(above + m[i]) >= target : cb < need && cb + c[i] >= need;
          if (hit) {
            s_prefix = (prefix << 8) | (unsigned)(255 - 8 * lane - i);
            s_need = need - cb;
            s_above = above;
            s_hit = c[i];
          }
          cb += c[i];
          above += m[i];
        }
      }
      __syncthreads();
      if (!s_hit) break;
    }
    return s_hit != 0;
  };
  if (by_k && walk(false, (unsigned)k, 0.0, SAMPLE_NEVER, 0)) {
    thr = s_prefix;
    ties = s_need;
    equal = s_hit;
  }
  __syncthreads();
  if (by_p && k > 1) {
    u64 kept = mass;
    if (by_k) {
      kept = 0;
      for (int i = tid; i < n; i += SM_THREADS) {
        const uint32_t key = key_at(i);
        if (key > thr) kept += mass_of(key);
      }
      kept = block_sum(kept, s_redl) + ties * mass_of(thr);
    }
    const double target = top_p * (double)kept;
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

  // the draw: largest z - log(-log u), ties to the lower index
  float best = -INFINITY;
  int token = V;
  const float* noise = a.noise + b * a.ns;
  for (int i = tid; i < n; i += SM_THREADS) {
    const uint32_t key = key_at(i);
    const int idx = list ? s_idx[i] : i;
    if (key <= SAMPLE_NEVER || key < thr || (key == thr && idx > last)) continue;
    const float z = z_of(sample_unkey(key));
    if (min_p > 0.f && key != sample_key(mx) && !(expf(z) >= min_p)) continue;
    const float u = noise[idx];
    float score = z - logf(-logf(u));
    if (!(score == score)) score = -INFINITY;
    if (score > best || (score == best && idx < token)) {
      best = score;
      token = idx;
    }
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
