// Rotary positions of new tokens and their append to a paged cache (tlf_rope_append), and rotary tables (tlf_rope_table).
//
// Pair (x_a, x_b) of a head at position p becomes (x_a c - x_b s, x_b c + x_a s), (c, s) = table[p][pair]: what is
// turned at position p and what is turned at p' then meet in q . k as a function of p - p'. The table is read, not computed:
// a float32 angle p f_k loses log2(p f_k) bits of the turn, and a row of it is shared by every head of the token.
//
// Bound by HBM for many tokens (7157 tokens, 16 / 8 heads x 128, 64 dims turned, interleaved: 24.3 us, 4.9 TB/s; 40 us before
// the table's rows went through shared memory and copied units stayed raw, 146 instructions a 16-byte unit), by the look-ups'
// dependent loads for few (64 tokens, 16 heads x 64: 3.2 us in a CUDA graph).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "k_serve.cuh"

namespace tlf {

struct RopeFreq {
  double f[128];  // of pair k
};

// One thread per (position, pair). The angle and its sine are taken in 64 bits: positions times frequencies reach 10^6 turns.
__global__ void k_rope_scaled_table(RopeFreq fr, int pairs, int max_pos, double magnitude, float2* table) {
  pdl_wait();
  const long long n = (long long)max_pos * pairs;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
    double s, c;
    sincos((double)(i / pairs) * fr.f[i % pairs], &s, &c);
    table[i] = make_float2((float)(c * magnitude), (float)(s * magnitude));
  }
  pdl_trigger();
}

cudaError_t launch_rope_scaled_table(const tlf_rope_config& cfg, int max_pos, float* table, cudaStream_t st) {
  RopeFreq fr{};
  const int pairs = cfg.rot_dim / 2;
  const double base =
      cfg.scaling == TLF_ROPE_NTK ? cfg.base * std::pow(cfg.factor, (double)cfg.rot_dim / (cfg.rot_dim - 2)) : cfg.base;
  for (int k = 0; k < pairs; ++k) {
    double f = std::pow(base, -2.0 * k / cfg.rot_dim);
    if (cfg.scaling == TLF_ROPE_LINEAR) f /= cfg.factor;
    if (cfg.scaling == TLF_ROPE_RAMP) {
      const double turns = cfg.original_len * f / (2.0 * 3.14159265358979323846);
      const double r = std::fmin(1.0, std::fmax(0.0, (turns - cfg.low_turns) / (cfg.high_turns - cfg.low_turns)));
      f = f * (1.0 - r) / cfg.factor + f * r;
    }
    fr.f[k] = f;
  }
  const long long n = (long long)max_pos * pairs;
  return launch_k(k_rope_scaled_table, dim3((unsigned)std::fmin(4096.0, std::ceil(n / 256.0))), dim3(256), 0, st, fr, pairs,
                  max_pos, cfg.magnitude, reinterpret_cast<float2*>(table));
}

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_TOKENS = 4;  // most tokens of a group

struct RopeDev {
  const void *q, *k, *v;
  long long qs, ks, vs;
  const int* positions;
  const float2* table;
  int max_pos, rot, interleaved, tokens, ctas;  // tokens: of a group
  void* q_out;
  int* entry_pos;
  float* entry_weight;
};

template <typename T>
__device__ __forceinline__ void store16(T* p, const float* x);
template <>
__device__ __forceinline__ void store16<float>(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
template <>
__device__ __forceinline__ void store16<bf16>(bf16* p, const float* x) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// VEC elements as they come from memory.
template <typename T, int VEC> struct RopeRaw {
  uint4 v;
  __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = v; }
  __device__ __forceinline__ void get(float* x) const { Vec16<T>::load(reinterpret_cast<const T*>(&v), x); }
};
template <typename T> struct RopeRaw<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ void store(T* p) const { *p = v; }
  __device__ __forceinline__ void get(float* x) const { x[0] = to_f32(v); }
};

// A CTA goes over groups of `tokens` (up to four) tokens. A ninth warp looks a group's rows, entries and positions up (a token's
// row is the number of rows that end at or before it; four dependent loads) and puts the positions' rows of the table into
// shared memory, where every head finds them, while the eight others still work on the group before, or wait for the first group's data. A thread of theirs keeps its unit, VEC elements (16 bytes) of a head or the two
// groups of VEC that a rotation in halves pairs up, and has it of all the group's tokens in flight; units that leave threads
// over get several threads, each with a share of the tokens. VEC = 1 takes what is not aligned to 16 bytes. TWO: a turned unit has
// two groups (halves, or single elements); copied units never leave their raw form.
template <typename T, typename QT, int VEC, bool TWO>
__global__ void __launch_bounds__(ROPE_THREADS + 32, 3) k_rope_chunk(ChunkDev c, RopeDev a) {
  pdl_wait();
  __shared__ long long s_dst[2][ROPE_TOKENS];  // element offset of the token's K in head 0 of its page, -1: no entry
  __shared__ int s_pos[2][ROPE_TOKENS];        // -1: out of range
  __shared__ __align__(16) float2 s_cs[2][ROPE_TOKENS][64];
  const int tid = threadIdx.x, lane = tid & 31;
  const int groups = (c.T + a.tokens - 1) / a.tokens;
  if (tid >= ROPE_THREADS) {
    constexpr int L = 32 / ROPE_TOKENS;  // lanes of a token
    for (int g = blockIdx.x, buf = 0; g < groups; g += gridDim.x, buf ^= 1) {
      const int j = lane / L, t = g * a.tokens + j;
      const bool on = j < a.tokens && t < c.T;
      int pos = on ? a.positions[t] : 0, b = 0;
      if (pos < 0 || pos >= a.max_pos) {
        if (lane % L == 0) sv_report(c.err, DEVERR_INDEX);
        pos = -1;
      }
      if (on)
        for (int i = lane % L; i < a.rot / 2; i += L) s_cs[buf][j][i] = a.table[(long long)max(pos, 0) * (a.rot / 2) + i];
      if (on)
        for (int i = lane % L; i < c.n; i += L) b += c.cu[i + 1] <= t;
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) b += __shfl_xor_sync(0xffffffffu, b, o);
      if (on && lane % L == 0) {
        long long dst = -1;
        const ChunkRow r = b < c.n ? chunk_row(c, b) : ChunkRow{0, 0, 0};
        const int i = t - r.t0, e = r.len - r.ql + i;
        if (pos >= 0 && i >= 0 && i < r.ql && e >= 0) {
          const int page = chunk_page(c.page_table, c.max_pages, c.n_pages, b, e / SV_PAGE, c.err);
          if (page >= 0) {
            const int off = e % SV_PAGE;
            dst = (long long)page * c.page_elems + ((long long)c.layer * 2 * c.Hkv * SV_PAGE + off) * c.hd;
            if (a.entry_pos) a.entry_pos[(long long)page * SV_PAGE + off] = pos;
            if (a.entry_weight) a.entry_weight[(long long)page * SV_PAGE + off] = 0.f;
          }
        } else {
          sv_report(c.err, DEVERR_INDEX);
        }
        s_pos[buf][j] = pos;
        s_dst[buf][j] = dst;
      }
      __syncthreads();
    }
    pdl_trigger();
    return;
  }

  const unsigned hd = c.hd, rot = a.rot;
  const unsigned ru = a.interleaved ? (VEC == 1 ? rot / 2 : rot / VEC) : rot / 2 / VEC;  // units of the turned dims
  const unsigned hu = ru + (hd - rot) / VEC;                                            // of a q or k head
  const unsigned vu = hd / VEC, qk = (unsigned)(c.Hq + c.Hkv) * hu, per = qk + c.Hkv * vu;
  const long long seg = (long long)SV_PAGE * hd;  // of a head in a page
  const unsigned shares = per >= ROPE_THREADS ? 1 : min(ROPE_THREADS / per, (unsigned)ROPE_TOKENS);
  const unsigned share = shares == 1 ? 0 : tid / per, w0 = tid - share * per, step_w = shares == 1 ? ROPE_THREADS : per;
  auto store_t = [](T* p, const float* x) {
    if (VEC == 1) *p = from_f32<T>(x[0]);
    else store16<T>(p, x);
  };
  auto store_q = [](QT* p, const float* x) {
    if (VEC == 1) *p = from_f32<QT>(x[0]);
    else {
#pragma unroll
      for (int i = 0; i < VEC; i += 16 / (int)sizeof(QT)) store16<QT>(p + i, x + i);
    }
  };
  for (int g = blockIdx.x, buf = 0; g < groups; g += gridDim.x, buf ^= 1) {
    const int first = g * a.tokens, nt = min(a.tokens, c.T - first);
    bool ready = false;  // the group's lookups
    for (unsigned w = w0; w < per || !ready; w += step_w) {
      const bool on = w < per && share < shares;
      // 0 q, 1 k, 2 v; head; dims at da (and db, paired with them)
      const bool is_v = w >= qk;
      const unsigned h = is_v ? (w - qk) / vu : w / hu, i = is_v ? w - qk - h * vu : w - h * hu;
      const bool is_q = !is_v && h < (unsigned)c.Hq, turned = !is_v && i < ru, two = TWO && turned;
      const unsigned da = is_v ? i * VEC : turned ? (two && a.interleaved ? 2 * i : i * VEC) : rot + (i - ru) * VEC;
      const unsigned db = a.interleaved ? da + 1 : da + rot / 2, kh = is_v ? h : h - c.Hq;
      const T* src = is_q ? static_cast<const T*>(a.q) + h * hd : static_cast<const T*>(is_v ? a.v : a.k) + kh * hd;
      const long long step = is_q ? a.qs : is_v ? a.vs : a.ks;
      RopeRaw<T, VEC> rx[ROPE_TOKENS], ry[ROPE_TOKENS];
#pragma unroll
      for (int n = 0; n < ROPE_TOKENS; ++n) {
        const int j = share + n * shares;
        if (on && j < nt) {
          rx[n].load(src + (long long)(first + j) * step + da);
          if (two) ry[n].load(src + (long long)(first + j) * step + db);
        }
      }
      if (!ready) {
        __syncthreads();
        ready = true;
      }
      if (!on) continue;
      const int pair = two ? i * VEC : da / 2;  // first pair
#pragma unroll
      for (int n = 0; n < ROPE_TOKENS; ++n) {
        const int j = share + n * shares;
        if (j >= nt) break;
        const int pos = s_pos[buf][j];
        const long long dst = s_dst[buf][j];
        T* to_k = static_cast<T*>(c.pool) + dst + (is_v ? c.Hkv + kh : kh) * seg;
        QT* to_q = static_cast<QT*>(a.q_out) + ((long long)(first + j) * c.Hq + h) * hd;
        if (!turned && (!is_q || (std::is_same<T, QT>::value && pos >= 0))) {
          if (is_q) rx[n].store(reinterpret_cast<T*>(to_q) + da);
          else if (dst >= 0) rx[n].store(to_k + da);
          continue;
        }
        float x[VEC], y[VEC];
        rx[n].get(x);
        if (TWO && two) ry[n].get(y);
        if (turned) {
          const float2* cs = s_cs[buf][j] + pair;
          if constexpr (VEC == 1) {
            const float2 f = *cs;
            const float xa = x[0], xb = y[0];
            x[0] = xa * f.x - xb * f.y;
            y[0] = xb * f.x + xa * f.y;
          } else if constexpr (TWO) {
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
              const float4 f = *reinterpret_cast<const float4*>(cs + e);
              float xa = x[e], xb = y[e];
              x[e] = xa * f.x - xb * f.y;
              y[e] = xb * f.x + xa * f.y;
              xa = x[e + 1], xb = y[e + 1];
              x[e + 1] = xa * f.z - xb * f.w;
              y[e + 1] = xb * f.z + xa * f.w;
            }
          } else {
#pragma unroll
            for (int e = 0; e < VEC; e += 4) {
              const float4 f = *reinterpret_cast<const float4*>(cs + e / 2);
              float xa = x[e], xb = x[e + 1];
              x[e] = xa * f.x - xb * f.y;
              x[e + 1] = xb * f.x + xa * f.y;
              xa = x[e + 2], xb = x[e + 3];
              x[e + 2] = xa * f.z - xb * f.w;
              x[e + 3] = xb * f.z + xa * f.w;
            }
          }
        }
        if (is_q) {
          if (pos < 0) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[e] = y[e] = 0.f;
          }
          store_q(to_q + da, x);
          if (two) store_q(to_q + db, y);
        } else if (dst >= 0) {
          store_t(to_k + da, x);
          if (two) store_t(to_k + db, y);
        }
      }
    }
  }
  pdl_trigger();
}

template <typename T, typename QT, int VEC>
static cudaError_t rope_launch(const ChunkDev& c, const RopeDev& a, cudaStream_t st) {
  const dim3 grid(std::min((c.T + a.tokens - 1) / a.tokens, a.ctas));
  if (VEC == 1 || !a.interleaved) return launch_k(k_rope_chunk<T, QT, VEC, true>, grid, dim3(ROPE_THREADS + 32), 0, st, c, a);
  return launch_k(k_rope_chunk<T, QT, VEC, false>, grid, dim3(ROPE_THREADS + 32), 0, st, c, a);
}

cudaError_t launch_rope_chunk(const ChunkDev& c, int dtype, const tlf_rope_args& a, int num_sms, cudaStream_t st) {
  RopeDev d{a.q, a.k, a.v, a.q_stride, a.k_stride, a.v_stride, a.positions, reinterpret_cast<const float2*>(a.table),
            a.max_pos, a.rot_dim, a.layout == TLF_ROPE_INTERLEAVED, 1, 3 * num_sms, a.q_out, a.entry_pos, a.entry_weight};
  const int eb = dtype == TLF_DTYPE_BF16 ? 2 : 4, vec = 16 / eb;
  const auto al = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  const bool wide = al(a.q) && al(a.k) && al(a.v) && al(a.q_out) && a.q_stride % vec == 0 &&
                    a.k_stride % vec == 0 && a.v_stride % vec == 0 &&
                    (d.interleaved ? a.rot_dim % vec == 0 : a.rot_dim / 2 % vec == 0);
  // few tokens: one a CTA
  d.tokens = std::min(ROPE_TOKENS, std::max(1, c.T / d.ctas));
  if (dtype == TLF_DTYPE_BF16) {
    if (a.q_f32) return wide ? rope_launch<bf16, float, 8>(c, d, st) : rope_launch<bf16, float, 1>(c, d, st);
    return wide ? rope_launch<bf16, bf16, 8>(c, d, st) : rope_launch<bf16, bf16, 1>(c, d, st);
  }
  return wide ? rope_launch<float, float, 4>(c, d, st) : rope_launch<float, float, 1>(c, d, st);
}

}  // namespace tlf
