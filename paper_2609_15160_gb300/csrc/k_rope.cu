// Rotary positions of new tokens and their append to a paged cache (tlf_rope_append), and rotary tables (tlf_rope_table).
//
// Pair (x_a, x_b) of a head at position p becomes (x_a c - x_b s, x_b c + x_a s), (c, s) = table[p][pair]: what is
// turned at position p and what is turned at p' then meet in q . k as a function of p - p'. The table is read, not computed:
// a float32 angle p f_k loses log2(p f_k) bits of the turn, and a row of it is shared by every head of the token.
#include <algorithm>
#include <cmath>

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
constexpr int ROPE_TOKENS = 4;  // most tokens of a CTA

struct RopeDev {
  const void *q, *k, *v;
  long long qs, ks, vs;
  const int* positions;
  const float2* table;
  int max_pos, rot, interleaved, tokens;  // tokens: of a CTA
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

// A CTA takes `tokens` tokens. Its warps look up their rows, entries and positions first (a token's row is the number of
// rows that end at or before it), then all threads go over the tokens' units: VEC elements (16 bytes) of a head, or the two
// groups of VEC that a rotation in halves pairs up. VEC = 1 takes what is not aligned to 16 bytes.
template <typename T, typename QT, int VEC>
__global__ void __launch_bounds__(ROPE_THREADS, 4) k_rope_chunk(ChunkDev c, RopeDev a) {
  pdl_wait();
  __shared__ long long s_dst[ROPE_TOKENS];  // element offset of the token's K in head 0 of its page, -1: no entry
  __shared__ int s_pos[ROPE_TOKENS];        // -1: out of range
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int first = blockIdx.x * a.tokens, nt = min(a.tokens, c.T - first);
  if (warp < nt) {
    const int t = first + warp;
    int b = 0;
    for (int i = lane; i < c.n; i += 32) b += c.cu[i + 1] <= t;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) b += __shfl_xor_sync(0xffffffffu, b, o);
    if (lane == 0) {
      int pos = a.positions[t];
      if (pos < 0 || pos >= a.max_pos) {
        sv_report(c.err, DEVERR_INDEX);
        pos = -1;
      }
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
      s_pos[warp] = pos;
      s_dst[warp] = dst;
    }
  }
  __syncthreads();

  const unsigned hd = c.hd, rot = a.rot;
  const unsigned ru = a.interleaved ? (VEC == 1 ? rot / 2 : rot / VEC) : rot / 2 / VEC;  // units of the turned dims
  const unsigned hu = ru + (hd - rot) / VEC;                                            // of a q or k head
  const unsigned vu = hd / VEC, qk = (unsigned)(c.Hq + c.Hkv) * hu, per = qk + c.Hkv * vu;
  const long long seg = (long long)SV_PAGE * hd;  // of a head in a page
  T* pool = static_cast<T*>(c.pool);
  auto load = [](const T* p, float* x) {
    if (VEC == 1) x[0] = to_f32(*p);
    else Vec16<T>::load(p, x);
  };
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
  // A thread keeps its unit and goes over the tokens, U of them in flight; units that leave threads over get several threads,
  // each with a share of the tokens.
  constexpr int U = 2;
  const unsigned shares = per >= ROPE_THREADS ? 1 : ROPE_THREADS / per;
  const int share = shares == 1 ? 0 : tid / per;
  if (share >= (int)shares) return;
  for (unsigned w = shares == 1 ? tid : tid - share * per; w < per; w += shares == 1 ? ROPE_THREADS : per) {
    if (w >= qk) {  // v: copied
      const unsigned h = (w - qk) / vu, d = (w - qk - h * vu) * VEC;
      const T* src = static_cast<const T*>(a.v) + h * hd + d;
      T* dst = pool + (c.Hkv + h) * seg + d;
      for (int j0 = share * U; j0 < nt; j0 += shares * U) {
        float x[U][VEC];
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (j0 + i < nt) load(src + (long long)(first + j0 + i) * a.vs, x[i]);
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (j0 + i < nt && s_dst[j0 + i] >= 0) store_t(dst + s_dst[j0 + i], x[i]);
      }
      continue;
    }
    const unsigned h = w / hu, i = w - h * hu;
    const bool is_q = h < (unsigned)c.Hq;
    const T* src = is_q ? static_cast<const T*>(a.q) + h * hd : static_cast<const T*>(a.k) + (h - c.Hq) * hd;
    const long long step = is_q ? a.qs : a.ks;
    T* kd = pool + ((long long)h - c.Hq) * seg;  // used for k only
    QT* qd = static_cast<QT*>(a.q_out) + (long long)first * c.Hq * hd + h * hd;
    // a unit is VEC dims at da; in halves (and element by element) also the VEC dims at db that they pair up with
    const bool turned = i < ru, two = turned && (!a.interleaved || VEC == 1);
    unsigned da, db = 0;
    if (!turned) {
      da = rot + (i - ru) * VEC;
    } else if (two) {
      da = a.interleaved ? 2 * i : i * VEC;
      db = a.interleaved ? 2 * i + 1 : i * VEC + rot / 2;
    } else {
      da = i * VEC;
    }
    const float2* cs0 = a.table + (two ? i * VEC : da / 2);
    for (int j0 = share * U; j0 < nt; j0 += shares * U) {
      float x[U][VEC], y[U][VEC];
#pragma unroll
      for (int n = 0; n < U; ++n)
        if (j0 + n < nt) {
          load(src + (long long)(first + j0 + n) * step + da, x[n]);
          if (two) load(src + (long long)(first + j0 + n) * step + db, y[n]);
        }
#pragma unroll
      for (int n = 0; n < U; ++n) {
        const int j = j0 + n;
        if (j >= nt) break;
        const int pos = s_pos[j];
        const float2* cs = cs0 + (long long)max(pos, 0) * (rot / 2);
        if (two) {
#pragma unroll
          for (int e = 0; e < VEC; e += VEC == 1 ? 1 : 2) {
            float4 f;  // two pairs
            if (VEC == 1) f = make_float4(cs->x, cs->y, 0.f, 0.f);
            else f = __ldg(reinterpret_cast<const float4*>(cs + e));
            const float xa = x[n][e], xb = y[n][e];
            x[n][e] = xa * f.x - xb * f.y;
            y[n][e] = xb * f.x + xa * f.y;
            if (VEC > 1) {
              const float va = x[n][e + (VEC > 1)], vb = y[n][e + (VEC > 1)];
              x[n][e + (VEC > 1)] = va * f.z - vb * f.w;
              y[n][e + (VEC > 1)] = vb * f.z + va * f.w;
            }
          }
        } else if (turned) {
#pragma unroll
          for (int e = 0; e + 3 < VEC; e += 4) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(cs + e / 2));
            float xa = x[n][e], xb = x[n][e + 1];
            x[n][e] = xa * f.x - xb * f.y;
            x[n][e + 1] = xb * f.x + xa * f.y;
            xa = x[n][e + 2], xb = x[n][e + 3];
            x[n][e + 2] = xa * f.z - xb * f.w;
            x[n][e + 3] = xb * f.z + xa * f.w;
          }
        }
        if (is_q) {
          if (pos < 0) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[n][e] = y[n][e] = 0.f;
          }
          store_q(qd + (long long)j * c.Hq * hd + da, x[n]);
          if (two) store_q(qd + (long long)j * c.Hq * hd + db, y[n]);
        } else if (s_dst[j] >= 0) {
          store_t(kd + s_dst[j] + da, x[n]);
          if (two) store_t(kd + s_dst[j] + db, y[n]);
        }
      }
    }
  }
  pdl_trigger();
}

template <typename T, typename QT, int VEC>
static cudaError_t rope_launch(const ChunkDev& c, const RopeDev& a, cudaStream_t st) {
  return launch_k(k_rope_chunk<T, QT, VEC>, dim3((c.T + a.tokens - 1) / a.tokens), dim3(ROPE_THREADS), 0, st, c, a);
}

cudaError_t launch_rope_chunk(const ChunkDev& c, int dtype, const tlf_rope_args& a, cudaStream_t st) {
  RopeDev d{a.q, a.k, a.v, a.q_stride, a.k_stride, a.v_stride, a.positions, reinterpret_cast<const float2*>(a.table),
            a.max_pos, a.rot_dim, a.layout == TLF_ROPE_INTERLEAVED, 1, a.q_out, a.entry_pos, a.entry_weight};
  const int eb = dtype == TLF_DTYPE_BF16 ? 2 : 4, vec = 16 / eb;
  const auto al = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  const bool wide = al(a.q) && al(a.k) && al(a.v) && al(a.q_out) && al(a.table) && a.q_stride % vec == 0 &&
                    a.k_stride % vec == 0 && a.v_stride % vec == 0 &&
                    (d.interleaved ? a.rot_dim % vec == 0 : a.rot_dim / 2 % vec == 0) && (a.rot_dim / 2) % 2 == 0;
  // few tokens: one a CTA; many: up to eight, so that a thread has several in flight
  d.tokens = std::min(ROPE_TOKENS, std::max(1, c.T / 608));
  if (dtype == TLF_DTYPE_BF16) {
    if (a.q_f32) return wide ? rope_launch<bf16, float, 8>(c, d, st) : rope_launch<bf16, float, 1>(c, d, st);
    return wide ? rope_launch<bf16, bf16, 8>(c, d, st) : rope_launch<bf16, bf16, 1>(c, d, st);
  }
  return wide ? rope_launch<float, float, 4>(c, d, st) : rope_launch<float, float, 1>(c, d, st);
}

}  // namespace tlf
