// Rotary positions of new tokens and their append to a paged cache (tlf_rope_append), and rotary tables (tlf_rope_table).
//
// Pair (x_a, x_b) of a head at position p becomes (x_a c - x_b s, x_b c + x_a s), (c, s) = table[p][pair]: what is
// turned at position p and what is turned at p' then meet in q . k as a function of p - p'. The table is read, not computed:
// a float32 angle p f_k loses log2(p f_k) bits of the turn, and a row of it is shared by every head of the token.
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
constexpr int ROPE_TOKENS = 8;  // most tokens of a CTA

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
__global__ void __launch_bounds__(ROPE_THREADS) k_rope_chunk(ChunkDev c, RopeDev a) {
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
  for (unsigned u = tid; u < nt * per; u += ROPE_THREADS) {
    const unsigned j = u / per, w = u - j * per;
    const long long t = first + (int)j, dst = s_dst[j];
    const int pos = s_pos[j];
    float x[VEC], y[VEC];
    if (w >= qk) {  // v: copied
      const unsigned h = (w - qk) / vu, d = (w - qk - h * vu) * VEC;
      if (dst < 0) continue;
      load(static_cast<const T*>(a.v) + t * a.vs + h * hd + d, x);
      store_t(pool + dst + (c.Hkv + h) * seg + d, x);
      continue;
    }
    const unsigned h = w / hu, i = w - h * hu;
    const bool is_q = h < (unsigned)c.Hq;
    if (!is_q && dst < 0) continue;
    const T* src = is_q ? static_cast<const T*>(a.q) + t * a.qs + h * hd
                        : static_cast<const T*>(a.k) + t * a.ks + (h - c.Hq) * hd;
    T* kd = pool + dst + ((long long)h - c.Hq) * seg;  // used for k only
    QT* qd = static_cast<QT*>(a.q_out) + (t * c.Hq + h) * hd;
    unsigned da, db = 0;
    bool two = false;
    if (i >= ru) {  // behind the turned dims
      da = rot + (i - ru) * VEC;
      load(src + da, x);
    } else if (!a.interleaved || VEC == 1) {
      const unsigned k = i * VEC;  // first pair
      da = a.interleaved ? 2 * k : k;
      db = a.interleaved ? 2 * k + 1 : k + rot / 2;
      two = true;
      load(src + da, x);
      load(src + db, y);
      const float2* cs = a.table + (long long)max(pos, 0) * (rot / 2) + k;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float2 f = cs[e];
        const float xa = x[e], xb = y[e];
        x[e] = xa * f.x - xb * f.y;
        y[e] = xb * f.x + xa * f.y;
      }
    } else {
      da = i * VEC;
      load(src + da, x);
      const float2* cs = a.table + (long long)max(pos, 0) * (rot / 2) + da / 2;
#pragma unroll
      for (int e = 0; e + 1 < VEC; e += 2) {
        const float2 f = cs[e / 2];
        const float xa = x[e], xb = x[e + 1];
        x[e] = xa * f.x - xb * f.y;
        x[e + 1] = xb * f.x + xa * f.y;
      }
    }
    if (is_q) {
      if (pos < 0) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = y[e] = 0.f;
      }
      store_q(qd + da, x);
      if (two) store_q(qd + db, y);
    } else {
      store_t(kd + da, x);
      if (two) store_t(kd + db, y);
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
                    (d.interleaved ? a.rot_dim % vec == 0 : a.rot_dim / 2 % vec == 0);
  const int units = (c.Hq + 2 * c.Hkv) * c.hd / (wide ? vec : 1);
  // few tokens: one a CTA; many: about four units a thread
  if (c.T > 1024) d.tokens = std::min(ROPE_TOKENS, std::max(1, 4 * ROPE_THREADS / units));
  if (dtype == TLF_DTYPE_BF16) {
    if (a.q_f32) return wide ? rope_launch<bf16, float, 8>(c, d, st) : rope_launch<bf16, float, 1>(c, d, st);
    return wide ? rope_launch<bf16, bf16, 8>(c, d, st) : rope_launch<bf16, bf16, 1>(c, d, st);
  }
  return wide ? rope_launch<float, float, 4>(c, d, st) : rope_launch<float, float, 1>(c, d, st);
}

}  // namespace tlf
