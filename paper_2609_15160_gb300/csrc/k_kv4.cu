// Rotary positions of new tokens and their append to a cache held in 4 bits (tlf_kv4_append), and entries back out of it
// (tlf_kv4_read).
//
// A lane has eight neighbouring dims of a head, which is a word of codes, so a group of 64 values is eight lanes and its least and
// largest value meet in three shuffles; the dims that a rotation pairs with a lane's own come from memory again (the same lines). A
// warp goes over a token's heads, 256 / head_dim at a time, so that a lane's dims, and with them its row of the rotary table, stay
// the same for all of them. Sums and products are rounded one by one: a code next to a border does not depend on how they are
// fused.
//
// Bound by instructions (69 % of the issue slots) and the latency of a token's passes, two waves of warps: 7157 tokens, 16 / 8 heads
// x 128, 64 dims turned: 33 us; reading them back 12 us. With the compiler's divisions 79 us. 64 tokens, 16 heads x 64: 6.3 us with
// their read, in a graph.
#include <algorithm>

#include "k_kv4.cuh"

namespace tlf {

struct Kv4Append {
  const void *q, *k, *v;
  long long qs, ks, vs;
  const int* positions;
  const float2* table;
  int max_pos, rot, interleaved, q_f32, parts;  // parts: warps that share a token's heads
  void* q_out;
  int* entry_pos;
  float* entry_weight;
};

// Row of token t: the number of rows that end at or before it. 32 rows a step.
__device__ __forceinline__ int token_row(const ChunkDev& c, int t) {
  const int lane = threadIdx.x & 31, step = (c.n + 31) / 32, at = (lane + 1) * step;
  const int lo = __popc(__ballot_sync(0xffffffffu, at <= c.n && c.cu[at] <= t)) * step;  // rows before lo end at or before it
  int b = lo;
  for (int i = lo; i < min(c.n, lo + step); i += 32) b += __popc(__ballot_sync(0xffffffffu, i + lane < min(c.n, lo + step) && c.cu[i + lane + 1] <= t));
  return b;
}

// The entry of token t: byte offset of K's block of head 0 and place in the page; -1 (reported) without one.
struct TokenEntry {
  long long block, slot;  // bytes from the pool's start; page * 64 + place
  int off;
};
__device__ __forceinline__ TokenEntry token_entry(const ChunkDev& c, int t, int block_bytes) {
  TokenEntry e{-1, 0, 0};
  const int b = token_row(c, t);
  const ChunkRow r = b < c.n ? chunk_row(c, b) : ChunkRow{0, 0, 0};
  const int i = t - r.t0, at = r.len - r.ql + i;
  if (i < 0 || i >= r.ql || at < 0) {
    sv_report(c.err, DEVERR_INDEX);
    return e;
  }
  const int page = chunk_page(c.page_table, c.max_pages, c.n_pages, b, at / SV_PAGE, c.err);
  if (page < 0) return e;
  e.off = at % SV_PAGE;
  e.slot = (long long)page * SV_PAGE + e.off;
  e.block = page * c.page_elems + (long long)c.layer * 2 * c.Hkv * block_bytes;
  return e;
}

// Eight elements. WIDE: aligned to 16 bytes.
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T* p, float* x) {
  if constexpr (WIDE) {
    constexpr int N = Vec16<T>::N;
#pragma unroll
    for (int i = 0; i < 8; i += N) Vec16<T>::load(p + i, x + i);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_f32(p[i]);
  }
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store8(T* p, const float* x) {
  if constexpr (!WIDE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = from_f32<T>(x[i]);
  } else if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// Eight elements as they come from memory, so that several units of a lane are in flight.
template <typename T, bool WIDE>
struct Raw8 {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
    } else {
      T* x = reinterpret_cast<T*>(v);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = p[i];
    }
  }
  __device__ __forceinline__ void get(float* x) const { load8<T, true>(reinterpret_cast<const T*>(v), x); }
};

// The eight codes of a lane's values, whose group of GL lanes the warp's lanes form; *pair: (d, lo) of the group. x: what a plain cache
// would hold.
//
// The quotient (x - lo) / d of the definition, rounded once, in three instructions: with r = 1 / d rounded to nearest, q = t r, q +
// (t - q d) r is t / d rounded to nearest (Markstein, 1990; d's significand is not all ones: it has 8 bits). Out of the range where no
// step under- or overflows the division itself. Adding 1.5 x 2^23 rounds to an integer, ties to even, in the low bits. EXACT: lo is the
// least value itself, as it is of bfloat16 values: t / d is in 0 .. 15 (1 + 2^-8), and needs no clamp.
template <int GL, bool EXACT>
__device__ __forceinline__ uint32_t quantise(float (&x)[8], uint32_t* pair, bool* bad) {
  constexpr float LARGEST = 0x1p126f, ROUND = 12582912.f;
  constexpr uint32_t ROUND_BITS = 0x4b400000u;
  auto least = [&] { return fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])), fminf(fminf(x[4], x[5]), fminf(x[6], x[7]))); };
  auto most = [&] { return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))); };
  float lo = least(), hi = most();
  uint64_t zero2 = 0;
#pragma unroll
  for (int i = 0; i < 8; i += 2) zero2 = f2_fma(f2_pack(x[i], x[i + 1]), 0, zero2);  // infinities and NaN: not a number
  const float2 zero = f2_unpack(zero2);
  const bool odd = !(zero.x + zero.y == 0.f) || !(fmaxf(-lo, hi) <= LARGEST);
  *bad = odd;
  if (odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] != x[i] ? 0.f : fmaxf(fminf(x[i], LARGEST), -LARGEST);
    lo = least();
    hi = most();
  }
#pragma unroll
  for (int o = 1; o < GL; o *= 2) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const bf16 lo16 = __float2bfloat16_rn(lo);
  lo = __bfloat162float(lo16);
  const bf16 d16 = __float2bfloat16_rn(__fdiv_rn(fmaxf(__fsub_rn(hi, lo), 0.f), 15.f));
  const float d = __bfloat162float(d16);
  *pair = (uint32_t)__bfloat16_as_ushort(d16) | (uint32_t)__bfloat16_as_ushort(lo16) << 16;
  uint32_t word = 0;
  if (d >= 0x1p-80f && d <= 0x1p80f) {
    const float r = __frcp_rn(d);
    constexpr uint32_t EIGHT = (uint32_t)(0x11111111ull * ROUND_BITS);  // what the eight shifted ROUND_BITS add up to
    const uint64_t lo2 = f2_pack(-lo, -lo), r2 = f2_pack(r, r), d2 = f2_pack(-d, -d), round2 = f2_pack(ROUND, ROUND);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {  // (two at a time, each step rounded as it would be alone)
      const uint64_t t = f2_add(f2_pack(x[i], x[i + 1]), lo2), q = f2_mul(t, r2);
      uint64_t n = f2_fma(f2_fma(q, d2, t), r2, q);
      if (!EXACT) {
        const float2 c = f2_unpack(n);
        n = f2_pack(fminf(fmaxf(c.x, 0.f), 15.f), fminf(fmaxf(c.y, 0.f), 15.f));
      }
      const float2 b = f2_unpack(f2_add(n, round2));
      word += (__float_as_uint(b.x) << (4 * i)) + (__float_as_uint(b.y) << (4 * i + 4));
    }
    word -= EIGHT;
  } else if (d > 0.f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) word |= (uint32_t)fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x[i], lo), d)), 0.f), 15.f) << (4 * i);
  }
  return word;
}

template <typename T, int HD, bool WIDE>
__global__ void __launch_bounds__(256, 3) k_kv4_append(ChunkDev c, Kv4Append a) {
  using F = Kv4<HD>;
  constexpr int L = HD / 8, HP = 32 / L, GL = F::GS / 8;  // lanes of a head, heads of a pass, lanes of a group
  pdl_wait();
  const int lane = threadIdx.x & 31, d0 = (lane % L) * 8, half = a.rot / 2;
  const int pq = (c.Hq + HP - 1) / HP, pk = (c.Hkv + HP - 1) / HP, passes = pq + 2 * pk;  // q's passes, then k's, then v's
  const bool turns = d0 < a.rot, pairs = turns && !a.interleaved;
  const int partner = d0 < half ? half : -half;
  const long long warps = (long long)gridDim.x * 8, all = (long long)c.T * a.parts;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < all; w += warps) {
    const int t = (int)(w / a.parts), part = (int)(w % a.parts);
    const T *q_row = static_cast<const T*>(a.q) + t * a.qs, *k_row = static_cast<const T*>(a.k) + t * a.ks, *v_row = static_cast<const T*>(a.v) + t * a.vs;
    // the lane's eight dims of pass p, and those that they are paired with; the next pass is in flight while one is worked on
    auto load = [&](Raw8<T, WIDE>& x, Raw8<T, WIDE>& y, int p) {
      const bool is_q = p < pq, is_v = p >= pq + pk;
      const int h = (is_q ? p : is_v ? p - pq - pk : p - pq) * HP + lane / L;
      if (h >= (is_q ? c.Hq : c.Hkv)) return;
      const T* src = (is_q ? q_row : is_v ? v_row : k_row) + (unsigned)h * HD;
      x.load(src + d0);
      if (is_v || !pairs) return;
      if constexpr (WIDE) {
        y.load(src + (d0 + partner));
      } else {
        T* to = reinterpret_cast<T*>(y.v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int d = d0 + i;
          if (d < a.rot) to[i] = src[d < half ? d + half : d - half];
        }
      }
    };
    Raw8<T, WIDE> rx{}, ry{};
    if (part < passes) load(rx, ry, part);
    int pos = a.positions[t];
    const bool there = pos >= 0 && pos < a.max_pos;
    if (!there) {
      if (lane == 0) sv_report(c.err, DEVERR_INDEX);
      pos = 0;
    }
    float2 cs[8];  // cosine and sine of each of the lane's dims
    const float2* row = a.table + (long long)pos * half;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = d0 + i;
      cs[i] = d >= a.rot ? make_float2(1.f, 0.f) : a.interleaved ? row[d / 2] : row[d < half ? d : d - half];
      // x_a c - x_b s, x_b c + x_a s: the sign of what the paired dim adds
      if (d < a.rot && (a.interleaved ? d % 2 == 0 : d < half)) cs[i].y = -cs[i].y;
    }
    TokenEntry e = token_entry(c, t, F::BLOCK);
    if (!there) e.block = -1;
    if (part == 0 && lane == 0 && e.block >= 0) {
      if (a.entry_pos) a.entry_pos[e.slot] = pos;
      if (a.entry_weight) a.entry_weight[e.slot] = 0.f;
    }
    uint8_t* blocks = static_cast<uint8_t*>(c.pool) + e.block;
    const unsigned code_at = e.off * (HD / 2) + d0 / 2, pair_at = F::CODES + (e.off * F::NG + d0 / F::GS) * 4;
    const long long out0 = (long long)t * c.Hq * HD;
    const int end = e.block >= 0 ? passes : pq;  // without an entry: the query alone
    for (int p = part; p < end; p += a.parts) {
      Raw8<T, WIDE> nx{}, ny{};
      if (p + a.parts < end) load(nx, ny, p + a.parts);
      const bool is_q = p < pq, is_v = p >= pq + pk;
      const int h = (is_q ? p : is_v ? p - pq - pk : p - pq) * HP + lane / L;
      const bool on = h < (is_q ? c.Hq : c.Hkv);
      float x[8];
      rx.get(x);
      if (!is_v && turns) {
        float y[8];
        if (pairs) {
          ry.get(y);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)  // (products and sums rounded one by one; two an instruction, the compiler fuses them)
          if (WIDE || d0 + i < a.rot) x[i] = __fadd_rn(__fmul_rn(x[i], cs[i].x), __fmul_rn(y[i], cs[i].y));
      }
      if (is_q) {
        if (on) {
          if (!there)
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.f;
          const unsigned to = (unsigned)h * HD + d0;
          if (a.q_f32) store8<float, WIDE>(static_cast<float*>(a.q_out) + out0 + to, x);
          else store8<T, WIDE>(static_cast<T*>(a.q_out) + out0 + to, x);
        }
      } else {
        if (sizeof(T) == 2 && !is_v) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = to_f32(from_f32<T>(x[i]));
        }
        if (!on)  // (the lanes of a head that is none take part in the groups' exchanges)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = 0.f;
        uint32_t pair;
        bool bad;
        const uint32_t word = quantise<GL, sizeof(T) == 2>(x, &pair, &bad);
        if (on) {
          if (bad) sv_report(c.err, SVERR_VALUE);
          uint8_t* block = blocks + (size_t)(is_v ? c.Hkv + h : h) * F::BLOCK;
          *reinterpret_cast<uint32_t*>(block + code_at) = word;
          if (d0 % F::GS == 0) *reinterpret_cast<uint32_t*>(block + pair_at) = pair;
        }
      }
      rx = nx;
      ry = ny;
    }
  }
  pdl_trigger();
}

struct Kv4Read {
  void *k, *v;
  long long ks, vs;
  int parts;
};
template <typename T, int HD, bool WIDE>
__global__ void __launch_bounds__(256) k_kv4_read(ChunkDev c, Kv4Read a) {
  using F = Kv4<HD>;
  constexpr int L = HD / 8, HP = 32 / L;
  pdl_wait();
  const int lane = threadIdx.x & 31, d0 = (lane % L) * 8, passes = (2 * c.Hkv + HP - 1) / HP;
  const long long warps = (long long)gridDim.x * 8, all = (long long)c.T * a.parts;
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < all; w += warps) {
    const int t = (int)(w / a.parts);
    const TokenEntry e = token_entry(c, t, F::BLOCK);
    constexpr int U = 4;  // passes in flight
    for (int p = (int)(w % a.parts); p < passes; p += U * a.parts) {
      uint32_t word[U], pair[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = (p + u * a.parts) * HP + lane / L;
        word[u] = pair[u] = 0;
        if (h < 2 * c.Hkv && e.block >= 0) {
          const uint8_t* block = static_cast<const uint8_t*>(c.pool) + e.block + (long long)h * F::BLOCK;
          word[u] = *reinterpret_cast<const uint32_t*>(block + e.off * (HD / 2) + d0 / 2);
          pair[u] = *reinterpret_cast<const uint32_t*>(block + F::CODES + (e.off * F::NG + d0 / F::GS) * 4);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = (p + u * a.parts) * HP + lane / L;
        const bool is_v = h >= c.Hkv;
        T* to = static_cast<T*>(is_v ? a.v : a.k);
        if (h >= 2 * c.Hkv || !to) continue;
        float x[8];
        kv4_values(word[u], kv4_pair(pair[u]), x);
        store8<T, WIDE>(to + t * (is_v ? a.vs : a.ks) + (long long)(is_v ? h - c.Hkv : h) * HD + d0, x);
      }
    }
  }
  pdl_trigger();
}

// Warps that share a token: one each where the tokens fill the GPU, else as many as it has passes (append and read, 16 / 8 heads x 128:
// 7157 tokens 44.9 us, with two 49.1; 1600 tokens 16.1, with one 17.9; 512 tokens 11.0, with one 14.2).
static int token_parts(int T, int passes, int num_sms) {
  return (int)std::min<long long>(passes, std::max<long long>(1, (long long)num_sms * 32 / std::max(1, T)));
}
static unsigned warp_grid(long long warps, int num_sms) { return (unsigned)std::min<long long>((warps + 7) / 8, 8LL * num_sms); }

template <typename T, int HD>
static cudaError_t append_launch(const ChunkDev& c, Kv4Append a, bool wide, int num_sms, cudaStream_t st) {
  constexpr int HP = 256 / HD;
  a.parts = token_parts(c.T, (c.Hq + HP - 1) / HP + 2 * ((c.Hkv + HP - 1) / HP), num_sms);
  const dim3 grid(warp_grid((long long)c.T * a.parts, num_sms));
  return wide ? launch_k(k_kv4_append<T, HD, true>, grid, dim3(256), 0, st, c, a) : launch_k(k_kv4_append<T, HD, false>, grid, dim3(256), 0, st, c, a);
}
cudaError_t launch_kv4_append(const ChunkDev& c, int dtype, const tlf_rope_args& a, int num_sms, cudaStream_t st) {
  const Kv4Append d{a.q, a.k, a.v, a.q_stride, a.k_stride, a.v_stride, a.positions, reinterpret_cast<const float2*>(a.table),
                    a.max_pos, a.rot_dim, a.layout == TLF_ROPE_INTERLEAVED, a.q_f32, 1, a.q_out, a.entry_pos, a.entry_weight};
  const int vec = dtype == TLF_DTYPE_BF16 ? 8 : 4;
  const auto al = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  const bool wide = al(a.q) && al(a.k) && al(a.v) && al(a.q_out) && a.q_stride % vec == 0 && a.k_stride % vec == 0 &&
                    a.v_stride % vec == 0 && (d.interleaved ? a.rot_dim % 8 == 0 : a.rot_dim % 16 == 0);
  if (dtype == TLF_DTYPE_BF16)
    return c.hd == 32   ? append_launch<bf16, 32>(c, d, wide, num_sms, st)
           : c.hd == 64 ? append_launch<bf16, 64>(c, d, wide, num_sms, st)
                        : append_launch<bf16, 128>(c, d, wide, num_sms, st);
  return c.hd == 16   ? append_launch<float, 16>(c, d, wide, num_sms, st)
         : c.hd == 32 ? append_launch<float, 32>(c, d, wide, num_sms, st)
         : c.hd == 64 ? append_launch<float, 64>(c, d, wide, num_sms, st)
                      : append_launch<float, 128>(c, d, wide, num_sms, st);
}

template <typename T, int HD>
static cudaError_t read_launch(const ChunkDev& c, Kv4Read a, bool wide, int num_sms, cudaStream_t st) {
  constexpr int HP = 256 / HD;
  a.parts = token_parts(c.T, (2 * c.Hkv + HP - 1) / HP, num_sms);
  const dim3 grid(warp_grid((long long)c.T * a.parts, num_sms));
  return wide ? launch_k(k_kv4_read<T, HD, true>, grid, dim3(256), 0, st, c, a) : launch_k(k_kv4_read<T, HD, false>, grid, dim3(256), 0, st, c, a);
}
cudaError_t launch_kv4_read(const ChunkDev& c, int dtype, const tlf_kv4_read_args& a, int num_sms, cudaStream_t st) {
  const long long row = (long long)c.Hkv * c.hd;
  const Kv4Read d{a.k, a.v, a.k_stride ? a.k_stride : row, a.v_stride ? a.v_stride : row, 1};
  const int vec = dtype == TLF_DTYPE_BF16 ? 8 : 4;
  const auto al = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  const bool wide = al(a.k) && al(a.v) && d.ks % vec == 0 && d.vs % vec == 0;
  if (dtype == TLF_DTYPE_BF16)
    return c.hd == 32   ? read_launch<bf16, 32>(c, d, wide, num_sms, st)
           : c.hd == 64 ? read_launch<bf16, 64>(c, d, wide, num_sms, st)
                        : read_launch<bf16, 128>(c, d, wide, num_sms, st);
  return c.hd == 16   ? read_launch<float, 16>(c, d, wide, num_sms, st)
         : c.hd == 32 ? read_launch<float, 32>(c, d, wide, num_sms, st)
         : c.hd == 64 ? read_launch<float, 64>(c, d, wide, num_sms, st)
                      : read_launch<float, 128>(c, d, wide, num_sms, st);
}

}  // namespace tlf
