// Attention of chunks of new tokens over caches in 4 bits, under a window or not (tlf_attn_window), bfloat16 calls. Items, their
// split over the CTAs and the join are those of k_chunk.cu.
//
// k_chunk_q4     up to 16 query rows an item: codes straight from shared memory into mma.sync fragments;
// k_chunk_pair4  more: codes turned into float16 tiles for tcgen05, pairs of 128-row tiles.
#include <algorithm>

#include <cuda_fp16.h>

#include "k_chunk4.cuh"
#include "k_kv4.cuh"

namespace tlf {

// ----------------------------------------------------------------------------
// Few rows
// ----------------------------------------------------------------------------
// Keys are the rows of the products and query rows their columns (8 a tile), S = K Q^T and O^T = V^T P^T: one instruction takes 16
// keys or dims. No code is ever converted: the bits of a code in the low end of a 16-bit half, n or 16 n, are the float16 number
// n 2^-24 or n 2^-20 (a subnormal, exact, and the tensor cores take those at full speed), so that a word's eight codes are four masked
// pairs; for 16 n the other operand (q), or the result (O), is a sixteenth. Sums are float32:
//   s = scale (sum over groups g of d_g (q . n)_g + lo_g (sum of q)_g),   O = sum_t p_t d_t,g n_t + sum_t p_t lo_t,g
// A lane's word of K has codes i and i + 4 in one register, which q's fragment follows; words of V of two neighbouring keys are
// paired by byte permutations. q is scaled by a power of two a row into float16's range.
//
// p_t d_t,g is rounded to float16, an operand's type, as the other kernels round p. What float16 has to hold is 2^(s - M) d: M + 8 is
// the running maximum of s + log2(d), the largest d of the entry's groups, not of s, so that values of any magnitude fit. It is refreshed
// when a p d passes 2^15, or a lane's sum of p 2^80. d counts as at least 2^-64 |lo| in all of this: a group that holds one value has
// none (and codes of 0, or 15 2^-64 of the value too much), and p lo then is below 2^79; and as at least 2^-60 in M: p is at most 2^68.
// So float32 holds the sums over 2^31 entries. Digits go where values are below 2^-80, and, where they are of 2^100 and more, with what
// weighs less than 2^-26.
//
// CTAs of teams of two warps, which take the pages in turn, a warp half of a page's 64 keys, 16 at a time in each step of the
// products; and a producer warp that copies a page's two blocks.
//
// Bound by the latency of dependent instructions: the twelve warps that 128 registers a thread leave room for issue in 53 % of the
// cycles. 16 single tokens over 32k entries, 16 / 8 heads x 128: 125 us with the join, 4.7 TB/s; 32 over up to 8192 entries, 16 heads x
// 64: 55 us; 32 rows of up to 16 tokens under a window of 4096, 16 heads x 64: 60 us. The first of them with one team and 16 keys a step
// 153 us, with more warps a CTA 163, with four CTAs an SM 153 and with two 132.
struct Q4Seg {  // a CTA's part of an item: blocks kb0 .. kb1 - 1 of nb; nb = 0: no more
  int b, h, token0, see0, nq, kb0, kb1, nb;
  static constexpr int RING = 4;
};
constexpr int Q4_WARPS(int hd, int nt) { return 4; }
constexpr int Q4_PER_SM(int hd, int nt) { return hd == 128 ? (nt == 2 ? 2 : 3) : nt == 2 ? 3 : 4; }
constexpr int Q4_NST(int hd, int nt) { return hd == 128 ? (nt == 2 ? 8 : 6) : hd == 64 ? 8 : 12; }
template <int HD, int NT>
struct Q4Shape {
  using F = Kv4<HD>;
  static constexpr int WARPS = Q4_WARPS(HD, NT), TEAMS = WARPS / 2;
  static constexpr int RT = 8 * NT, THREADS = 32 * (WARPS + 1), STAGE = 2 * F::BLOCK;
  static constexpr int PER_SM = Q4_PER_SM(HD, NT);
  static constexpr int NST = Q4_NST(HD, NT);  // a multiple of TEAMS: a stage is always the same team's
  static_assert(NST % TEAMS == 0, "");
  static constexpr int OS = HD + 4;  // floats of a merge buffer's row
  static constexpr int OFF_O = NST * STAGE, OFF_ML = OFF_O + TEAMS * RT * OS * 4, OFF_BAR = OFF_ML + WARPS * RT * 8;
  static constexpr int NBAR = 2 * NST + 2 * Q4Seg::RING;
  static constexpr int OFF_INT = OFF_BAR + NBAR * 8, OFF_SEG = OFF_INT + (NST + 2) / 2 * 8, OFF_BASE = OFF_SEG + Q4Seg::RING * (int)sizeof(Q4Seg);
  static int bytes(int n) { return OFF_BASE + (n + 1) * 8 + 128; }
};

__device__ __forceinline__ void mma_f16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {  // of halves: row lane / 4, columns 2 (lane % 4)..
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

template <int HD, int NT>
__global__ void __launch_bounds__(Q4Shape<HD, NT>::THREADS, Q4Shape<HD, NT>::PER_SM) k_chunk_q4(ChunkAttn a) {
  using Sh = Q4Shape<HD, NT>;
  using F = Kv4<HD>;
  constexpr int NST = Sh::NST, NG = F::NG, W = F::GS / 32, MT = F::GS / 16, OS = Sh::OS, RT = Sh::RT;  // W: words of K a lane has of a group
  constexpr uint32_t LO = 0x000f000fu, HI = 0x00f000f0u;
  constexpr float NONE = -3e38f;  // M before the first key
  extern __shared__ uint8_t smem_raw[];
  __shared__ long long s_red[33];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~uintptr_t(127));
  float* s_o = reinterpret_cast<float*>(sm + Sh::OFF_O);
  float2* s_ml = reinterpret_cast<float2*>(sm + Sh::OFF_ML);
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + Sh::OFF_BAR);
  volatile int* s_skip = reinterpret_cast<volatile int*>(sm + Sh::OFF_INT);  // [NST] the page is not there
  volatile int* abort_flag = s_skip + NST;
  Q4Seg* s_seg = reinterpret_cast<Q4Seg*>(sm + Sh::OFF_SEG);
  long long* s_base = reinterpret_cast<long long*>(sm + Sh::OFF_BASE);
  auto full = [&](int st) { return smem_u32(&bars[st]); };
  auto empty = [&](int st) { return smem_u32(&bars[NST + st]); };
  auto seg_full = [&](unsigned i) { return smem_u32(&bars[2 * NST + i % Q4Seg::RING]); };
  auto seg_empty = [&](unsigned i) { return smem_u32(&bars[2 * NST + Q4Seg::RING + i % Q4Seg::RING]); };
  const ChunkDev& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(full(i), 1);
      mbar_init(empty(i), 2);
    }
    for (unsigned i = 0; i < Q4Seg::RING; ++i) {
      mbar_init(seg_full(i), 1);
      mbar_init(seg_empty(i), 1);
    }
    *abort_flag = 0;
    fence_barrier_init();
  }
  pdl_wait();
  const WindowSplit sp = split_of<KEYS_4BIT>(a);
  const int sinks = sp.sinks();
  chunk_plan(c, sp, s_base, s_red);
  pdl_trigger();
  const long long all = s_base[c.n], per = chunk_share(a, all);
  long long pos = blockIdx.x * per;
  const long long end = pos + per < all ? pos + per : all;
  const int G = c.G, qt = 1 << a.sp.qt_log;
  // a bounded wait; once one has run out, the others are skipped and everybody winds down
  auto wait = [&](uint32_t b, uint32_t parity) {
    if (mbar_try_wait(b, parity & 1u)) return true;
    if (*abort_flag) return false;
    if (mbar_wait(b, parity & 1u, a.werr)) return true;
    *abort_flag = 1;
    return false;
  };
  unsigned seq = 0;  // pages that this CTA's ring has taken

  if (warp == Sh::WARPS) {
    // ---------------- producer ----------------
    bool ok = true;
    for (unsigned segs = 0;; ++segs) {
      ChunkItem it{};
      Q4Seg s{};
      if (pos < end) {
        it = chunk_item(c, sp, s_base, pos);
        if (segs == 0 && lane == 0) join_note(a, &it, per);
        if (pos < it.first) pos = it.first;
      } else if (segs == 0 && lane == 0) {
        join_note(a, nullptr, per);
      }
      if (pos < end) {
        const int q0 = it.t << a.sp.qt_log;
        s = Q4Seg{it.b, it.h, it.t0 + q0, it.s0 + q0, min(qt, it.ql - q0), (int)(pos - it.first),
                  (int)(end - it.first < it.nb ? end - it.first : it.nb), it.nb};
        pos = it.first + s.kb1;
      }
      if (lane == 0) {
        ok = ok && (segs < Q4Seg::RING || wait(seg_empty(segs), segs / Q4Seg::RING - 1));
        if (ok) {
          s_seg[segs % Q4Seg::RING] = s;
          mbar_arrive(seg_full(segs));
        }
      }
      if (s.nb == 0) break;
      const long long k_at = ((long long)c.layer * 2 * c.Hkv + s.h) * F::BLOCK, v_at = k_at + (long long)c.Hkv * F::BLOCK;
      for (int g0 = s.kb0; g0 < s.kb1; g0 += 32) {
        int mine = -1;
        const int at = block_at<KEYS_4BIT>(g0 + lane, sinks, it.skip);
        if (g0 + lane < s.kb1 && at * 64 < it.len) mine = chunk_page(c.page_table, c.max_pages, c.n_pages, s.b, at, c.err);
        for (int i = 0; i < min(32, s.kb1 - g0); ++i, ++seq) {
          const int page = __shfl_sync(0xffffffffu, mine, i), st = seq % NST;
          if (lane == 0 && ok) {
            ok = seq < NST || wait(empty(st), seq / NST - 1);
            if (ok) {
              s_skip[st] = page < 0;
              if (page < 0) {
                mbar_arrive(full(st));
              } else {
                mbar_arrive_expect_tx(full(st), Sh::STAGE);
                const uint8_t* src = static_cast<const uint8_t*>(c.pool) + page * c.page_elems;
                const uint32_t dst = smem_u32(sm + st * Sh::STAGE);
                bulk_g2s(dst, src + k_at, F::BLOCK, full(st));
                bulk_g2s(dst + F::BLOCK, src + v_at, F::BLOCK, full(st));
              }
            }
          }
          __syncwarp();
        }
      }
    }
    if (*abort_flag) drain_copies();
    return;
  }

  const int g = lane >> 2, cl = lane & 3;
  // the key of row r of the products, of 8: two keys a lane pair up (V), and loads of neighbouring lanes meet few bank conflicts
  auto kappa = [](int r) { return HD == 128 ? (r & 1 ? 4 + ((r / 2 + 1) & 3) : r / 2) : r; };
  const int team = warp >> 1, half = (warp & 1) * 32;
  const int ka = half + kappa(g);                                     // K, pairs: keys ka, ka + 8, ka + 16, ka + 24 of the page
  const int va = half + kappa(2 * cl), vb = half + kappa(2 * cl + 1);  // V: keys va, vb, va + 8, vb + 8, ..
  for (unsigned segs = 0;; ++segs) {
    // the warps leave together or not at all: they meet at barriers below, which know no time limit
    if (bar_any(1, 32 * Sh::WARPS, !wait(seg_full(segs), segs / Q4Seg::RING))) break;
    const Q4Seg it = s_seg[segs % Q4Seg::RING];
    if (it.nb == 0) break;
    const int nq = it.nq, rows = nq * G, see0 = it.see0, see_last = see0 + nq - 1;
    const int skip = sp.skip_at(see0), gone_to = hidden_to(see0, a.window), edge_to = hidden_to(see_last, a.window);
    // 2^24 and the scale together may pass float32's range; where they could, q of finite scores is small, and the power goes to q's
    const bool vast = a.scale > 0x1p64f;
    // q of row g of every tile: dims 64 grp + 8 w + i, words w = 2 cl, 2 cl + 1 (head_dim 32: w = cl)
    uint32_t qf[NT][NG][W][4];
    float fa[NT][2], qs[NT][NG][2];  // of this lane's columns 2 cl, 2 cl + 1: what the scaled q counts, scale times the sums of q
    int see[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int r = t * 8 + g;
      float x[NG][W][8], sum[NG], mx = 0.f;
      const bf16* row = static_cast<const bf16*>(a.q) + (it.token0 + (long long)(r / G)) * a.qs + (long long)(it.h * G + r % G) * HD;
      const bool wide = reinterpret_cast<uintptr_t>(row) % 16 == 0;
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        sum[n] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const int d = n * F::GS + (cl * W + w) * 8;
          if (r < rows && wide) Vec16<bf16>::load(row + d, x[n][w]);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (r >= rows) x[n][w][i] = 0.f;
            else if (!wide) x[n][w][i] = to_f32(row[d + i]);
            sum[n] += x[n][w][i];
            mx = fmaxf(mx, fabsf(x[n][w][i]));
          }
        }
        sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 1);
        sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 2);
      }
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      // a power of two that puts the largest into 2^14 .. 2^15
      const int e = max(-112, min(126, (int)(__float_as_uint(mx) >> 23) - 127));
      const float up = __uint_as_float((uint32_t)(14 - e + 127) << 23), down = __uint_as_float((uint32_t)(max(e - 14, -126) + 127) << 23);
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float f = i & 1 ? up * 0.0625f : up;
            qf[t][n][w][i] = pack_f16(x[n][w][i] * f, x[n][w][i + 4] * f);
          }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int from = 4 * (2 * cl + j), rj = t * 8 + 2 * cl + j;
        fa[t][j] = __shfl_sync(0xffffffffu, down, from) * (vast ? 0x1p64f : 1.f);
#pragma unroll
        for (int n = 0; n < NG; ++n) qs[t][n][j] = __shfl_sync(0xffffffffu, sum[n], from) * a.scale;
        // rows past the tile's see what its first query sees, with q = 0; nobody reads them
        see[t][j] = see0 + (rj < rows ? rj / G : 0);
      }
    }
    const float fb = a.scale * (vast ? 0x1p-40f : 0x1p24f);
    float m[NT][2], l[NT][2], ol[NT][NG][2], o[NT][NG][MT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        m[t][j] = NONE;
        l[t][j] = 0.f;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          ol[t][n][j] = 0.f;
#pragma unroll
          for (int i = 0; i < MT; ++i) o[t][n][i][2 * j] = o[t][n][i][2 * j + 1] = 0.f;
        }
      }

    for (int kb = it.kb0; kb < it.kb1; ++kb, ++seq) {
      if ((int)(seq % Sh::TEAMS) != team) continue;
      const int st = seq % NST;
      const bool ok = __all_sync(0xffffffffu, wait(full(st), seq / NST));
      const int page0 = block_at<KEYS_4BIT>(kb, sinks, skip) * 64, key0 = page0 + half;
      if (ok && !s_skip[st] && key0 <= see_last && !(key0 >= a.first && key0 + 31 <= gone_to)) {
        const uint8_t *sk = sm + st * Sh::STAGE, *sv = sk + F::BLOCK;
        uint64_t s2[NT][4];  // scores of keys ka + 8 x, both columns
        {
          uint64_t dn[NT][4], lo[NT][4];
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            float acc[NT][2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              uint32_t wa[W], wb[W];
              const uint8_t* p = sk + (ka + 16 * u) * (HD / 2) + n * 32 + cl * (4 * W);
              if constexpr (W == 2) {
                *reinterpret_cast<uint2*>(wa) = *reinterpret_cast<const uint2*>(p);
                *reinterpret_cast<uint2*>(wb) = *reinterpret_cast<const uint2*>(p + 8 * (HD / 2));
              } else {
                wa[0] = *reinterpret_cast<const uint32_t*>(p);
                wb[0] = *reinterpret_cast<const uint32_t*>(p + 8 * (HD / 2));
              }
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][u][i] = 0.f;
#pragma unroll
              for (int w = 0; w < W; ++w) {
                const uint32_t xa = wa[w] >> 8, xb = wb[w] >> 8;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                  mma_f16(acc[t][u], wa[w] & LO, wb[w] & LO, wa[w] & HI, wb[w] & HI, qf[t][n][w][0], qf[t][n][w][1]);
                  mma_f16(acc[t][u], xa & LO, xb & LO, xa & HI, xb & HI, qf[t][n][w][2], qf[t][n][w][3]);
                }
              }
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float2 p = kv4_pair(*reinterpret_cast<const uint32_t*>(sk + F::CODES + ((ka + 8 * x) * NG + n) * 4));
              const uint64_t d2 = f2_pack(p.x, p.x), lo2 = f2_pack(p.y, p.y);
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                const uint64_t ac = f2_pack(acc[t][x / 2][2 * (x & 1)], acc[t][x / 2][2 * (x & 1) + 1]), q2 = f2_pack(qs[t][n][0], qs[t][n][1]);
                dn[t][x] = n == 0 ? f2_mul(d2, ac) : f2_fma(d2, ac, dn[t][x]);
                lo[t][x] = n == 0 ? f2_mul(lo2, q2) : f2_fma(lo2, q2, lo[t][x]);
              }
            }
          }
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const uint64_t fa2 = f2_pack(fa[t][0], fa[t][1]), fb2 = f2_pack(fb, fb);
#pragma unroll
            for (int x = 0; x < 4; ++x) s2[t][x] = f2_fma(f2_mul(dn[t][x], fa2), fb2, lo[t][x]);
          }
        }
        uint32_t vp[4][NG];  // the pairs of V, of the same keys
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint8_t* at = sv + F::CODES + (ka + 8 * x) * NG * 4;
          if constexpr (NG == 2) *reinterpret_cast<uint2*>(vp[x]) = *reinterpret_cast<const uint2*>(at);
          else vp[x][0] = *reinterpret_cast<const uint32_t*>(at);
        }
        if (key0 + 31 > see0 || (key0 <= edge_to && key0 + 31 >= a.first)) {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int key = page0 + ka + 8 * x;
            const bool past = key >= a.first;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              float2 s = f2_unpack(s2[t][x]);
              if (key > see[t][0] || (past && key <= hidden_to(see[t][0], a.window))) s.x = -INFINITY;
              if (key > see[t][1] || (past && key <= hidden_to(see[t][1], a.window))) s.y = -INFINITY;
              s2[t][x] = f2_pack(s.x, s.y);
            }
            if (key > see_last || (past && key <= gone_to))  // nobody sees it: its pairs may be anything
#pragma unroll
              for (int n = 0; n < NG; ++n) vp[x][n] = 0;
          }
        }
        uint64_t p2[NT][4];
        uint32_t ph[NT][4][NG];  // p d of the two columns
        uint64_t psum[NT];
        // d of a pair, or 2^-64 |lo| (on the bits: a float's exponent less 64)
        auto step_of = [](uint32_t w) { return __uint_as_float((uint32_t)max(max((int)(w << 16), (int)(w & 0x7fff0000u) - (64 << 23)), 0)); };
        auto weigh = [&] {
          bool grow = false;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const uint64_t m2 = f2_pack(-m[t][0], -m[t][1]);
            uint32_t big = 0;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float2 e = f2_unpack(f2_add(s2[t][x], m2));
              const float2 p = make_float2(ex2_fast(e.x), ex2_fast(e.y));
              p2[t][x] = f2_pack(p.x, p.y);
#pragma unroll
              for (int n = 0; n < NG; ++n) {
                const float d = step_of(vp[x][n]);
                const float2 pd = f2_unpack(f2_mul(p2[t][x], f2_pack(d, d)));
                ph[t][x][n] = pack_f16(pd.x, pd.y);
                big |= ph[t][x][n] + 0x08000800u;  // the sign bit of a half from 2^15 on, infinities and NaN too
              }
            }
            const uint64_t sum2 = f2_add(f2_add(p2[t][0], p2[t][1]), f2_add(p2[t][2], p2[t][3]));
            const float2 sum = f2_unpack(sum2);
            grow |= (big & 0x80008000u) != 0 || !(fmaxf(sum.x, sum.y) <= 0x1p80f);
            psum[t] = sum2;
          }
          return __any_sync(0xffffffffu, grow);
        };
        if (weigh()) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float top = NONE;
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                float d = fmaxf(step_of(vp[x][0]), 0x1p-60f);
                if constexpr (NG == 2) d = fmaxf(d, step_of(vp[x][1]));
                const float2 s = f2_unpack(s2[t][x]);
                top = fmaxf(top, (j ? s.y : s.x) + (log2f(d) - 8.f));
              }
#pragma unroll
              for (int w = 4; w < 32; w *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
              if (top > m[t][j]) {
                const float f = ex2_fast(m[t][j] - top);
                m[t][j] = top;
                l[t][j] *= f;
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                  ol[t][n][j] *= f;
#pragma unroll
                  for (int i = 0; i < MT; ++i) {
                    o[t][n][i][j] *= f;
                    o[t][n][i][2 + j] *= f;
                  }
                }
              }
            }
          weigh();
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float2 ls = f2_unpack(f2_add(f2_pack(l[t][0], l[t][1]), psum[t]));
          l[t][0] = ls.x, l[t][1] = ls.y;
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            uint64_t o2 = f2_pack(ol[t][n][0], ol[t][n][1]);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float lo = kv4_pair(vp[x][n]).y;
              o2 = f2_fma(p2[t][x], f2_pack(lo, lo), o2);
              ph[t][x][n] = transpose_8x8(ph[t][x][n]);
            }
            const float2 os = f2_unpack(o2);
            ol[t][n][0] = os.x, ol[t][n][1] = os.y;
          }
        }
        // V: dims 8 g .. 8 g + 7 of a group (head_dim 32: 4 g .. 4 g + 3)
#pragma unroll
        for (int n = 0; n < NG; ++n) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            uint32_t w[4];
            const int at[4] = {va, vb, va + 8, vb + 8};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint8_t* q = sv + (at[i] + 16 * u) * (HD / 2) + n * 32 + g * (F::GS / 16);
              if constexpr (F::GS == 64) w[i] = *reinterpret_cast<const uint32_t*>(q);
              else w[i] = *reinterpret_cast<const uint16_t*>(q);
            }
#pragma unroll
            for (int h = 0; h < MT / 2; ++h) {
              const uint32_t sel = h ? 0x7632u : 0x5410u;
              const uint32_t x = __byte_perm(w[0], w[1], sel), y = __byte_perm(w[2], w[3], sel), x8 = x >> 8, y8 = y >> 8;
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                mma_f16(o[t][n][2 * h], x & LO, x & HI, y & LO, y & HI, ph[t][2 * u][n], ph[t][2 * u + 1][n]);
                mma_f16(o[t][n][2 * h + 1], x8 & LO, x8 & HI, y8 & LO, y8 & HI, ph[t][2 * u][n], ph[t][2 * u + 1][n]);
              }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }

    // the warps' parts: each to the item's maximum, the upper half's added to the lower's, then all
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int w = 4; w < 32; w *= 2) {
          l[t][j] += __shfl_xor_sync(0xffffffffu, l[t][j], w);
#pragma unroll
          for (int n = 0; n < NG; ++n) ol[t][n][j] += __shfl_xor_sync(0xffffffffu, ol[t][n][j], w);
        }
        // (M goes up by the power of two in l where that is positive: parts whose values differ by more than 2^126 meet at one M)
        float2 ml = make_float2(m[t][j], l[t][j]);
        if (ml.y > 0x1p20f) {
          ml.x += (float)((int)(__float_as_uint(ml.y) >> 23) - 127);
          ml.y *= ex2_fast(m[t][j] - ml.x);
        }
        if (g == 0) s_ml[warp * RT + t * 8 + 2 * cl + j] = ml;
      }
    bar_named(1, 32 * Sh::WARPS);
    auto row_max = [&](int r) {
      float mm = NONE;
#pragma unroll
      for (int w = 0; w < Sh::WARPS; ++w) mm = fmaxf(mm, s_ml[w * RT + r].x);
      return mm;
    };
    auto put = [&](bool add) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float f = ex2_fast(m[t][j] - row_max(t * 8 + 2 * cl + j));
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            float* to = s_o + (warp % Sh::TEAMS * RT + t * 8 + 2 * cl + j) * OS + n * F::GS + g * (2 * MT);
#pragma unroll
            for (int i = 0; i < MT; i += 2) {  // dims in pairs: 2^24 n, and 2^24 16 n
              float4 v = make_float4(o[t][n][i][j] * 0x1p24f, o[t][n][i][2 + j] * 0x1p20f, o[t][n][i + 1][j] * 0x1p24f, o[t][n][i + 1][2 + j] * 0x1p20f);
              v.x = (v.x + ol[t][n][j]) * f, v.y = (v.y + ol[t][n][j]) * f, v.z = (v.z + ol[t][n][j]) * f, v.w = (v.w + ol[t][n][j]) * f;
              float4* at = reinterpret_cast<float4*>(to + 2 * i);
              if (add) {
                const float4 u = *at;
                v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
              }
              *at = v;
            }
          }
        }
    };
    if (warp >= Sh::TEAMS) put(false);
    bar_named(1, 32 * Sh::WARPS);
    if (warp < Sh::TEAMS) put(true);
    bar_named(1, 32 * Sh::WARPS);
    const bool whole = it.kb0 == 0 && it.kb1 == it.nb;
    const size_t part = (size_t)(2 * blockIdx.x + (it.kb0 == 0)) * a.rows;
    for (int i = tid; i < rows * (HD / 4); i += 32 * Sh::WARPS) {
      const int r = i / (HD / 4), d = (i % (HD / 4)) * 4;
      float4 v = *reinterpret_cast<const float4*>(s_o + r * OS + d);
#pragma unroll
      for (int x = 1; x < Sh::TEAMS; ++x) {
        const float4 u = *reinterpret_cast<const float4*>(s_o + (x * RT + r) * OS + d);
        v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
      }
      const float mm = row_max(r);
      float ll = 0.f;
#pragma unroll
      for (int x = 0; x < Sh::WARPS; ++x) {
        const float2 ml = s_ml[x * RT + r];
        ll += ml.y * ex2_fast(ml.x - mm);
      }
      if (whole) {
        const long long token = it.token0 + r / G;
        const int head = it.h * G + r % G;
        const float inv = ll != 0.f ? 1.f / ll : 0.f;
        bf16* out = static_cast<bf16*>(a.out) + token * a.os + (long long)head * HD + d;
        const uint32_t lo = pack_bf16(v.x * inv, v.y * inv), hi = pack_bf16(v.z * inv, v.w * inv);
        if (reinterpret_cast<uintptr_t>(out) % 8 == 0) {
          *reinterpret_cast<uint2*>(out) = make_uint2(lo, hi);
        } else {
          const uint32_t w2[2] = {lo, hi};
#pragma unroll
          for (int x = 0; x < 4; ++x) out[x] = __ushort_as_bfloat16((unsigned short)(w2[x / 2] >> (16 * (x & 1))));
        }
        if (d == 0 && a.lse) a.lse[token * c.Hq + head] = ll != 0.f ? (mm + log2f(ll)) * LN2 : -INFINITY;
      } else {
        *reinterpret_cast<float4*>(a.part_o + (part + r) * HD + d) = v;
        if (d == 0) a.part_ml[part + r] = make_float2(ll != 0.f ? mm : -INFINITY, ll);
      }
    }
    bar_named(1, 32 * Sh::WARPS);  // the buffers and the item's words are read
    if (tid == 0) mbar_arrive(seg_empty(segs));
  }
}

// ----------------------------------------------------------------------------
// Many rows: tcgen05 (head_dim 64 and 128)
// ----------------------------------------------------------------------------
// Items, roles and tensor memory are k_chunk_pair's (k_chunk.cu): two tiles of 128 MMA rows, blocks of 64 keys, softmax with a thread a
// row, an issuing warp a tile. What is different is where K and V come from: the producer copies a page's two blocks of codes, and four
// warps (12-15) turn them into float16 tiles. With K' = d (n - 8), which is exact in float16 (8 bits times 3, or a power of two), scores
// are exact but for float32's sums:
//   q . k = sum q K' + sum over groups g of (lo_g + 8 d_g) (sum of q)_g
// the second part as 16 more columns of the product: lo_0, lo_1, 8 d_0, 8 d_1 in K, three times beside the sums of q in three float16
// that hold 33 bits (12 columns with two groups; the last four are zeros). V' = lo + d n is rounded to float16, and so is P. Codes
// become numbers in one multiply-add a pair: the bits n (or 16 n) of a masked word are the float16 n 2^-24. A word's eight values come
// out in the order 0 4 1 5 2 6 3 7; q is put into that order, O is read out of it.
//
// Ranges: K of a block is divided by a power of two (the largest of |lo| and 16 d of the entries that some query sees gets into 2^-6 ..
// 2^-5: what an entry has below 2^-18 of that is rounded), q of a row multiplied by one (2^8 .. 2^9); the softmax undoes both. V is
// divided by 2^(e + 6), which goes into the score: M + 6 is the largest s_t + e, O = sum 2^(s_t + e - M) V_t / 2^(e + 6),
// l = sum 2^(s_t + e - M) 2^-e, so that what has to be held in 16 bits is relative to the row's largest term. e is the block's, by its
// largest entry; in a block with entries smaller than 2^-6 of that (as the first tokens' values may be, which take most of the
// probability), or with none above 2^-40, every entry has its own, e_t, by 2^-e_t in shared memory, and l adds up 2^(s_t - M) where
// the term of O is too small for float32 (own_block, which is slow: all blocks by it take 1310 us where it is 448).
// e is at least -88, so that 2^14 2^88 times 2^26 entries of a part stay in float32, as 64 / l does with values of 2^126. Where values of
// a row's blocks lie further than 2^100 apart, the weights of the small ones are lost.
//
// Bound by the softmax warps' chain, as k_chunk_pair is, which the codes' warps make longer: their instructions and accesses of
// shared memory meet its own and the MMAs' reads. A block of 64 keys and two tiles takes 2240 cycles at head_dim 128, of which the
// tensor pipe works half. 4 x 2048 tokens over up to 10240 entries, 16 / 8 heads x 128: 448 us with the join, 1090 TFLOP/s (395 with
// nothing converted, k_chunk_pair over bfloat16 371); 16 heads x 64: 398 us. Tried and slower: other splits of the registers (168 / 80,
// 152 / 96), waits that sleep, the softmax's two halves in a loop (492).
constexpr int PAIR4_THREADS = 512;
template <int HD>
struct Pair4Shape {
  using F = Kv4<HD>;
  static constexpr int ATOMS = HD / 64, QCOL = 128 * 128, Q_BYTES = ATOMS * QCOL;  // a tile of 128 rows of q
  static constexpr int COL = 64 * 128, T_BYTES = ATOMS * COL;                      // 64 rows of K or V
  static constexpr int QX = 128 * 32, KX = 64 * 32, RAW = 2 * F::BLOCK;            // the 16 more columns; a page's codes and pairs
  static constexpr int NST = HD == 128 ? 3 : 4, NRAW = HD == 128 ? 4 : 6;
  static constexpr int OFF_K = 2 * Q_BYTES, OFF_V = OFF_K + NST * T_BYTES, OFF_QX = OFF_V + NST * T_BYTES, OFF_KX = OFF_QX + 2 * QX,
                       OFF_RAW = OFF_KX + NST * KX, OFF_BAR = OFF_RAW + NRAW * RAW;
  static constexpr int NBAR = 4 * NST + 3 * NRAW + 2 + 2 + 4 + 4 + 4 + 1 + 2 * PairSeg::RING;
  static constexpr int FLAGS = 16;  // more than the blocks that the producer can be ahead of the softmax
  static constexpr int WS = 8;      // .. that the codes' warps can
  static constexpr int OFF_INT = OFF_BAR + NBAR * 8, OFF_INFO = (OFF_INT + (FLAGS + 4) * 4 + 15) / 16 * 16,
                       OFF_W = OFF_INFO + FLAGS * 16, OFF_SEG = OFF_W + WS * 64 * 4;
  static constexpr int OFF_BASE = OFF_SEG + PairSeg::RING * (int)sizeof(PairSeg);
  static int bytes(int n) { return std::max(OFF_BASE + (n + 1) * 8 + 1024, tmem_min_smem(512)); }
  static constexpr uint32_t OCOL = 256;
};
// Instruction descriptor: kind::f16, A = B = float16, D = float32, both K-major.
constexpr uint32_t idesc_f16_f32(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }
// Descriptor of a K-major tile of 16 columns: rows of 32 bytes, swizzled in atoms of 8 rows (the halves of rows 4-7 change places).
__device__ __forceinline__ uint64_t smem_desc_x(uint32_t saddr) {
  return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)1u << 16 | (uint64_t)(256u >> 4) << 32 | (uint64_t)1u << 46 | (uint64_t)6u << 61;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(max(-126, min(127, e)) + 127) << 23); }
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ uint32_t twice_f16(float x) { return pack_f16(x, x); }
__device__ __forceinline__ void st_shared_16(uint32_t at, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Eight values of a word, x -> n d + c (d24, d20: d times 2^24 and 2^20), in the order 0 4 1 5 2 6 3 7.
__device__ __forceinline__ uint4 f16_values(uint32_t w, uint32_t d24, uint32_t d20, uint32_t c) {
  const uint32_t x = w >> 8;
  return make_uint4(fma_f16x2(w & 0x000f000fu, d24, c), fma_f16x2(w & 0x00f000f0u, d20, c), fma_f16x2(x & 0x000f000fu, d24, c),
                    fma_f16x2(x & 0x00f000f0u, d20, c));
}

// Values that an asynchronous load has put into registers: no use of them moves up past this point.
__device__ __forceinline__ void hold_32(uint32_t* r) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
}

__device__ __forceinline__ void tmem_put_8(uint32_t taddr, const uint32_t* r) {  // completes at the next wait::st
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// The softmax of a block whose entries have powers of V of their own, a row a thread: P into tensor memory, O rescaled if the row's
// maximum grows (once the P V before has landed), l from the entries' powers; also of blocks whose scores may be so large that their
// differences to the maximum have to be exact. False: a wait ran out. Not inlined: a second body of the softmax in the kernel, or a branch in the one, cost 15 to 30 us of 450 where no block has any.
struct OwnBlock {
  uint32_t t_s, t_o;
  float scale;
  uint64_t seen;     // columns that the row sees
  const float* w;    // 2^-e_t; NULL: that of the block, w0
  float w0;
  uint32_t o_done;   // barrier of the P V before, with its parity; 0: there is none
  uint32_t parity;
  volatile int* abort_flag;
  uint32_t* werr;
  float m, l;
};
template <int HD>
__device__ __noinline__ bool own_block(OwnBlock& b) {
  const uint32_t t_s = b.t_s;
  const float scale = b.scale, w0 = b.w0;
  const float4* w4 = reinterpret_cast<const float4*>(b.w);
  float pm = -INFINITY, s[16];
  auto weights = [&](int k, float (&w)[4]) {  // 2^-e_t of entries k .. k + 3
    const float4 v = w4 ? w4[k / 4] : make_float4(w0, w0, w0, w0);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  };
  // e_t: 127 less the exponent's bits, which 2^23 takes in as they are
  auto power = [](float w) { return (0x1p23f + 127.f) - __uint_as_float(0x4b000000u | __float_as_uint(w) >> 23); };
#pragma unroll 1
  for (int c0 = 0; c0 < 64; c0 += 16) {
    const uint32_t seen = (uint32_t)(b.seen >> c0);
    tmem_ld_16(t_s + c0, s);
#pragma unroll
    for (int k = 0; k < 16; k += 4) {
      float w[4];
      weights(c0 + k, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) pm = fmaxf(pm, seen >> (k + j) & 1 ? fmaf(s[k + j], scale, power(w[j])) : -INFINITY);
    }
  }
  const bool grow = pm - b.m > 14.f;
  if (__any_sync(0xffffffffu, grow)) {
    const float m_new = pm - 6.f, cr = grow ? exp2f(b.m - m_new) : 1.f;
    if (b.o_done) {
      bool ok = *b.abort_flag == 0 && mbar_wait(b.o_done, b.parity, b.werr);
      if (!__all_sync(0xffffffffu, ok)) {
        *b.abort_flag = 1;
        return false;
      }
      tc_fence_after();
#pragma unroll 1
      for (int c0 = 0; c0 < HD; c0 += 16) {
        tmem_ld_16(b.t_o + c0, s);
#pragma unroll
        for (int k = 0; k < 16; ++k) s[k] *= cr;
        tmem_st_16(b.t_o + c0, s);
      }
    }
    if (grow) {
      b.l *= cr;
      b.m = m_new;
    }
  }
  const float mref = b.m == -INFINITY ? 0.f : b.m;
  float l = b.l;
#pragma unroll 1
  for (int c0 = 0; c0 < 64; c0 += 16) {
    const uint32_t seen = (uint32_t)(b.seen >> c0);
    uint32_t pk[8];
    float p[16];
    bool none = false;  // a term of O too small for float32
    tmem_ld_16(t_s + c0, s);
#pragma unroll
    for (int k = 0; k < 16; k += 4) {
      float w[4];
      weights(c0 + k, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        p[k + j] = seen >> (k + j) & 1 ? ex2_fast(fmaf(s[k + j], scale, power(w[j])) - mref) : 0.f;
        l = fmaf(p[k + j], w[j], l);
        none |= p[k + j] == 0.f && (seen >> (k + j) & 1);
      }
    }
    if (__any_sync(0xffffffffu, none)) {
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (p[k] == 0.f && (seen >> k & 1)) l += ex2_fast(fmaf(s[k], scale, -mref));
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) pk[k] = pack_f16(p[2 * k], p[2 * k + 1]);
    tmem_put_8(t_s + c0 / 2, pk);  // (over scores that have been read)
    tmem_st_wait_done();
  }
  b.l = l;
  return true;
}

template <int HD>
__global__ void __launch_bounds__(PAIR4_THREADS, 1) k_chunk_pair4(ChunkAttn a, int g_log, const __grid_constant__ CUtensorMap q_map) {
  using Sh = Pair4Shape<HD>;
  using F = Kv4<HD>;
  constexpr int NST = Sh::NST, NRAW = Sh::NRAW, NG = F::NG;
  extern __shared__ uint8_t smem_raw[];
  __shared__ long long s_red[33];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + Sh::OFF_BAR);
  volatile int* s_flag = reinterpret_cast<volatile int*>(sm + Sh::OFF_INT);  // the block's page is not there
  volatile int* abort_flag = s_flag + Sh::FLAGS;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + Sh::OFF_INT) + Sh::FLAGS + 1;
  // of a block: the power of two that its raw scores are to be multiplied by (beside the scale and the row's power), e, 2^-e, and bits:
  // 1 the page is not there, 2 entries have powers of their own
  float4* s_info = reinterpret_cast<float4*>(sm + Sh::OFF_INFO);
  float* s_w = reinterpret_cast<float*>(sm + Sh::OFF_W);  // [WS][64] 2^-e_t
  PairSeg* s_seg = reinterpret_cast<PairSeg*>(sm + Sh::OFF_SEG);
  long long* s_base = reinterpret_cast<long long*>(sm + Sh::OFF_BASE);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  // block b of this CTA: its place in the rings, and the use's parity
  auto k_full = [&](unsigned b) { return bar(b % NST); };
  auto k_empty = [&](unsigned b) { return bar(NST + b % NST); };
  auto v_full = [&](unsigned b) { return bar(2 * NST + b % NST); };
  auto v_empty = [&](unsigned b) { return bar(3 * NST + b % NST); };
  auto raw_full = [&](unsigned b) { return bar(4 * NST + b % NRAW); };
  auto raw_empty = [&](unsigned b) { return bar(4 * NST + NRAW + b % NRAW); };
  auto c_full = [&](unsigned b) { return bar(4 * NST + 2 * NRAW + b % NRAW); };
  constexpr int B0 = 4 * NST + 3 * NRAW;
  auto q_full = [&](int x) { return bar(B0 + x); };
  auto q_ready = [&](int x) { return bar(B0 + 2 + x); };
  // block n of tile x, as in k_chunk_pair: S written, P written, P V done
  auto s_full = [&](int x, unsigned n) { return bar(B0 + 4 + 2 * x + (n & 1)); };
  auto p_full = [&](int x, unsigned n) { return bar(B0 + 8 + 2 * x + (n & 1)); };
  auto o_done = [&](int x, unsigned n) { return bar(B0 + 12 + 2 * x + (n & 1)); };
  const uint32_t q_free = bar(B0 + 16);
  auto seg_full = [&](unsigned i) { return bar(B0 + 17 + i % PairSeg::RING); };
  auto seg_empty = [&](unsigned i) { return bar(B0 + 17 + PairSeg::RING + i % PairSeg::RING); };
  const ChunkDev& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(k_full(i), 3);
      mbar_init(k_empty(i), 2);
      mbar_init(v_full(i), 2);
      mbar_init(v_empty(i), 2);
    }
    for (int i = 0; i < NRAW; ++i) {
      mbar_init(raw_full(i), 1);
      mbar_init(raw_empty(i), 5);
      mbar_init(c_full(i), 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(q_full(x), 1);
      mbar_init(q_ready(x), 4);
      for (unsigned n = 0; n < 2; ++n) {
        mbar_init(s_full(x, n), 1);
        mbar_init(p_full(x, n), 4);
        mbar_init(o_done(x, n), 1);
      }
    }
    mbar_init(q_free, 2);
    for (unsigned i = 0; i < PairSeg::RING; ++i) {
      mbar_init(seg_full(i), 1);
      mbar_init(seg_empty(i), 15);  // the other warps
    }
    *abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&q_map);
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  pdl_wait();
  const WindowSplit sp = split_of<KEYS_4BIT>(a);
  const int sinks = sp.sinks();
  chunk_plan(c, sp, s_base, s_red);
  tc_fence_before();
  __syncthreads();  // barriers initialised, tensor memory allocated
  tc_fence_after();
  pdl_trigger();  // not before: a dependent CTA on this SM could take the columns that warp 9 still waits for
  const uint32_t tmem = *tmem_slot;
  const long long all = s_base[c.n], per = chunk_share(a, all);
  long long pos = blockIdx.x * per;
  const long long end = pos + per < all ? pos + per : all;
  const int qt_log = a.sp.qt_log, QT = 1 << (qt_log - 1);  // queries of a tile
  // a bounded wait; once any role has given up, the others skip their waits and wind down
  auto wait = [&](uint32_t b, uint32_t parity) {
    if (mbar_try_wait(b, parity & 1u)) return true;
    if (*abort_flag) return false;
    if (mbar_wait(b, parity & 1u, a.werr)) return true;
    *abort_flag = 1;
    return false;
  };
  // waits taken by the whole warp
  auto wait_w = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, wait(b, parity)); };
  PairSeg s;
  unsigned segs = 0;  // read or published

  // registers of the launch: 512 x 128 = 65536; shares: 256 x 160 + 256 x 88 = 63488
  if (warp >= 8) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
  if (warp == 8) {
    // ---------------- producer ----------------
    unsigned blk = 0;
    for (bool ok = true;;) {
      s.nb = 0;
      ChunkItem it{};
      if (pos < end) {
        it = chunk_item(c, sp, s_base, pos);
        if (segs == 0 && lane == 0) join_note(a, &it, per);
        if (pos < it.first) pos = it.first;
      } else if (segs == 0 && lane == 0) {
        join_note(a, nullptr, per);
      }
      if (pos < end) {
        const int q0 = it.t << qt_log, left = it.ql - q0;
        s = PairSeg{it.b, it.h, it.t0 + q0, it.s0 + q0, {}, {}, (int)(pos - it.first), (int)(end - it.first < it.nb ? end - it.first : it.nb), it.nb, 0};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          s.nq[x] = max(0, min(QT, left - x * QT));
          const int last = s.see0 + x * QT + s.nq[x] - 1;  // entry of the tile's last query
          const int nb = s.nq[x] > 0 ? (last < 0 ? 1 : last / 64 + 1 - it.skip) : 0;
          s.e[x] = max(0, min(s.kb1, nb) - s.kb0);
        }
        pos = it.first + s.kb1;
      }
      if (lane == 0) {
        ok = ok && (segs < PairSeg::RING || wait(seg_empty(segs), segs / PairSeg::RING - 1));
        if (ok) {
          s_seg[segs % PairSeg::RING] = s;
          mbar_arrive(seg_full(segs));
        }
      }
      if (s.nb == 0) break;
      const int E = s.kb1 - s.kb0;
      if (lane == 0) {
        ok = ok && (segs == 0 || wait(q_free, segs - 1));
        for (int x = 0; x < 2; ++x) {
          if (!ok || s.e[x] == 0) continue;
          mbar_arrive_expect_tx(q_full(x), Sh::Q_BYTES);
#pragma unroll
          for (int k = 0; k < Sh::ATOMS; ++k)
            tma_load_3d(smem_u32(sm + x * Sh::Q_BYTES + k * Sh::QCOL), &q_map, k * 64, s.h << g_log, s.token0 + x * QT, q_full(x));
        }
      }
      const long long k_at = ((long long)c.layer * 2 * c.Hkv + s.h) * F::BLOCK, v_at = k_at + (long long)c.Hkv * F::BLOCK;
      for (int g0 = 0; g0 < E; g0 += 32) {
        int mine = -1;  // the pages of 32 blocks, one a lane
        const int at = block_at<KEYS_4BIT>(s.kb0 + g0 + lane, sinks, it.skip);
        if (g0 + lane < E && at * 64 < it.len) mine = chunk_page(c.page_table, c.max_pages, c.n_pages, s.b, at, c.err);
        for (int i = 0; i < min(32, E - g0); ++i, ++blk) {
          const int page = __shfl_sync(0xffffffffu, mine, i);
          if (lane == 0 && ok) {
            ok = blk < NRAW || wait(raw_empty(blk), blk / NRAW - 1);
            if (ok) {
              s_flag[blk % Sh::FLAGS] = page < 0;
              if (page < 0) {
                mbar_arrive(raw_full(blk));
              } else {
                mbar_arrive_expect_tx(raw_full(blk), Sh::RAW);
                const uint8_t* src = static_cast<const uint8_t*>(c.pool) + page * c.page_elems;
                const uint32_t dst = smem_u32(sm + Sh::OFF_RAW + (blk % NRAW) * Sh::RAW);
                bulk_g2s(dst, src + k_at, F::BLOCK, raw_full(blk));
                bulk_g2s(dst + F::BLOCK, src + v_at, F::BLOCK, raw_full(blk));
              }
            }
          }
          __syncwarp();
        }
      }
      ++segs;
    }
  } else if (warp == 11) {
    // ---------------- pairs to what the codes' warps need ----------------
    // The block's powers of two, and in the place of each pair (d, lo) two float16: 2^24 d' and 8 d' for K, 2^24 d' and lo' for V. A
    // lane has keys 2 lane and 2 lane + 1.
    unsigned b = 0;
    for (bool ok = true; ok && wait_w(seg_full(segs), segs / PairSeg::RING); ++segs) {
      s = s_seg[segs % PairSeg::RING];
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(segs));
      if (s.nb == 0) break;
      // no query sees entries from `behind` on, nor, under a window, those from `first` up to gone_to: what they hold is not looked at
      const int behind = s.see0 + s.nq[0] + s.nq[1], skip = sp.skip_at(s.see0), gone_to = hidden_to(s.see0, a.window);
      for (int i = s.kb0; i < s.kb1; ++i, ++b) {
        const int page0 = block_at<KEYS_4BIT>(i, sinks, skip) * 64;
        if (!wait_w(raw_full(b), b / NRAW)) { ok = false; break; }
        uint8_t* raw = sm + Sh::OFF_RAW + (b % NRAW) * Sh::RAW + F::CODES + lane * (8 * NG);
        uint32_t pr[2][2 * NG];  // of K and V; key, group
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if constexpr (NG == 2) *reinterpret_cast<uint4*>(pr[x]) = *reinterpret_cast<const uint4*>(raw + x * F::BLOCK);
          else *reinterpret_cast<uint2*>(pr[x]) = *reinterpret_cast<const uint2*>(raw + x * F::BLOCK);
        }
        const bool gone = s_flag[b % Sh::FLAGS] != 0;
        bool hides[2] = {false, false};
        if (gone || page0 + 63 >= behind || (page0 <= gone_to && page0 + 63 >= a.first)) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int e = page0 + 2 * lane + k;
            hides[k] = gone || e >= behind || (e >= a.first && e <= gone_to);
            if (hides[k])
#pragma unroll
              for (int n = 0; n < NG; ++n) pr[0][k * NG + n] = pr[1][k * NG + n] = 0;
          }
        }
        // exponents, on the bits of |lo| and 16 d (0 stays small: 2^-123): halves of a word
        auto sizes = [](uint32_t w) { return (w & 0x7fff7fffu) + 0x00000200u; };
        auto larger = [&](const uint32_t* p) { return NG == 2 ? __vmaxu2(sizes(p[0]), sizes(p[NG - 1])) : sizes(p[0]); };
        auto exponent = [](uint32_t w, int low) { return max(low, min(126, (int)(max(w & 0xffffu, w >> 16) >> 7) - 127)); };
        uint32_t own_size[2];
        int e[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          own_size[0] = larger(pr[x]);
          own_size[1] = larger(pr[x] + NG);
          const uint32_t v = __vmaxu2(own_size[0], own_size[1]);
          e[x] = exponent(__reduce_max_sync(0xffffffffu, max(v & 0xffffu, v >> 16)), x == 0 ? -118 : -88);
        }
        // does an entry that somebody sees lie below 2^-6 of the largest?
        const bool small = (!hides[0] && exponent(own_size[0], -88) < e[1] - 6) || (!hides[1] && exponent(own_size[1], -88) < e[1] - 6);
        const bool own = e[1] < -40 || __any_sync(0xffffffffu, small);
        uint32_t lo16[2] = {0, 0}, d16[2] = {0, 0};  // of K, for the 16 more columns
        int et[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (x == 1) et[k] = own && !hides[k] ? exponent(own_size[k], -88) : e[1];
            const int by = (x == 0 ? e[0] : et[k]) + 6;
            const float f = pow2(-by), more = by > 126 ? pow2(126 - by) : 1.f;
#pragma unroll
            for (int n = 0; n < NG; ++n) {
              float2 p = kv4_pair(pr[x][k * NG + n]);
              p.x = p.x * f * more;
              p.y = p.y * f * more;
              pr[x][k * NG + n] = pack_f16(p.x * 0x1p24f, x == 0 ? 8.f * p.x : p.y);
              if (x == 0) {
                const uint32_t both = pack_f16(p.y, 8.f * p.x);
                lo16[k] |= (both & 0xffffu) << (16 * n);
                d16[k] |= (both >> 16) << (16 * n);
              }
            }
          }
          if constexpr (NG == 2) *reinterpret_cast<uint4*>(raw + x * F::BLOCK) = *reinterpret_cast<const uint4*>(pr[x]);
          else *reinterpret_cast<uint2*>(raw + x * F::BLOCK) = *reinterpret_cast<const uint2*>(pr[x]);
        }
        fence_proxy_async_smem();  // (the next copy into this place comes after)
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(c_full(b));
          mbar_arrive(raw_empty(b));
        }
        if (b >= NST && !wait_w(k_empty(b), b / NST - 1)) { ok = false; break; }
        // lo, 8 d of the groups, three times
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int key = 2 * lane + k;
          uint8_t* to = sm + Sh::OFF_KX + (b % NST) * Sh::KX + key * 32;
          const int flip = ((key >> 2) & 1) << 4;
          *reinterpret_cast<uint4*>(to + flip) = make_uint4(lo16[k], d16[k], lo16[k], d16[k]);
          *reinterpret_cast<uint4*>(to + (flip ^ 16)) = make_uint4(lo16[k], d16[k], 0, 0);
          // (what the softmax reads with S: the issuer has seen k_full before it)
          if (own) s_w[(b % Sh::WS) * 64 + key] = pow2(-et[k]);
        }
        if (lane == 0)
          s_info[b % Sh::FLAGS] = make_float4(__int_as_float(e[0] + 6), (float)e[1], pow2(-e[1]), __int_as_float((gone ? 1 : 0) | (own ? 2 : 0)));
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(k_full(b));
      }
    }
  } else if (warp >= 12) {
    // ---------------- codes to float16 tiles ----------------
    // Warps 12 and 13 make K's, 14 and 15 V's; neither waits for the other's places. A warp has 32 of the keys; a lane two of them and
    // every other 16 bytes of their codes (8 lanes: 4 keys x 2: their writes meet no bank twice).
    const int kv = (warp - 12) >> 1, odd = lane & 1, key0 = (warp & 1) * 32 + (lane >> 3) * 4 + ((lane >> 1) & 3);  // and key0 + 16
    const uint32_t stage0 = smem_u32(sm) + (kv == 0 ? Sh::OFF_K : Sh::OFF_V) + key0 * 128, sign = kv == 0 ? 0x80008000u : 0u;
    uint32_t to[4];  // the lane's 16-byte places in a row: key0 and key0 + 16 have the same
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = stage0 + (((odd * 4 + i) ^ (key0 & 7)) << 4);
    const uint8_t* from = sm + Sh::OFF_RAW + kv * F::BLOCK;
    unsigned b = 0;
    for (bool ok = true; ok && wait_w(seg_full(segs), segs / PairSeg::RING); ++segs) {
      const int kb0 = s_seg[segs % PairSeg::RING].kb0, kb1 = s_seg[segs % PairSeg::RING].kb1, nb = s_seg[segs % PairSeg::RING].nb;
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(segs));
      if (nb == 0) break;
      for (int i = kb0; i < kb1; ++i, ++b) {
        if (!wait_w(raw_full(b), b / NRAW)) { ok = false; break; }
        const uint8_t* raw = from + (b % NRAW) * Sh::RAW;
        uint4 code[2][NG];
        uint32_t pair[2][NG];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int n = 0; n < NG; ++n) code[x][n] = *reinterpret_cast<const uint4*>(raw + (key0 + 16 * x) * (HD / 2) + n * 32 + odd * 16);
        if (!wait_w(c_full(b), b / NRAW)) { ok = false; break; }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int n = 0; n < NG; ++n) pair[x][n] = *reinterpret_cast<const uint32_t*>(raw + F::CODES + ((key0 + 16 * x) * NG + n) * 4);
        __syncwarp();
        if (lane == 0) mbar_arrive(raw_empty(b));
        if (b >= NST && !wait_w(kv == 0 ? k_empty(b) : v_empty(b), b / NST - 1)) { ok = false; break; }
        const uint32_t st = (b % NST) * Sh::T_BYTES;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            const uint32_t d24 = __byte_perm(pair[x][n], 0, 0x1010), add = __byte_perm(pair[x][n], 0, 0x3232) ^ sign;
            const uint32_t d20 = fma_f16x2(d24, 0x2c002c00u, 0), w[4] = {code[x][n].x, code[x][n].y, code[x][n].z, code[x][n].w};  // (a sixteenth)
#pragma unroll
            for (int j = 0; j < 4; ++j) st_shared_16(to[j] + st + n * Sh::COL + x * 2048, f16_values(w[j], d24, d20, add));
          }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(kv == 0 ? k_full(b) : v_full(b));
      }
    }
  } else if (warp == 9 || warp == 10) {
    // ---------------- MMA issuers, one a tile ----------------
    if (elect_one()) {
      constexpr uint32_t IDS = idesc_f16_f32(128, 64), IDO = idesc_f16_f32(128, HD) | (1u << 16);  // (V MN-major)
      constexpr uint64_t QCOL_E = Sh::QCOL >> 4, T_E = Sh::T_BYTES >> 4, COL_E = Sh::COL >> 4, V16_E = 2048 >> 4, KX_E = Sh::KX >> 4;
      const int x = warp - 9;
      const uint64_t qd = smem_desc_sw128(smem_u32(sm + x * Sh::Q_BYTES)), dk = smem_desc_sw128(smem_u32(sm + Sh::OFF_K));
      const uint64_t dv = smem_desc_sw128_mn(smem_u32(sm + Sh::OFF_V), Sh::COL);
      const uint64_t qx = smem_desc_x(smem_u32(sm + Sh::OFF_QX + x * Sh::QX)), dkx = smem_desc_x(smem_u32(sm + Sh::OFF_KX));
      const uint32_t t_s = tmem + 128u * x, t_o = tmem + Sh::OCOL + (uint32_t)(HD * x);
      unsigned blk = 0, qn = 0, n = 0;  // n: blocks of the tile whose P V has been issued
      auto issue_s = [&](unsigned b, unsigned n) {
        const uint64_t kd = dk + (uint64_t)(b % NST) * T_E;
#pragma unroll
        for (int kc = 0; kc < Sh::ATOMS; ++kc)
#pragma unroll
          for (int k = 0; k < 4; ++k)  // K = 16 an MMA: +32 bytes (encoded +2) inside the atom column
            tc_mma_f16(t_s + 64u * (n & 1), qd + kc * QCOL_E + 2 * k, kd + kc * COL_E + 2 * k, IDS, (kc | k) ? 1u : 0u);
        tc_mma_f16(t_s + 64u * (n & 1), qx, dkx + (uint64_t)(b % NST) * KX_E, IDS, 1u);
        tc_commit(s_full(x, n));
      };
      bool ok = true;
      auto next = [&] {
        if (!wait(seg_full(segs), segs / PairSeg::RING)) return false;
        s = s_seg[segs % PairSeg::RING];
        mbar_arrive(seg_empty(segs));
        ++segs;
        return s.nb > 0;
      };
      while (ok && next()) {
        const int E = s.kb1 - s.kb0, e = x ? s.e[1] : s.e[0];
        ok = e == 0 || wait(q_ready(x), qn++);
        for (int i = 0; i < min(2, E) && ok; ++i) {  // S of the first two blocks
          ok = wait(k_full(blk + i), (blk + i) / NST);
          if (!ok) break;
          tc_fence_after();
          if (i < e) issue_s(blk + i, n + i);
          tc_commit(k_empty(blk + i));
        }
        if (ok && E <= 2) tc_commit(q_free);
        for (int i = 0; i < E && ok; ++i) {
          const unsigned b = blk + i;
          const bool more = i + 2 < E;
          // (what this tile does not use it waits for and releases all the same, in step with the other)
          ok = wait(v_full(b), b / NST) && (!more || wait(k_full(b + 2), (b + 2) / NST)) && (i >= e || wait(p_full(x, n), n >> 1));
          if (!ok) break;
          if (i < e) {
            tc_fence_after();
            const uint64_t vd = dv + (uint64_t)(b % NST) * T_E;
#pragma unroll
            for (int k = 0; k < 4; ++k)  // K = 16 keys an MMA: 8 columns of P, +2048 bytes (16 rows) of V
              mma_ts(t_o, t_s + 64u * (n & 1) + 8u * k, vd + V16_E * k, IDO, i > 0 || k > 0 ? 1u : 0u);
            tc_commit(o_done(x, n));
            if (i + 2 < e) issue_s(b + 2, n + 2);
            ++n;
          }
          tc_commit(v_empty(b));
          if (more) tc_commit(k_empty(b + 2));
          if (i + 3 == E) tc_commit(q_free);
        }
        blk += E;
      }
    }
    __syncwarp();
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    // ---------------- softmax: thread = MMA row = TMEM lane ----------------
    const int x = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_off = (uint32_t)(quad * 32) << 16;
    const uint32_t t_s = tmem + lane_off + 128u * (uint32_t)x;
    const uint32_t t_o = tmem + lane_off + Sh::OCOL + (uint32_t)(HD * x);
    const int qi = row >> g_log, g = row & ((1 << g_log) - 1);
    unsigned n = 0, blk = 0, qn = 0;  // blocks of this tile, and of the CTA; items of this tile
    const uint32_t scale_bits = __float_as_uint(a.scale < 0x1p-100f ? a.scale * 0x1p64f : a.scale), scale_frac = scale_bits & 0x7fffffu;
    const int scale_exp = (int)(scale_bits >> 23) - (a.scale < 0x1p-100f ? 64 : 0);
    bool ok = true;
    auto next = [&] {
      if (!wait_w(seg_full(segs), segs / PairSeg::RING)) return false;
      s = s_seg[segs % PairSeg::RING];
      __syncwarp();
      if (lane == 0) mbar_arrive(seg_empty(segs));
      ++segs;
      return s.nb > 0;
    };
    while (ok && next()) {
      const bool row_ok = qi < s.nq[x];
      const int see = row_ok ? s.see0 + x * QT + qi : -1;  // a row past the tile's queries sees nothing
      const int see0 = s.see0 + x * QT;                    // of the tile's first query
      const int skip = sp.skip_at(s.see0), hid = hidden_to(see, a.window), edge_to = hidden_to(see0 + s.nq[x] - 1, a.window);
      int eq = 0;  // the power of two that q of the row was multiplied by
      if (s.e[x] > 0) {
        // ---- this row of q: to float16, in the codes' order, with the groups' sums beside
        if (!wait_w(q_full(x), qn++)) { ok = false; break; }
        uint8_t* qr = sm + x * Sh::Q_BYTES + row * 128;
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < HD / 8; ++j) {
          const uint4 v = *reinterpret_cast<const uint4*>(qr + (j / 8) * Sh::QCOL + (((j % 8) ^ (row & 7)) << 4));
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) most = max(most, max(w[k] & 0x7fff0000u, (w[k] & 0x7fffu) << 16));
        }
        eq = 8 - max(-112, min(126, (int)(most >> 23) - 127));
        const float up = pow2(eq);
        float sum[NG];
#pragma unroll
        for (int nn = 0; nn < NG; ++nn) {
          sum[nn] = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            uint4* at = reinterpret_cast<uint4*>(qr + nn * Sh::QCOL + ((j ^ (row & 7)) << 4));
            float f[8];
            Vec16<bf16>::load(reinterpret_cast<const bf16*>(at), f);
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const __half2 hh = __floats2half2_rn(f[k] * up, f[k + 4] * up);
              const float2 back = __half22float2(hh);  // (what the products will see)
              sum[nn] += back.x + back.y;
              w[k] = *reinterpret_cast<const uint32_t*>(&hh);
            }
            *at = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
        uint32_t terms[3];  // of both groups' sums
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          const __half2 hh = __floats2half2_rn(sum[0], NG == 2 ? sum[NG - 1] : 0.f);
          const float2 back = __half22float2(hh);
          sum[0] -= back.x;
          if (NG == 2) sum[NG - 1] -= back.y;
          terms[k] = *reinterpret_cast<const uint32_t*>(&hh);
        }
        uint8_t* xr = sm + Sh::OFF_QX + x * Sh::QX + row * 32;
        const int flip = (row >> 2) & 1;
        *reinterpret_cast<uint4*>(xr + (flip << 4)) = make_uint4(terms[0], terms[0], terms[1], terms[1]);
        *reinterpret_cast<uint4*>(xr + ((1 ^ flip) << 4)) = make_uint4(terms[2], terms[2], 0, 0);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_ready(x));
      }
      const int row_exp = scale_exp - eq;
      float m_run = -INFINITY, l_run = 0.f;  // m: of the scores in base 2 plus the power of V
      for (int i = 0; i < s.e[x]; ++i, ++n) {
        if (!wait_w(s_full(x, n), n >> 1)) { ok = false; break; }
        tc_fence_after();
        const int key0 = block_at<KEYS_4BIT>(s.kb0 + i, sinks, skip) * 64;
        const uint32_t t_sn = t_s + 64u * (n & 1);
        uint32_t su[64];
        tmem_ld_32_issue(t_sn, su);
        tmem_ld_32_issue(t_sn + 32, su + 32);
        const float4 info = s_info[(blk + i) % Sh::FLAGS];
        const bool gone = __float_as_int(info.w) & 1;
        // (on the exponents: the powers of the keys and of q may each pass float32's range where their product does not)
        const int ex = max(1, min(254, row_exp + __float_as_int(info.x)));
        const float scale = __uint_as_float(scale_frac | (uint32_t)ex << 23), vscale = info.y;
        const bool edge = key0 + 63 > see0 || (key0 <= edge_to && key0 + 63 >= a.first) || gone;
        // columns 0..see - key0 are visible, but for first - key0..hid - key0 under a window (beside the edges a row past the tile's
        // queries may take what its q gives: nobody reads it)
        auto seen = [&] { return gone ? 0 : low_bits(see - key0 + 1) & (low_bits(a.first - key0) | ~low_bits(hid - key0 + 1)); };
        // raw scores are below 2^13: past 2^26 in all, the maximum and the scores have to be rounded alike, which own_block does
        const bool own = __float_as_int(info.w) & 2;
        if (__any_sync(0xffffffffu, own || ex > 127 + 13)) {
          tmem_ld_wait();
          OwnBlock ob{t_sn, t_o, scale, edge ? seen() : ~0ull, own ? s_w + ((blk + i) % Sh::WS) * 64 : nullptr, info.z,
                      i > 0 ? o_done(x, n - 1) : 0, ((n - 1) >> 1) & 1, abort_flag, a.werr, m_run, l_run};
          ok = own_block<HD>(ob);
          if (!ok) break;
          m_run = ob.m;
          l_run = ob.l;
        } else {
          tmem_ld_wait();
          hold_32(su);
          hold_32(su + 32);
          if (edge) {
            const uint64_t m = seen();
            const uint32_t bits[2] = {(uint32_t)m, (uint32_t)(m >> 32)};
#pragma unroll
            for (int k = 0; k < 64; ++k)
              if (!(bits[k / 32] & (1u << (k % 32)))) su[k] = 0xff800000u;  // -inf
          }
          float pm4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int k = 0; k < 64; ++k) pm4[k & 3] = fmaxf(pm4[k & 3], __uint_as_float(su[k]));
          const float pm = fmaf(fmaxf(fmaxf(pm4[0], pm4[1]), fmaxf(pm4[2], pm4[3])), scale, vscale);
          // O is rescaled only when a row's maximum grows by more than 8 in base 2, after the P V before has landed; P is 2^6 then
          const bool grow = pm - m_run > 14.f;
          if (__any_sync(0xffffffffu, grow)) {
            const float m_new = pm - 6.f, cr = grow ? exp2f(m_run - m_new) : 1.f;  // 0 when m_run was -inf
            if (i > 0) {
              if (!wait_w(o_done(x, n - 1), (n - 1) >> 1)) { ok = false; break; }
              tc_fence_after();
#pragma unroll
              for (int c0 = 0; c0 < HD; c0 += 16) {
                float o[16];
                tmem_ld_16(t_o + (uint32_t)c0, o);
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] *= cr;
                tmem_st_16(t_o + (uint32_t)c0, o);
              }
            }
            if (grow) {
              l_run *= cr;
              m_run = m_new;
            }
          }
          const float mref = m_run == -INFINITY ? 0.f : vscale - m_run;  // no visible key so far: any finite value
          const uint64_t scale2 = f2_pack(scale, scale), mref2 = f2_pack(mref, mref);
          uint64_t ps[2] = {0, 0};  // (two sums each)
#pragma unroll
          for (int c0 = 0; c0 < 64; c0 += 32) {
            uint32_t pk[16];
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              const float2 e = f2_unpack(f2_fma(f2_pack(__uint_as_float(su[c0 + k]), __uint_as_float(su[c0 + k + 1])), scale2, mref2));
              const float p0 = ex2_fast(e.x), p1 = ex2_fast(e.y);
              ps[k / 2 & 1] = f2_add(ps[k / 2 & 1], f2_pack(p0, p1));
              pk[k / 2] = pack_f16(p0, p1);
            }
            tmem_put_16(t_sn + (uint32_t)(c0 / 2), pk);
          }
          const float2 sum = f2_unpack(f2_add(ps[0], ps[1]));
          l_run = fmaf(sum.x + sum.y, info.z, l_run);
          tmem_st_wait_done();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(x, n));
      }
      // the last P V, then the row out: O / l, or its part
      const bool whole = s.kb0 == 0 && s.kb1 == s.nb;
      const long long token = s.token0 + x * QT + qi;
      const int head = (s.h << g_log) + g;
      const int slot = 2 * blockIdx.x + (s.kb0 == 0), prow = x * 128 + row;  // of the part
      bf16* orow = static_cast<bf16*>(a.out) + token * a.os + (long long)head * HD;
      const bool wide = reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && a.os % 8 == 0;
      if (ok && s.e[x] > 0) {
        if (!wait_w(o_done(x, n - 1), (n - 1) >> 1)) break;
        tc_fence_after();
        float inv = 64.f * (whole ? (l_run != 0.f ? 1.f / l_run : 0.f) : 1.f);  // (V was divided by 2^6 more)
        if (!whole && l_run > 0x1p20f) {  // (as in k_chunk_q4)
          const float up = m_run + (float)((int)(__float_as_uint(l_run) >> 23) - 127), by = ex2_fast(m_run - up);
          inv *= by;
          l_run *= by;
          m_run = up;
        }
#pragma unroll
        for (int c0 = 0; c0 < HD; c0 += 32) {
          float o[32];
          tmem_ld_32(t_o + (uint32_t)c0, o);
          if (!row_ok) continue;
#pragma unroll
          for (int k = 0; k < 32; k += 8) {  // eight dims, out of the codes' order
            const float y[8] = {o[k] * inv, o[k + 2] * inv, o[k + 4] * inv, o[k + 6] * inv, o[k + 1] * inv, o[k + 3] * inv, o[k + 5] * inv, o[k + 7] * inv};
            if (!whole) {
              *reinterpret_cast<float4*>(a.part_o + pair_part(slot, prow, c0 + k, HD)) = make_float4(y[0], y[1], y[2], y[3]);
              *reinterpret_cast<float4*>(a.part_o + pair_part(slot, prow, c0 + k + 4, HD)) = make_float4(y[4], y[5], y[6], y[7]);
            } else if (wide) {
              *reinterpret_cast<uint4*>(orow + c0 + k) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j) orow[c0 + k + j] = from_f32<bf16>(y[j]);
            }
          }
        }
        tc_fence_before();
      } else if (row_ok && !whole) {  // the tile has no block here: an empty part
        for (int k = 0; k < HD; ++k) a.part_o[pair_part(slot, prow, k, HD)] = 0.f;
      }
      if (row_ok) {
        if (!whole) a.part_ml[(size_t)slot * PAIR_ROWS + prow] = make_float2(m_run, l_run);
        else if (a.lse) a.lse[token * c.Hq + head] = l_run != 0.f ? (m_run + log2f(l_run)) * LN2 : -INFINITY;
      }
      blk += s.kb1 - s.kb0;
    }
  }
  if (*abort_flag) drain_copies();
  tc_fence_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

// ----------------------------------------------------------------------------
// Launches
// ----------------------------------------------------------------------------
template <int HD, int NT>
static cudaError_t q4_launch(const ChunkAttn& a, cudaStream_t st) {
  using Sh = Q4Shape<HD, NT>;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_q4<HD, NT>), Sh::bytes(SV_MAX_ROWS))) return e;
  return launch_k(k_chunk_q4<HD, NT>, dim3(a.ctas), dim3(Sh::THREADS), Sh::bytes(a.c.n), st, a);
}
int chunk4_per_sm(int hd, int rows) { return Q4_PER_SM(hd, rows > 8 ? 2 : 1); }
template <int HD>
static cudaError_t pair4_launch(const ChunkAttn& a, cudaStream_t st) {
  CUtensorMap qm;
  if (!chunk_q_map(&qm, a)) return cudaErrorInvalidValue;
  using Sh = Pair4Shape<HD>;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_pair4<HD>), Sh::bytes(SV_MAX_ROWS))) return e;
  int g_log = 0;
  while ((2 << g_log) <= a.c.G) ++g_log;
  return launch_k(k_chunk_pair4<HD>, dim3(a.ctas), dim3(PAIR4_THREADS), Sh::bytes(a.c.n), st, a, g_log, qm);
}
cudaError_t launch_chunk4(const ChunkAttn& a, cudaStream_t st) {
  if (a.rows == PAIR_ROWS) return a.c.hd == 64 ? pair4_launch<64>(a, st) : pair4_launch<128>(a, st);
  if (a.rows == 8) return a.c.hd == 32 ? q4_launch<32, 1>(a, st) : a.c.hd == 64 ? q4_launch<64, 1>(a, st) : q4_launch<128, 1>(a, st);
  return a.c.hd == 32 ? q4_launch<32, 2>(a, st) : a.c.hd == 64 ? q4_launch<64, 2>(a, st) : q4_launch<128, 2>(a, st);
}

}  // namespace tlf
