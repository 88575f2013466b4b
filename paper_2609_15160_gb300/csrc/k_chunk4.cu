// Attention of chunks of new tokens over caches in 4 bits, under a window or not (tlf_attn_window), bfloat16 calls. Items, their
// split over the CTAs and the join are those of k_chunk.cu.
//
// k_chunk_q4   up to 16 query rows an item: codes straight from shared memory into mma.sync fragments.
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
// p_t d_t,g is rounded to float16, an operand's type, as the other kernels round p. What float16 has to hold is 2^(s - M) d: M is the
// running maximum of s + log2(d), the largest d of the entry's groups, not of s, so that values of any magnitude fit. It is refreshed
// when a product passes 2^15 (or p, where d is tiny, 2^100).
//
// CTAs of four warps, each with 16 of a page's 64 keys, and a producer warp that copies a page's two blocks.
struct Q4Seg {  // a CTA's part of an item: blocks kb0 .. kb1 - 1 of nb; nb = 0: no more
  int b, h, token0, see0, nq, kb0, kb1, nb;
  static constexpr int RING = 4;
};
template <int HD, int NT>
struct Q4Shape {
  using F = Kv4<HD>;
  static constexpr int RT = 8 * NT, WARPS = 4, THREADS = 32 * (WARPS + 1), STAGE = 2 * F::BLOCK;
  static constexpr int PER_SM = NT == 2 ? 2 : HD == 128 ? 3 : 4;
  static constexpr int NST = HD == 128 ? (NT == 2 ? 9 : 6) : HD == 64 ? 9 : 12;
  static constexpr int OS = HD + 4;  // floats of a merge buffer's row
  static constexpr int OFF_O = NST * STAGE, OFF_ML = OFF_O + 2 * RT * OS * 4, OFF_BAR = OFF_ML + WARPS * RT * 8;
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
      mbar_init(empty(i), Sh::WARPS);
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
  const int ka = warp * 16 + kappa(g);                                        // K, pairs: keys ka, ka + 8 of the page
  const int va = warp * 16 + kappa(2 * cl), vb = warp * 16 + kappa(2 * cl + 1);  // V: keys va, vb, va + 8, vb + 8
  for (unsigned segs = 0;; ++segs) {
    // the warps leave together or not at all: they meet at barriers below, which know no time limit
    if (bar_any(1, 32 * Sh::WARPS, !wait(seg_full(segs), segs / Q4Seg::RING))) break;
    const Q4Seg it = s_seg[segs % Q4Seg::RING];
    if (it.nb == 0) break;
    const int nq = it.nq, rows = nq * G, see0 = it.see0, see_last = see0 + nq - 1;
    const int skip = sp.skip_at(see0), gone_to = hidden_to(see0, a.window), edge_to = hidden_to(see_last, a.window);
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
      const int e = max(-100, min(126, (int)(__float_as_uint(mx) >> 23) - 127));
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
        fa[t][j] = __shfl_sync(0xffffffffu, down, from);
#pragma unroll
        for (int n = 0; n < NG; ++n) qs[t][n][j] = __shfl_sync(0xffffffffu, sum[n], from) * a.scale;
        // rows past the tile's see what its first query sees, with q = 0; nobody reads them
        see[t][j] = see0 + (rj < rows ? rj / G : 0);
      }
    }
    const float fb = a.scale * 0x1p24f;
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
      const int st = seq % NST;
      const bool ok = __all_sync(0xffffffffu, wait(full(st), seq / NST));
      const int page0 = block_at<KEYS_4BIT>(kb, sinks, skip) * 64, key0 = page0 + warp * 16;
      if (ok && !s_skip[st] && key0 <= see_last && !(key0 >= a.first && key0 + 15 <= gone_to)) {
        const uint8_t *sk = sm + st * Sh::STAGE, *sv = sk + F::BLOCK;
        float acc[NT][NG][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int n = 0; n < NG; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][n][i] = 0.f;
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          uint32_t wa[W], wb[W];
          const uint8_t* p = sk + ka * (HD / 2) + n * 32 + cl * (4 * W);
          if constexpr (W == 2) {
            *reinterpret_cast<uint2*>(wa) = *reinterpret_cast<const uint2*>(p);
            *reinterpret_cast<uint2*>(wb) = *reinterpret_cast<const uint2*>(p + 8 * (HD / 2));
          } else {
            wa[0] = *reinterpret_cast<const uint32_t*>(p);
            wb[0] = *reinterpret_cast<const uint32_t*>(p + 8 * (HD / 2));
          }
#pragma unroll
          for (int w = 0; w < W; ++w) {
            const uint32_t xa = wa[w] >> 8, xb = wb[w] >> 8;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              mma_f16(acc[t][n], wa[w] & LO, wb[w] & LO, wa[w] & HI, wb[w] & HI, qf[t][n][w][0], qf[t][n][w][1]);
              mma_f16(acc[t][n], xa & LO, xb & LO, xa & HI, xb & HI, qf[t][n][w][2], qf[t][n][w][3]);
            }
          }
        }
        // the pairs of keys ka and ka + 8, of K and of V
        uint32_t kp[2][NG], vp[2][NG];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int at = F::CODES + (ka + 8 * x) * NG * 4;
          if constexpr (NG == 2) {
            *reinterpret_cast<uint2*>(kp[x]) = *reinterpret_cast<const uint2*>(sk + at);
            *reinterpret_cast<uint2*>(vp[x]) = *reinterpret_cast<const uint2*>(sv + at);
          } else {
            kp[x][0] = *reinterpret_cast<const uint32_t*>(sk + at);
            vp[x][0] = *reinterpret_cast<const uint32_t*>(sv + at);
          }
        }
        float s[NT][2][2];  // [key][column]
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float dn = 0.f, lo = 0.f;
#pragma unroll
              for (int n = 0; n < NG; ++n) {
                const float2 p = kv4_pair(kp[x][n]);
                dn = fmaf(p.x, acc[t][n][2 * x + j], dn);
                lo = fmaf(p.y, qs[t][n][j], lo);
              }
              s[t][x][j] = fmaf(dn * fa[t][j], fb, lo);
            }
        if (key0 + 15 > see0 || (key0 <= edge_to && key0 + 15 >= a.first)) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int key = page0 + ka + 8 * x;
            const bool past = key >= a.first;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int j = 0; j < 2; ++j)
                if (key > see[t][j] || (past && key <= hidden_to(see[t][j], a.window))) s[t][x][j] = -INFINITY;
            if (key > see_last || (past && key <= gone_to))  // nobody sees it: its pairs may be anything
#pragma unroll
              for (int n = 0; n < NG; ++n) vp[x][n] = 0;
          }
        }
        float p[NT][2][2];
        uint32_t ph[NT][NG][2];  // p d of the two columns, keys ka and ka + 8
        auto weigh = [&] {
          bool grow = false;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            uint32_t big = 0;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
              for (int j = 0; j < 2; ++j) p[t][x][j] = ex2_fast(s[t][x][j] - m[t][j]);
#pragma unroll
              for (int n = 0; n < NG; ++n) {
                const float d = kv4_pair(vp[x][n]).x;
                ph[t][n][x] = pack_f16(p[t][x][0] * d, p[t][x][1] * d);
                big |= ph[t][n][x] + 0x08000800u;  // the sign bit of a half from 2^15 on, infinities and NaN too
              }
            }
            grow |= (big & 0x80008000u) != 0 || !(fmaxf(p[t][0][0], p[t][1][0]) <= 0x1p100f) || !(fmaxf(p[t][0][1], p[t][1][1]) <= 0x1p100f);
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
              for (int x = 0; x < 2; ++x) {
                float d = kv4_pair(vp[x][0]).x;
                if constexpr (NG == 2) d = fmaxf(d, kv4_pair(vp[x][1]).x);
                top = fmaxf(top, s[t][x][j] + log2f(fmaxf(d, 0x1p-100f)));
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
#pragma unroll
          for (int j = 0; j < 2; ++j) l[t][j] += p[t][0][j] + p[t][1][j];
#pragma unroll
          for (int n = 0; n < NG; ++n) {
            const float la = kv4_pair(vp[0][n]).y, lb = kv4_pair(vp[1][n]).y;
#pragma unroll
            for (int j = 0; j < 2; ++j) ol[t][n][j] = fmaf(p[t][0][j], la, fmaf(p[t][1][j], lb, ol[t][n][j]));
#pragma unroll
            for (int x = 0; x < 2; ++x) ph[t][n][x] = transpose_8x8(ph[t][n][x]);
          }
        }
        // V: dims 8 g .. 8 g + 7 of a group (head_dim 32: 4 g .. 4 g + 3)
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          uint32_t w[4];
          const int at[4] = {va, vb, va + 8, vb + 8};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint8_t* q = sv + at[i] * (HD / 2) + n * 32 + g * (F::GS / 16);
            if constexpr (F::GS == 64) w[i] = *reinterpret_cast<const uint32_t*>(q);
            else w[i] = *reinterpret_cast<const uint16_t*>(q);
          }
#pragma unroll
          for (int half = 0; half < MT / 2; ++half) {
            const uint32_t sel = half ? 0x7632u : 0x5410u;
            const uint32_t u = __byte_perm(w[0], w[1], sel), v = __byte_perm(w[2], w[3], sel), u8 = u >> 8, v8 = v >> 8;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              mma_f16(o[t][n][2 * half], u & LO, u & HI, v & LO, v & HI, ph[t][n][0], ph[t][n][1]);
              mma_f16(o[t][n][2 * half + 1], u8 & LO, u8 & HI, v8 & LO, v8 & HI, ph[t][n][0], ph[t][n][1]);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }

    // the warps' parts: each to the item's maximum, the upper two added to the lower two, then both
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
        if (g == 0) s_ml[warp * RT + t * 8 + 2 * cl + j] = make_float2(m[t][j], l[t][j]);
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
            float* to = s_o + ((warp & 1) * RT + t * 8 + 2 * cl + j) * OS + n * F::GS + g * (2 * MT);
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
    if (warp >= 2) put(false);
    bar_named(1, 32 * Sh::WARPS);
    if (warp < 2) put(true);
    bar_named(1, 32 * Sh::WARPS);
    const bool whole = it.kb0 == 0 && it.kb1 == it.nb;
    const size_t part = (size_t)(2 * blockIdx.x + (it.kb0 == 0)) * a.rows;
    for (int i = tid; i < rows * (HD / 4); i += 32 * Sh::WARPS) {
      const int r = i / (HD / 4), d = (i % (HD / 4)) * 4;
      const float4 u = *reinterpret_cast<const float4*>(s_o + r * OS + d), w = *reinterpret_cast<const float4*>(s_o + (RT + r) * OS + d);
      const float4 v = make_float4(u.x + w.x, u.y + w.y, u.z + w.z, u.w + w.w);
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
// Launches
// ----------------------------------------------------------------------------
template <int HD, int NT>
static cudaError_t q4_launch(const ChunkAttn& a, cudaStream_t st) {
  using Sh = Q4Shape<HD, NT>;
  if (cudaError_t e = ensure_kernel_attrs(reinterpret_cast<const void*>(k_chunk_q4<HD, NT>), Sh::bytes(SV_MAX_ROWS))) return e;
  return launch_k(k_chunk_q4<HD, NT>, dim3(a.ctas), dim3(Sh::THREADS), Sh::bytes(a.c.n), st, a);
}
int chunk4_per_sm(int hd, int rows) { return rows > 8 ? 2 : hd == 128 ? 3 : 4; }
cudaError_t launch_chunk4(const ChunkAttn& a, cudaStream_t st) {
  if (a.rows == 8) return a.c.hd == 32 ? q4_launch<32, 1>(a, st) : a.c.hd == 64 ? q4_launch<64, 1>(a, st) : q4_launch<128, 1>(a, st);
  return a.c.hd == 32 ? q4_launch<32, 2>(a, st) : a.c.hd == 64 ? q4_launch<64, 2>(a, st) : q4_launch<128, 2>(a, st);
}

}  // namespace tlf
