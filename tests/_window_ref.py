"""Plain 64-bit forms of the 4-bit cache, windowed attention and the page operators."""
import math

import numpy as np

import _serve_ref as R

PAGE = 64
LARGEST = np.float32(2.0 ** 126)


def groups(hd):
    return max(1, hd // 64)


def bits(x):
    """The bit patterns of float32 values that are bfloat16's."""
    return (np.ascontiguousarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)


def quantise(x):
    """(codes [..., hd / 2] uint8, pairs [..., groups, 2] uint16 bits) of float32 values [..., hd] that a plain cache would hold."""
    x = np.where(np.isnan(x), np.float32(0), np.asarray(x, np.float32))
    x = np.clip(x, -LARGEST, LARGEST).reshape(*x.shape[:-1], groups(x.shape[-1]), min(64, x.shape[-1]))
    lo = R.bf16(x.min(-1, keepdims=True))
    d = R.bf16(np.maximum(x.max(-1, keepdims=True) - lo, np.float32(0)) / np.float32(15))
    with np.errstate(divide="ignore", invalid="ignore"):
        n = np.where(d > 0, np.clip(np.rint((x - lo) / d), 0, 15), 0).astype(np.uint8)
    n = n.reshape(*n.shape[:-2], n.shape[-2] * n.shape[-1])
    return n[..., 0::2] | n[..., 1::2] << 4, np.concatenate([bits(d), bits(lo)], -1)


def parts(pool, hd):
    """Views (codes [..., 64, hd / 2], pairs [..., 64, groups, 2] uint16) of blocks [..., bytes]."""
    n = PAGE * hd // 2
    codes = pool[..., :n].reshape(*pool.shape[:-1], PAGE, hd // 2)
    return codes, np.ascontiguousarray(pool[..., n:]).view(np.uint16).reshape(*pool.shape[:-1], PAGE, groups(hd), 2)


def blocks(codes, pairs):
    """Blocks [..., bytes] of codes [..., 64, hd / 2] and pairs [..., 64, groups, 2]."""
    lead = codes.shape[:-2]
    return np.concatenate([codes.reshape(*lead, -1), np.ascontiguousarray(pairs, np.uint16).view(np.uint8).reshape(*lead, -1)], -1)


def terms(codes, pairs):
    """(lo, d n), each [..., hd] in 64 bits."""
    f = (pairs.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    n = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], pairs.shape[-2], 2 * codes.shape[-1] // pairs.shape[-2])
    with np.errstate(invalid="ignore"):
        dn = f[..., :1] * n
    to = codes.shape[:-1] + (2 * codes.shape[-1],)
    return np.broadcast_to(f[..., 1:], dn.shape).reshape(to), dn.reshape(to)


class Cache4(R.Cache):
    """A Cache whose pool is held in 4 bits (pool4); pool has the float32 values that it was made from."""

    def __init__(self, *a, **kw):
        super().__init__(*a, **kw)
        # some keys and values larger, some heads off centre
        self.pool *= 1 + 3 * (self.rng.random(self.pool.shape[:-1] + (1,)) < 0.05)
        self.pool += self.rng.standard_normal(self.pool.shape[2:4] + (1, self.hd)).astype(np.float32)
        self.pool4 = blocks(*quantise(self.round(self.pool)))

    def two(self, b, kv):
        """(lo, d n) of K (0) or V (1) of the row's entries [entries, kv heads, hd]."""
        p, o = self.at(b, np.arange(max(0, self.lens[b])))
        codes, pairs = parts(self.pool4, self.hd)
        return terms(codes[p, self.layer, kv, :, o], pairs[p, self.layer, kv, :, o])

    def device(self, **more):
        import torch
        pool, self.pool = self.pool, np.zeros(1, np.float32)
        d = super().device(**more)
        self.pool = pool
        d["pool"] = torch.tensor(self.pool4).cuda()
        return d


def sees(c, b, i, window, first):
    """Which of the row's entries its i-th new token sees."""
    e, at = np.arange(max(0, c.lens[b])), c.lens[b] - c.new[b] + i
    return (e <= at) & (((e > at - window) | (e < first)) if window else True)


def attention(c, window=0, first=0, scale=None):
    """out, lse, the bound sum p |terms of v| of out, the largest sum of |terms of q k| of a score."""
    scale = scale or 1 / math.sqrt(c.hd)
    four = isinstance(c, Cache4)
    out, spread = np.zeros((c.T, c.hq, c.hd)), np.zeros((c.T, c.hq, c.hd))
    lse, most = np.full((c.T, c.hq), -np.inf), np.zeros((c.T, c.hq))
    G = c.hq // c.hkv
    for b in range(c.n):
        if four:
            (kl, kn), (vl, vn) = c.two(b, 0), c.two(b, 1)
            with np.errstate(invalid="ignore"):
                k, v, ka, va = kl + kn, vl + vn, np.abs(kl) + np.abs(kn), np.abs(vl) + np.abs(vn)
        else:
            k, v = (x.astype(np.float64) for x in c.kv(b))
            ka, va = np.abs(k), np.abs(v)
        for i in range(c.new[b]):
            t, m = c.cu[b] + i, sees(c, b, i, window, first)
            if not m.any():
                continue
            for g in range(c.hkv):
                q = c.q[t, g * G:(g + 1) * G].astype(np.float64)
                s = scale * (k[m, g] @ q.T)
                h = slice(g * G, (g + 1) * G)
                most[t, h] = (scale * (ka[m, g] @ np.abs(q).T)).max(0)
                top = s.max(0)
                lse[t, h] = top + np.log(np.exp(s - top).sum(0))
                p = np.exp(s - lse[t, h])
                with np.errstate(invalid="ignore"):
                    out[t, h] = p.T @ v[m, g]
                    spread[t, h] = p.T @ va[m, g]
    return out, lse, spread, most


def fork(pool, table, lens, parents, refs, reserve, window=0, first=0, side=None):
    """(pool, table, lens, refs, err) after a fork; pool [pages, .., 64 entries ..] with the entries on axis `side` (bytes of 4-bit
    blocks: see fork4)."""
    pages, width = len(refs), table.shape[1]
    pool, n_in = pool.copy(), len(lens)
    free = [p for p in range(pages) if refs[p] == 0]
    out, lens_out, err, seen, at = np.full((len(parents), width), -1, np.int32), np.zeros(len(parents), np.int32), 0, set(), 0
    src = pool.copy()
    for b, r in enumerate(parents):
        if r < -1 or r >= n_in:
            err, r = err | 2, -1
        n = int(lens[r]) if r >= 0 else 0
        if n < 0 or n > width * PAGE:
            err, n = err | 2, min(max(n, 0), width * PAGE)
        full, need = n // PAGE, -(-(n + reserve) // PAGE)
        if need > width:
            err, need = err | 2, width
        lens_out[b] = n
        for s in range(need):
            old = int(table[r, s]) if r >= 0 else -1
            old = old if 0 <= old < pages else -1
            if s < full:
                gone = window > 0 and PAGE * (s + 1) <= n - window + 1 and PAGE * s >= first
                out[b, s] = -1 if gone else old
                continue
            holds = s == full and n % PAGE != 0
            if r >= 0 and r not in seen and old >= 0 and refs[old] == 1:
                out[b, s] = old
                continue
            page = free[at] if at < len(free) else -1
            at += 1
            if page < 0:
                err |= 16
            if holds and old < 0:
                err, page = err | 2, -1
            if holds and page >= 0:
                copy_entries(pool, src, page, old, n % PAGE, side)
            if holds and page < 0:
                lens_out[b] = full * PAGE
            out[b, s] = page
        if r >= 0:
            seen.add(r)
    refs_out = np.array(refs, np.int64)
    for t, d in ((table, -1), (out, 1)):
        for p in np.asarray(t).ravel():
            if 0 <= p < pages:
                refs_out[p] += d
            elif p != -1:
                err |= 2
    return pool, out, lens_out, refs_out.astype(np.int32), err


def copy_entries(pool, src, to, fr, n, side):
    if side is None:  # [pages, layers, 2, heads, 64, hd]
        pool[to, :, :, :, :n] = src[fr, :, :, :, :n]
    else:             # 4-bit blocks of head_dim `side`
        at = PAGE * side // 2
        pool[to, ..., :n * side // 2] = src[fr, ..., :n * side // 2]
        pool[to, ..., at:at + n * 4 * groups(side)] = src[fr, ..., at:at + n * 4 * groups(side)]


def compact(pool, table, refs):
    used = np.asarray(refs) > 0
    live = int(used.sum())
    fr, to = [p for p in range(live, len(refs)) if used[p]], [p for p in range(live) if not used[p]]
    pool, refs_out, where = pool.copy(), np.where(used, refs, 0), np.arange(len(refs))
    pool[to], refs_out[to], where[fr] = pool[fr], refs_out[fr], to
    refs_out[live:] = 0
    return pool, np.where(table >= 0, where[np.maximum(table, 0)], -1).astype(np.int32), refs_out.astype(np.int32), live
