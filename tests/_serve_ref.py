"""Plain 64-bit forms of the operators on paged caches and logits, and seeded problems for their tests."""
import math

import numpy as np

PAGE = 64


def bf16(x):
    """float32 values of x rounded to bfloat16."""
    import torch
    return torch.tensor(np.asarray(x, np.float32)).bfloat16().float().numpy()


class Cache:
    """Ragged rows over a shuffled pool: row b has old[b] + new[b] entries, the last new[b] of them new."""

    def __init__(self, old, new, hq, hkv, hd, dtype="bf16", layers=2, layer=1, seed=0, spare=3):
        rng = np.random.default_rng(seed)
        self.old, self.new = np.asarray(old, np.int64), np.asarray(new, np.int64)
        self.lens = self.old + self.new
        self.n, self.hq, self.hkv, self.hd, self.dtype, self.layers, self.layer = len(old), hq, hkv, hd, dtype, layers, layer
        need = np.maximum(0, (self.lens + PAGE - 1) // PAGE)
        self.pages, most = int(need.sum()) + spare, max(1, int(need.max()))
        perm = rng.permutation(self.pages)
        self.table = np.full((self.n, most), -1, np.int32)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = perm[at:at + k]
            at += k
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.T = int(self.cu[-1])
        self.rng = rng
        draw = lambda *s: self.round(rng.standard_normal(s).astype(np.float32))  # noqa: E731
        self.pool = draw(self.pages, layers, 2, hkv, PAGE, hd)
        self.q = draw(max(1, self.T), hq, hd) * 2

    def round(self, x):
        return bf16(x) if self.dtype == "bf16" else np.asarray(x, np.float32)

    def at(self, b, e):
        return self.table[b, e // PAGE], e % PAGE

    def kv(self, b):
        p, o = self.at(b, np.arange(max(0, self.lens[b])))
        return self.pool[p, self.layer, 0, :, o], self.pool[p, self.layer, 1, :, o]

    def device(self, **more):
        import torch
        dt = torch.bfloat16 if self.dtype == "bf16" else torch.float32
        d = dict(pool=torch.tensor(self.pool).to(dt).cuda(), table=torch.tensor(self.table).cuda(),
                 cu=torch.tensor(self.cu).cuda(), lens=torch.tensor(self.lens.astype(np.int32)).cuda(),
                 q=torch.tensor(self.q).to(dt).cuda(), err=torch.zeros(1, dtype=torch.int32, device="cuda"))
        d.update({k: torch.tensor(v).cuda() for k, v in more.items()})
        return d


def attention(c, scale=None):
    """out [T, hq, hd], lse [T, hq], the bound sum p |v| of out, the largest sum of |q k| of a score, weights per row."""
    scale = scale or 1 / math.sqrt(c.hd)
    out, spread = np.zeros((c.T, c.hq, c.hd)), np.zeros((c.T, c.hq, c.hd))
    lse, terms = np.full((c.T, c.hq), -np.inf), np.zeros((c.T, c.hq))
    weights = [np.zeros(max(0, n)) for n in c.lens]
    G = c.hq // c.hkv
    for b in range(c.n):
        k, v = (x.astype(np.float64) for x in c.kv(b))
        for i in range(c.new[b]):
            t, seen = c.cu[b] + i, c.lens[b] - c.new[b] + i + 1
            if seen <= 0:
                continue
            for h in range(c.hq):
                q = c.q[t, h].astype(np.float64)
                s = scale * (k[:seen, h // G] @ q)
                terms[t, h] = (scale * (np.abs(k[:seen, h // G]) @ np.abs(q))).max()
                m = s.max()
                lse[t, h] = m + np.log(np.exp(s - m).sum())
                p = np.exp(s - lse[t, h])
                with np.errstate(invalid="ignore"):
                    out[t, h] = p @ v[:seen, h // G]
                    spread[t, h] = p @ np.abs(v[:seen, h // G])
                weights[b][:seen] += p
    return out, lse, spread, terms, weights


def turn(x, cs, rot, layout):
    """x [..., heads, hd] turned by cs [..., rot / 2, 2] (leading extents alike)."""
    y = x.astype(np.float64).copy()
    c, s = cs[..., None, :, 0].astype(np.float64), cs[..., None, :, 1].astype(np.float64)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    xa, xb = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
    return y


def evict(weight, pos, next_pos, budget, n_first, n_recent):
    """Entry whose contents each of the entries 0 .. min(len, budget) - 1 holds afterwards (one row)."""
    n = len(weight)
    if n <= budget:
        return np.arange(n)
    w = np.where(np.isnan(weight), -np.inf, weight).astype(np.float64)
    guarded = (pos < n_first) | (pos >= next_pos - n_recent)
    order = sorted(range(n), key=lambda e: (not guarded[e], np.isnan(weight[e]) and not guarded[e], -w[e], e))
    stays = np.zeros(n, bool)
    stays[order[:budget]] = True
    src = np.arange(budget)
    src[~stays[:budget]] = np.nonzero(stays[budget:])[0] + budget
    return src


def sample(l, u, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, how far the draw is from another token) of one row."""
    l = np.where(l > -np.inf, l, -np.inf).astype(np.float64)
    l = np.minimum(l, float(np.finfo(np.float32).max))
    V = len(l)
    if l.max() == -np.inf:
        return -1, -np.inf, np.inf
    greedy = not T > 0
    z = (l - l.max()) / (1.0 if greedy else float(np.float32(T)))
    w = np.exp(z)
    order = np.lexsort((np.arange(V), -l))
    order = order[:int((l > -np.inf).sum())]
    k = 1 if greedy else (top_k if top_k > 0 else V)
    order = order[:k]
    wk, top_p, min_p = w[order], float(np.float32(top_p)), float(np.float32(min_p))
    n, edge = len(order), np.inf
    if top_p < 1:
        before = np.cumsum(wk) - wk
        n = max(1, int((before < top_p * wk.sum()).sum()))
        edge = np.abs(before[1:] / wk.sum() - top_p).min() if len(order) > 1 else np.inf
    n = max(1, min(n, int((wk >= min_p).sum())))
    if min_p > 0 and len(order) > 1:
        edge = min(edge, np.abs(wk[1:] / min_p - 1).min())
    kept = order[:n]
    with np.errstate(divide="ignore", invalid="ignore"):
        race = z[kept] - np.log(-np.log(u[kept].astype(np.float64)))
    race = np.where(np.isnan(race), -np.inf, race)
    best = race.max()
    token = kept[race == best].min()
    rest = race[kept != token]
    gap = best - rest.max() if len(rest) and np.isfinite(best) else np.inf
    return int(token), z[token] - math.log(w.sum()), min(gap, edge)
