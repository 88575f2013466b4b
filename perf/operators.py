"""Timed cases of the operators around a served model's paged cache and its logits.

Four operators, each through the call that a serving program makes (the ctypes binding of libtlf):

- ``append``   rotary positions on the queries and keys of new tokens, keys and values into their pages
               (``tlf_rope_append``);
- ``attend``   attention of every row's chunk of new tokens over its paged cache, causal inside the chunk
               (``tlf_attn_chunk``); with ``weights`` it also adds to every cache entry the attention weight that the
               chunk's queries gave it, which is what the eviction goes by;
- ``evict``    every row's cache down to a budget of entries: the heaviest stay, with the first and the most recent ones
               (``tlf_cache_evict``);
- ``sample``   the next token of every row from its logits: temperature, top-k, top-p, min-p, with given random numbers
               (``tlf_sample``).

The plain forms are elementary torch operations in 32 bits on padded rows. ``exact`` restates each operator in 64 bits,
row by row. Lengths, pages and parameters of a ragged batch follow from the case, values from the seed.
"""
import math

import numpy as np
import torch

own = False  # True: run() calls the library; False: the plain forms

PAGE = 64
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ----------------------------------------------------------------------------
# Cases
# ----------------------------------------------------------------------------

def listed():
    return [
        # one decoding step of a serving batch, multi-head: latency
        dict(name="append-64x1", op="append", rows=64, new_lo=1, new_hi=1, old_lo=1000, old_hi=2048, hq=16, hkv=16, hd=64,
             rot=64, layout="half", dtype="bf16"),
        # prompts of several sequences at once, grouped-query, half of each head rotated, interleaved pairs
        dict(name="append-4x2048", op="append", rows=4, new_lo=1500, new_hi=2048, old_lo=0, old_hi=1000, hq=16, hkv=8,
             hd=128, rot=64, layout="interleaved", dtype="bf16"),
        # a tiny float32 model, a few tokens a row: latency
        dict(name="attend-f32-4x5", op="attend", rows=4, new_lo=1, new_hi=5, old_lo=0, old_hi=60, hq=4, hkv=4, hd=16,
             dtype="f32", weights=False),
        # single tokens over long contexts, grouped-query: bandwidth
        dict(name="attend-16x1-32k", op="attend", rows=16, new_lo=1, new_hi=1, old_lo=32000, old_hi=32700, hq=16, hkv=8,
             hd=128, dtype="bf16", weights=False),
        # short turns (or drafted tokens to verify) on a ragged batch, multi-head
        dict(name="attend-32x8", op="attend", rows=32, new_lo=1, new_hi=16, old_lo=128, old_hi=8192, hq=16, hkv=16, hd=64,
             dtype="bf16", weights=False),
        # long turns on long conversations, grouped-query: tensor cores
        dict(name="attend-4x2048", op="attend", rows=4, new_lo=1800, new_hi=2048, old_lo=4000, old_hi=8192, hq=16, hkv=8,
             hd=128, dtype="bf16", weights=False),
        # single tokens under a cache budget: attention that keeps account of what it looks at
        dict(name="weigh-32x1", op="attend", rows=32, new_lo=1, new_hi=1, old_lo=1000, old_hi=8192, hq=16, hkv=16, hd=64,
             dtype="bf16", weights=True),
        # prompts that will be cut to a budget
        dict(name="weigh-4x1000", op="attend", rows=4, new_lo=700, new_hi=1024, old_lo=0, old_hi=4000, hq=16, hkv=8, hd=128,
             dtype="bf16", weights=True),
        # caches a page over their budget, as in a running service: latency
        dict(name="evict-32x2048", op="evict", rows=32, len_lo=1900, len_hi=2112, budget=2048, first=4, recent=128, hkv=16,
             hd=64, layers=4, dtype="bf16"),
        # long prompts cut to a budget
        dict(name="evict-4x32k", op="evict", rows=4, len_lo=30000, len_hi=32768, budget=8192, first=4, recent=1024, hkv=8,
             hd=128, layers=2, dtype="bf16"),
        # one user's next token: latency
        dict(name="sample-1x32000", op="sample", rows=1, vocab=32000, spread=3.5),
        # a large batch, every row with its own parameters
        dict(name="sample-256x50304", op="sample", rows=256, vocab=50304, spread=3.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "evict", "sample"])
    if op == "sample":
        rows, vocab = _log(rng, 1, 256), _log(rng, 256, 50304)
        return dict(op="sample", rows=rows, vocab=vocab, spread=round(rng.uniform(1.5, 5.0), 2))
    hq, hkv, hd, dtype = rng.choice([(16, 16, 64, "bf16"), (16, 8, 128, "bf16"), (8, 8, 64, "bf16"), (8, 2, 128, "bf16"),
                                     (12, 4, 64, "bf16"), (4, 2, 32, "bf16"), (4, 4, 16, "f32"), (8, 2, 64, "f32")])
    if op == "append":
        rows = _log(rng, 1, 128)
        hi = _log(rng, 1, max(1, 8192 // rows))
        rot = rng.choice([hd, hd // 2])
        return dict(op="append", rows=rows, new_lo=rng.randint(0, hi), new_hi=hi, old_lo=0, old_hi=_log(rng, 1, 1500), hq=hq,
                    hkv=hkv, hd=hd, rot=rot, layout=rng.choice(["half", "interleaved"]), dtype=dtype)
    if op == "evict":
        rows = _log(rng, 1, 32)
        hi = _log(rng, 100, 131072 // rows)
        budget = rng.randint(64, hi)
        first = rng.randint(0, min(8, budget // 4))
        return dict(op="evict", rows=rows, len_lo=rng.randint(1, hi), len_hi=hi, budget=budget, first=first,
                    recent=rng.randint(0, budget // 2), hkv=hkv, hd=hd, layers=rng.randint(1, 2), dtype=dtype)
    kind = rng.choice(["one", "few", "many"])
    weights = rng.random() < 0.35
    if dtype == "f32":  # small models
        rows, new = _log(rng, 1, 16), 1 if kind == "one" else _log(rng, 2, 64 if kind == "few" else 300)
        old = _log(rng, 1, 2000)
    elif kind == "one":
        rows, new = _log(rng, 1, 64), 1
        old = _log(rng, 1, min(32700, 400000 // rows))
    elif kind == "few":
        rows, new = _log(rng, 1, 48), _log(rng, 2, 48)
        old = _log(rng, 1, min(16000, 200000 // rows))
    else:
        rows, new = _log(rng, 1, 6), _log(rng, 49, 2048)
        old = _log(rng, 1, 8192)
    return dict(op="attend", rows=rows, new_lo=new if kind == "one" else rng.randint(0, new), new_hi=new,
                old_lo=rng.randint(0, old), old_hi=old, hq=hq, hkv=hkv, hd=hd, dtype=dtype, weights=weights)


def _lengths(c, what):
    """Ragged lengths of the rows, from the case alone; the longest one occurs."""
    lo, hi = c[what + "_lo"], c[what + "_hi"]
    r = np.random.RandomState((lo * 31 + hi * 17 + c["rows"]) % (1 << 31))
    v = r.randint(lo, hi + 1, c["rows"])
    v[r.randint(c["rows"])] = hi
    return v.astype(np.int64)


def work(c):
    if c["op"] == "sample":  # the logits once; the random numbers of the few kept tokens are left out
        return {"bytes": c["rows"] * (4.0 * c["vocab"] + 24), "flops": 4.0 * c["rows"] * c["vocab"]}
    eb = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "evict":
        lens = _lengths(c, "len")
        kept = np.minimum(lens, c["budget"])
        # weights and positions in and out; an entry beyond the budget that stays moves once: in expectation its share of the
        # entries that the weights decide on
        free = np.maximum(1, lens - c["first"] - c["recent"])
        beyond = np.maximum(0, lens - c["budget"])
        recent = np.minimum(beyond, c["recent"])
        moved = recent + (beyond - recent) * np.clip((kept - c["first"] - c["recent"]) / free, 0, 1)
        moved = np.where(lens > c["budget"], moved, 0).sum()
        return {"bytes": float(lens.sum() * 8 + kept.sum() * 8 + moved * 2 * c["layers"] * 2 * c["hkv"] * c["hd"] * eb),
                "flops": float(lens.sum())}
    new, old = _lengths(c, "new").astype(float), _lengths(c, "old").astype(float)
    T = new.sum()
    if c["op"] == "append":
        return {"bytes": float(T * (2 * (c["hq"] + 2 * c["hkv"]) * c["hd"] * eb + c["rot"] * 4 + 8)),
                "flops": float(T * (c["hq"] + c["hkv"]) * c["rot"] * 3)}
    keys = np.where(new > 0, old + new, 0).sum()
    pairs = (new * old + new * (new + 1) / 2).sum()
    b = keys * 2 * c["hkv"] * c["hd"] * eb + T * c["hq"] * (2 * c["hd"] * eb + 4)
    if c["weights"]:
        b += (old + new).sum() * 8
    return {"bytes": float(b), "flops": float(4 * c["hd"] * c["hq"] * pairs)}


# ----------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------

def _pages(lens, gen_case):
    """Page table of ragged rows over a shuffled pool with some spare pages: (table [rows][most], pages)."""
    need = (lens + PAGE - 1) // PAGE
    most, total = max(1, int(need.max())), int(need.sum()) + 3
    perm = gen_case.permutation(total)
    table = np.full((len(lens), most), -1, np.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = perm[at:at + k]
        at += k
    return table, total


def _rope_table(rot, max_pos, device):
    """(cos, sin) of position x frequency, base 10000, positions stretched by 2 (linear scaling), from 64 bits."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    ang = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None] / 2.0 * inv
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()


def prepare(c, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 13)
    s = {"case": c}
    if c["op"] == "sample":
        B, V = c["rows"], c["vocab"]
        r = np.random.RandomState(int(seed) % (1 << 31))
        s["logits"] = torch.randn(B, V, device=dev, generator=g) * c["spread"]
        s["logits"][torch.rand(B, V, device=dev, generator=g) < 0.01] = -math.inf  # tokens that a grammar forbids
        s["noise"] = torch.rand(B, V, device=dev, generator=g)
        pick = lambda v: torch.tensor(r.choice(v, B), device=dev)  # noqa: E731
        s["temperature"] = pick([0.0, 0.6, 0.7, 0.8, 1.0, 1.0, 1.3]).float()
        s["top_k"] = pick([0, 0, 20, 50, 200]).int()
        s["top_p"] = pick([1.0, 0.8, 0.9, 0.95]).float()
        s["min_p"] = pick([0.0, 0.0, 0.02, 0.1]).float()
        s["tokens"] = torch.empty(B, dtype=torch.int32, device=dev)
        s["logprobs"] = torch.empty(B, dtype=torch.float32, device=dev)
        return s

    dt, hkv, hd = DTYPES[c["dtype"]], c["hkv"], c["hd"]
    rc = np.random.RandomState(c["rows"] * 101 + hd)
    i32 = lambda v: torch.tensor(np.ascontiguousarray(v, dtype=np.int32), device=dev)  # noqa: E731
    if c["op"] == "evict":
        lens = _lengths(c, "len")
        table, pages = _pages(lens, rc)
        s["layers"], s["lens"], s["most"] = c["layers"], i32(lens), int(lens.max())
        s["pool"] = torch.randn(pages, c["layers"], 2, hkv, PAGE, hd, device=dev, generator=g).to(dt)
        # weights as attention leaves them: a heavy tail, and entries that nothing has looked at yet
        w = torch.rand(pages, PAGE, device=dev, generator=g).log().neg().pow(3)
        w[torch.rand(pages, PAGE, device=dev, generator=g) < 0.1] = 0
        s["weight"], s["weight_out"] = w, torch.zeros_like(w)
        s["page_table"] = i32(table)
        # positions: entries in the order of their tokens, some tokens left out
        pos = torch.full((pages, PAGE), -1, dtype=torch.int32, device=dev)
        nxt = []
        for b, n in enumerate(lens):
            p = np.arange(n) + np.cumsum(rc.rand(n) < 0.1)
            e = np.arange(n)
            pos[s["page_table"][b].long()[torch.tensor(e // PAGE, device=dev)], torch.tensor(e % PAGE, device=dev)] = i32(p)
            nxt.append(int(p[-1]) + 1)
        s["pos"], s["pos_out"], s["next_pos"] = pos, torch.full_like(pos, -1), i32(nxt)
        s["lens_out"] = torch.zeros_like(s["lens"])
        return s

    new, old = _lengths(c, "new"), _lengths(c, "old")
    lens = old + new
    table, pages = _pages(lens, rc)
    T = int(new.sum())
    s.update(T=T, most_new=max(1, int(new.max())), most=max(1, int(lens.max())), layers=2, layer=1, lens=i32(lens),
             page_table=i32(table), cu=i32(np.concatenate([[0], np.cumsum(new)])))
    s["pool"] = torch.randn(pages, 2, 2, hkv, PAGE, hd, device=dev, generator=g).to(dt)
    if c["op"] == "append":
        s["qkv"] = torch.randn(max(1, T), (c["hq"] + 2 * hkv) * hd, device=dev, generator=g).to(dt)
        # a token's position: ahead of its entry, since some tokens left none in this cache
        p = np.concatenate([o + np.arange(n) + o // 8 for o, n in zip(old, new)]) if T else np.zeros(0)
        s["positions"] = i32(p)
        s["max_pos"] = c["old_hi"] + c["new_hi"] + c["old_hi"] // 8 + 1
        s["table"] = _rope_table(c["rot"], s["max_pos"], dev)
        s["q_out"] = torch.zeros(max(1, T), c["hq"], hd, dtype=dt, device=dev)
        s["pos"] = torch.full((pages, PAGE), -1, dtype=torch.int32, device=dev)
        return s
    # queries that look at some keys more than at others
    s["q"] = (torch.randn(max(1, T), c["hq"], hd, device=dev, generator=g) * 1.5).to(dt)
    s["out"] = torch.zeros(max(1, T), c["hq"], hd, dtype=dt, device=dev)
    s["lse"] = torch.zeros(max(1, T), c["hq"], dtype=torch.float32, device=dev)
    if c["weights"]:
        s["weight"] = torch.rand(pages, PAGE, device=dev, generator=g) * 4
        s["weight_out"] = torch.zeros_like(s["weight"])
    return s


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    return {"append": _append, "attend": _attend, "evict": _evict, "sample": _sample}[s["case"]["op"]](s)


def _run_own(s):
    from paper_2609_15160_gb300 import tlf
    c = s["case"]
    stream = torch.cuda.current_stream()
    if "args" not in s:  # the buffers' descriptions and the workspace, which a program makes once and keeps with the buffers
        s["args"] = _describe(tlf, s, c)
    a = s["args"]
    if c["op"] == "sample":
        tlf.tlf_sample(a, stream)
        return s["tokens"], s["logprobs"]
    if c["op"] == "append":
        tlf.tlf_rope_append(a[0], a[1], stream)
        return s["q_out"], s["pool"], s["pos"]
    if c["op"] == "evict":
        tlf.tlf_cache_evict(a[0], a[1], a[1].numel(), stream)
        return s["pool"], s["pos_out"], s["weight_out"], s["lens_out"]
    tlf.tlf_attn_chunk(a[0], a[1], a[2], a[2].numel(), stream)
    return (s["out"], s["lse"], s["weight_out"]) if c["weights"] else (s["out"], s["lse"])


def _describe(tlf, s, c):
    if c["op"] == "sample":
        return tlf.sample_args(s["logits"], s["noise"], s["tokens"], s["logprobs"], temperature=s["temperature"],
                               top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    space = lambda n: torch.empty(max(1, n), dtype=torch.uint8, device="cuda")  # noqa: E731
    if c["op"] == "evict":
        a = tlf.evict_args(s["pool"], s["page_table"], s["lens"], s["next_pos"], s["pos"], s["pos_out"], s["weight"],
                           s["weight_out"], s["lens_out"], budget=c["budget"], n_first=c["first"], n_recent=c["recent"])
        return a, space(tlf.tlf_cache_evict_scratch_bytes(a))
    b = tlf.chunk_args(s["pool"], s["page_table"], s["cu"], s["lens"], n_heads=c["hq"], n_tokens=s["T"], layer=s["layer"],
                       max_chunk=s["most_new"])
    if c["op"] == "append":
        h, k = c["hq"] * c["hd"], c["hkv"] * c["hd"]
        q, kk, v = s["qkv"].split([h, k, k], 1)
        return b, tlf.rope_args(q, kk, v, s["positions"], s["table"], s["q_out"], layout=c["layout"], entry_pos=s["pos"])
    a = tlf.attn_chunk_args(s["q"], s["out"], lse=s["lse"], weight_in=s["weight"] if c["weights"] else None,
                            weight_out=s["weight_out"] if c["weights"] else None)
    return b, a, space(tlf.tlf_attn_chunk_scratch_bytes(b, a))


# ---- the plain forms ----

def _token_rows(s):
    """Row, index in the row's chunk and cache entry of every new token."""
    t = torch.arange(s["T"], device="cuda")
    row = torch.searchsorted(s["cu"][1:].long().contiguous(), t, right=True)
    i = t - s["cu"].long()[row]
    return row, i, s["lens"].long()[row] - (s["cu"][1:] - s["cu"][:-1]).long()[row] + i


def _append(s):
    c = s["case"]
    T, hq, hkv, hd, rot = s["T"], c["hq"], c["hkv"], c["hd"], c["rot"]
    row, _, e = _token_rows(s)
    page = s["page_table"].long()[row, e // PAGE]
    x = s["qkv"][:T].float().view(T, hq + 2 * hkv, hd)
    cs = s["table"][s["positions"].long()]
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    y = x[:, :hq + hkv, :rot]
    if c["layout"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0::2], y[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    turned = torch.cat([turned, x[:, :hq + hkv, rot:]], -1).to(s["pool"].dtype)
    s["q_out"][:T] = turned[:, :hq]
    s["pool"][page, s["layer"], 0, :, e % PAGE] = turned[:, hq:]
    s["pool"][page, s["layer"], 1, :, e % PAGE] = x[:, hq + hkv:].to(s["pool"].dtype)
    s["pos"][page, e % PAGE] = s["positions"]
    return s["q_out"], s["pool"], s["pos"]


def _attend(s):
    c = s["case"]
    T, hq, hkv, hd, n, most = s["T"], c["hq"], c["hkv"], c["hd"], c["rows"], s["most"]
    G, mq = hq // hkv, s["most_new"]
    row, i, e = _token_rows(s)
    keys = torch.arange(most, device="cuda")
    page = s["page_table"].long()[:, keys // PAGE].clamp_min(0)
    lens = s["lens"].long()
    live = keys < lens[:, None]
    if c["weights"]:
        s["weight_out"].zero_()
    if T:
        kv = s["pool"][page, s["layer"], :, :, keys % PAGE]  # [n, most, 2, hkv, hd]
        k, v = kv[:, :, 0].float().permute(0, 2, 3, 1), kv[:, :, 1].float().permute(0, 2, 1, 3)
        v = v * live[:, None, :, None]
        q = torch.zeros(n, mq, hq, hd, device="cuda")
        q[row, i] = s["q"][:T].float()
        at = torch.full((n, mq), -1, device="cuda", dtype=torch.long)  # the last entry that a query sees
        at[row, i] = e
        q = q.view(n, mq, hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * mq, hd)
        p = torch.matmul(q, k).mul_(1 / math.sqrt(hd)).view(n, hkv, G, mq, most)
        p.masked_fill_((keys > at[:, :, None])[:, None, None], -math.inf)
        m = p.amax(-1, keepdim=True).clamp_min(-3e38)
        p = p.sub_(m).exp_()
        l = p.sum(-1, keepdim=True)
        p = p.div_(torch.where(l > 0, l, 1.0))
        o = torch.matmul(p.view(n, hkv, G * mq, most), v).view(n, hkv, G, mq, hd).permute(0, 3, 1, 2, 4).reshape(n, mq, hq, hd)
        s["out"][:T] = o[row, i].to(s["out"].dtype)
        s["lse"][:T] = (m + l.log())[..., 0].permute(0, 3, 1, 2).reshape(n, mq, hq)[row, i]
    if c["weights"]:
        b, e = live.nonzero(as_tuple=True)
        add = p.sum((1, 2, 3)) if T else torch.zeros(n, most, device="cuda")
        at = page[b, e], e % PAGE
        s["weight_out"][at] = s["weight"][at] + add[b, e]
        return s["out"], s["lse"], s["weight_out"]
    return s["out"], s["lse"]


def _evict(s):
    c = s["case"]
    n, most, budget = c["rows"], s["most"], c["budget"]
    e = torch.arange(most, device="cuda")
    lens = s["lens"].long()
    live = e < lens[:, None]
    page = s["page_table"].long()[:, e // PAGE].clamp_min(0)
    w, pos = s["weight"][page, e % PAGE], s["pos"][page, e % PAGE]
    w = torch.where((pos < c["first"]) | (pos >= s["next_pos"][:, None] - c["recent"]), math.inf, w).masked_fill(~live, -1)
    order = w.sort(dim=1, descending=True, stable=True).indices  # ties: the entry that comes first
    keep = torch.zeros_like(live).scatter_(1, order[:, :budget], True) & live
    # entries that stay and lie beyond the budget fill the holes below it, both in order
    hole, mover = ~keep & live & (e < budget) & (lens > budget)[:, None], keep & (e >= budget)
    hb, he = hole.nonzero(as_tuple=True)
    mb, me = mover.nonzero(as_tuple=True)
    src = torch.where(live, e, 0)
    src[hb, he] = me  # as many holes as movers in every row
    s["pool"][page[hb, he], :, :, :, he % PAGE] = s["pool"][page[mb, me], :, :, :, me % PAGE]
    s["lens_out"].copy_(torch.minimum(lens, torch.tensor(budget, device="cuda")))
    b, at = (e < s["lens_out"].long()[:, None]).nonzero(as_tuple=True)
    to, fr = (page[b, at], at % PAGE), (page[b, src[b, at]], src[b, at] % PAGE)
    s["pos_out"][to] = s["pos"][fr]
    s["weight_out"][to] = s["weight"][fr]
    return s["pool"], s["pos_out"], s["weight_out"], s["lens_out"]


def _sample(s):
    x = s["logits"]
    B, V = x.shape
    l = torch.where(x > -math.inf, x, -math.inf).clamp_max(3.4028234663852886e38)
    l, idx = l.sort(dim=1, descending=True, stable=True)
    valid = l > -math.inf
    greedy = s["temperature"] <= 0
    z = (l - l[:, :1]) / torch.where(greedy, 1.0, s["temperature"])[:, None]
    w = torch.where(valid, z, -math.inf).exp()
    rank = torch.arange(V, device="cuda")
    k = torch.where(greedy, 1, torch.where(s["top_k"] > 0, s["top_k"], V))
    top = rank < k[:, None]
    wk = w * top
    before = wk.cumsum(1) - wk
    p = s["top_p"][:, None]
    keep = top & valid & ((rank == 0) | (((before < p * wk.sum(1, keepdim=True)) | (p >= 1)) & (w >= s["min_p"][:, None])))
    score = z - (-s["noise"].gather(1, idx).log()).log()
    score = torch.where(score == score, score, -math.inf)
    best = score.masked_fill(~keep, -math.inf).amax(1, keepdim=True)
    win = torch.where(keep & (score == best), idx, V).amin(1)
    there = win < V
    zt = (x.gather(1, win.clamp_max(V - 1)[:, None]) - l[:, :1]) / torch.where(greedy, 1.0, s["temperature"])[:, None]
    s["tokens"].copy_(torch.where(there, win, -1))
    s["logprobs"].copy_(torch.where(there, zt[:, 0] - w.sum(1).log(), -math.inf))
    return s["tokens"], s["logprobs"]


# ----------------------------------------------------------------------------
# In 64 bits, row by row
# ----------------------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "sample":
        out = []
        for b in range(c["rows"]):
            x = s["logits"][b].double()
            T = float(s["temperature"][b])
            logp = torch.log_softmax(x / (T if T > 0 else 1.0), 0)
            order = torch.argsort(x, descending=True, stable=True)
            n = int((x > -math.inf).sum())
            if T <= 0:
                n = 1
            elif int(s["top_k"][b]) > 0:
                n = min(n, int(s["top_k"][b]))
            q = logp[order[:n]].exp()
            if float(s["top_p"][b]) < 1:
                n = min(n, max(1, int((((q.cumsum(0) - q) / q.sum()) < s["top_p"][b].double()).sum())))
            n = min(n, max(1, int(((q / q[0]) >= s["min_p"][b].double()).sum())))
            kept = order[:n]
            race = logp[kept] - torch.log(-torch.log(s["noise"][b, kept].double()))
            out.append(logp[kept[race.argmax()]])
        return None, torch.stack(out)

    pt, lens = s["page_table"].long(), s["lens"].tolist()
    if c["op"] == "evict":
        pool, pos_out, w_out = s["pool"].double(), s["pos_out"].clone(), s["weight_out"].double()
        for b, n in enumerate(lens):
            e = torch.arange(n, device="cuda")
            page, off = pt[b, e // PAGE], e % PAGE
            w, pos = s["weight"][page, off].double(), s["pos"][page, off]
            fr = e[:min(n, c["budget"])].clone()
            if n > c["budget"]:
                r = w.clone()
                r[(pos < c["first"]) | (pos >= int(s["next_pos"][b]) - c["recent"])] = math.inf
                stays = torch.zeros(n, dtype=torch.bool, device="cuda")
                stays[torch.argsort(r, descending=True, stable=True)[:c["budget"]]] = True
                holes, movers = e[:c["budget"]][~stays[:c["budget"]]], e[c["budget"]:][stays[c["budget"]:]]
                fr[holes] = movers
                pool[page[holes], :, :, :, off[holes]] = s["pool"][page[movers], :, :, :, off[movers]].double()
            k = len(fr)
            pos_out[page[:k], off[:k]] = pos[fr]
            w_out[page[:k], off[:k]] = w[fr]
        return pool, None, w_out, None

    cu = s["cu"].tolist()
    if c["op"] == "append":
        hq, hkv, hd, rot = c["hq"], c["hkv"], c["hd"], c["rot"]
        q_out, pool = s["q_out"].double(), s["pool"].double()
        for b, n in enumerate(lens):
            t0, t1 = cu[b], cu[b + 1]
            if t1 == t0:
                continue
            x = s["qkv"][t0:t1].double().view(t1 - t0, -1, hd)
            ang = torch.view_as_complex(s["table"][s["positions"][t0:t1].long()].double())[:, None]
            y = x[:, :hq + hkv].clone()
            if c["layout"] == "half":
                z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * ang
                y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
            else:
                z = torch.complex(y[..., 0:rot:2].contiguous(), y[..., 1:rot:2].contiguous()) * ang
                y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
            q_out[t0:t1] = y[:, :hq]
            e = torch.arange(n - (t1 - t0), n, device="cuda")
            pool[pt[b, e // PAGE], s["layer"], 0, :, e % PAGE] = y[:, hq:]
            pool[pt[b, e // PAGE], s["layer"], 1, :, e % PAGE] = x[:, hq + hkv:]
        return q_out, pool, None

    hq, hkv, hd = c["hq"], c["hkv"], c["hd"]
    if work(c)["flops"] > 2e12:
        return None
    out, lse = s["out"].double(), s["lse"].double()
    weight = s["weight_out"].double() if c["weights"] else None
    for b, n in enumerate(lens):
        t0, t1 = cu[b], cu[b + 1]
        e = torch.arange(n, device="cuda")
        at = pt[b, e // PAGE], e % PAGE
        add = torch.zeros(n, dtype=torch.float64, device="cuda")
        for h in range(hkv if t1 > t0 else 0):
            k = s["pool"][at[0], s["layer"], 0, h, at[1]].double()
            v = s["pool"][at[0], s["layer"], 1, h, at[1]].double()
            sees = e[None] <= (n - (t1 - t0) + torch.arange(t1 - t0, device="cuda"))[:, None]
            for j in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                sc = (s["q"][t0:t1, j].double() @ k.T / math.sqrt(hd)).masked_fill(~sees, -math.inf)
                lse[t0:t1, j] = torch.logsumexp(sc, 1)
                p = torch.exp(sc - lse[t0:t1, j, None])
                out[t0:t1, j] = p @ v
                add += p.sum(0)
        if weight is not None:
            weight[at] = s["weight"][at].double() + add
    return (out, lse, weight) if c["weights"] else (out, lse)
