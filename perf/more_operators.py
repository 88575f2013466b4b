"""Timed cases of the operators around a served model's cache in 4 bits, its window and its pages.

Four operators, each through the call that a serving program makes (the ctypes binding of libtlf):

- ``pack``     rotary positions on the queries and keys of new tokens, keys and values into a cache held in 4 bits
               (``tlf_kv4_append``), and what the new entries stand for back out of it (``tlf_kv4_read``);
- ``attend``   attention of every row's chunk of new tokens over its paged cache, causal inside the chunk, all of it or a
               sliding window with a few first entries that stay visible (``tlf_attn_window``); the cache in 4 bits (``kv4``)
               or in the type of the queries;
- ``fork``     new rows that take over the pages of parents: full pages shared, a partly filled last page copied, room for
               the next tokens, pages that the window has left given up (``tlf_cache_fork``);
- ``compact``  the pages in use moved to the front of the pool (``tlf_cache_compact``).

The plain forms are elementary torch operations in 32 bits on padded rows. ``exact`` restates each operator in 64 bits,
row by row. Lengths, pages and parameters of a ragged batch follow from the case, values from the seed.

The 4-bit cache: a group of ``gs = min(head_dim, 64)`` values of an entry is held as codes n in 0..15 and a pair (d, lo) of
bfloat16 and stands for lo + d n. A page's block of one layer, K or V, and head: 64 x head_dim / 2 bytes of codes (two dims a
byte, the even one in the low half), then 64 x (head_dim / gs) pairs.
"""
import math

import numpy as np
import torch

own = False  # True: run() calls the library; False: the plain forms

PAGE = 64
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGEST = 2.0 ** 126  # magnitudes that a 4-bit group takes


# ----------------------------------------------------------------------------
# Cases
# ----------------------------------------------------------------------------

def listed():
    return [
        # one decoding step of a serving batch, multi-head: latency
        dict(name="pack-64x1", op="pack", rows=64, new_lo=1, new_hi=1, old_lo=1000, old_hi=2048, hq=16, hkv=16, hd=64, rot=64,
             layout="half", dtype="bf16"),
        # prompts of several sequences at once, grouped-query, half of each head rotated, interleaved pairs
        dict(name="pack-4x2048", op="pack", rows=4, new_lo=1500, new_hi=2048, old_lo=0, old_hi=1000, hq=16, hkv=8, hd=128,
             rot=64, layout="interleaved", dtype="bf16"),
        # a tiny float32 model, a few tokens a row: latency
        dict(name="attend4-f32-4x5", op="attend", rows=4, new_lo=1, new_hi=5, old_lo=0, old_hi=60, hq=4, hkv=4, hd=16,
             dtype="f32", kv4=True, window=0, first=0),
        # single tokens over long contexts, grouped-query: bandwidth
        dict(name="attend4-16x1-32k", op="attend", rows=16, new_lo=1, new_hi=1, old_lo=32000, old_hi=32700, hq=16, hkv=8,
             hd=128, dtype="bf16", kv4=True, window=0, first=0),
        # short turns (or drafted tokens to verify) on a ragged batch, multi-head, under a window
        dict(name="attend4-32x8-w4096", op="attend", rows=32, new_lo=1, new_hi=16, old_lo=128, old_hi=8192, hq=16, hkv=16,
             hd=64, dtype="bf16", kv4=True, window=4096, first=4),
        # long turns on long conversations, grouped-query: tensor cores
        dict(name="attend4-4x2048", op="attend", rows=4, new_lo=1800, new_hi=2048, old_lo=4000, old_hi=8192, hq=16, hkv=8,
             hd=128, dtype="bf16", kv4=True, window=0, first=0),
        # single tokens of streams that have run for long and keep a window and four sinks
        dict(name="window-64x1-w1024", op="attend", rows=64, new_lo=1, new_hi=1, old_lo=4000, old_hi=30000, hq=16, hkv=8,
             hd=128, dtype="bf16", kv4=False, window=1024, first=4),
        # long turns of such streams: tensor cores on a band
        dict(name="window-4x2048-w1024", op="attend", rows=4, new_lo=1800, new_hi=2048, old_lo=4000, old_hi=8192, hq=16, hkv=8,
             hd=128, dtype="bf16", kv4=False, window=1024, first=4),
        # a step of beam search: every row goes on from some row, some from the same one: latency
        dict(name="fork-64-of-64", op="fork", rows=64, parents=64, len_lo=20, len_hi=1000, reserve=1, window=0, first=0, hkv=16,
             hd=64, layers=2, dtype="bf16"),
        # sixteen answers to every prompt: the prompts' pages are shared, their last pages copied
        dict(name="fork-512-of-32", op="fork", rows=512, parents=32, len_lo=500, len_hi=8000, reserve=64, window=0, first=0,
             hkv=8, hd=128, layers=6, dtype="bf16"),
        # a small pool after some sequences have ended
        dict(name="compact-16", op="compact", rows=16, len_lo=10, len_hi=1000, live=0.6, hkv=8, hd=64, layers=2, dtype="bf16"),
        # a large one that is to give memory back
        dict(name="compact-96", op="compact", rows=96, len_lo=200, len_hi=8000, live=0.6, hkv=8, hd=128, layers=2,
             dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["pack", "attend", "attend", "attend", "attend", "fork", "compact"])
    hq, hkv, hd, dtype = rng.choice([(16, 16, 64, "bf16"), (16, 8, 128, "bf16"), (8, 8, 64, "bf16"), (8, 2, 128, "bf16"),
                                     (12, 4, 64, "bf16"), (4, 2, 32, "bf16"), (4, 4, 16, "f32"), (8, 2, 64, "f32")])
    if op == "pack":
        rows = _log(rng, 1, 128)
        hi = _log(rng, 1, max(1, 8192 // rows))
        return dict(op="pack", rows=rows, new_lo=rng.randint(0, hi), new_hi=hi, old_lo=0, old_hi=_log(rng, 1, 1500), hq=hq,
                    hkv=hkv, hd=hd, rot=rng.choice([hd, hd // 2]), layout=rng.choice(["half", "interleaved"]), dtype=dtype)
    window = rng.choice([0, _log(rng, 1, 8192)])
    first = rng.choice([0, 4, _log(rng, 1, 200)]) if window else 0
    if op == "fork":
        parents = _log(rng, 1, 64)
        rows = _log(rng, 1, 512)
        return dict(op="fork", rows=rows, parents=parents, len_lo=rng.randint(0, 300), len_hi=_log(rng, 300, 8000),
                    reserve=_log(rng, 1, 200), window=window, first=first, hkv=hkv, hd=hd, layers=rng.randint(1, 4), dtype=dtype)
    if op == "compact":
        return dict(op="compact", rows=_log(rng, 1, 96), len_lo=rng.randint(0, 300), len_hi=_log(rng, 300, 8000),
                    live=round(rng.uniform(0.2, 0.95), 2), hkv=hkv, hd=hd, layers=rng.randint(1, 2), dtype=dtype)
    kind = rng.choice(["one", "few", "many"])
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
                old_lo=rng.randint(0, old), old_hi=old, hq=hq, hkv=hkv, hd=hd, dtype=dtype, kv4=rng.random() < 0.6,
                window=window, first=first)


def _lengths(c, what, rows=None):
    """Ragged lengths of the rows, from the case alone; the longest one occurs."""
    lo, hi = c[what + "_lo"], c[what + "_hi"]
    n = rows or c["rows"]
    r = np.random.RandomState((lo * 31 + hi * 17 + n) % (1 << 31))
    v = r.randint(lo, hi + 1, n)
    v[r.randint(n)] = hi
    return v.astype(np.int64)


def _groups(hd):
    return max(1, hd // 64)


def _entry_bytes(c):
    """K and V of an entry in one layer."""
    if c.get("kv4") or c["op"] == "pack":
        return 2 * c["hkv"] * (c["hd"] // 2 + 4 * _groups(c["hd"]))
    return 2 * c["hkv"] * c["hd"] * (2 if c["dtype"] == "bf16" else 4)


def _parents(c):
    """The parent of every new row: most go on from some row, a few are empty."""
    r = np.random.RandomState(c["rows"] * 7 + c["parents"])
    p = r.randint(0, c["parents"], c["rows"]) if c["rows"] <= 2 * c["parents"] else np.arange(c["rows"]) * c["parents"] // c["rows"]
    return np.where(r.rand(c["rows"]) < 0.03, -1, p)


def _live(c):
    """Pages of the pool and, in the order of the rows' slots, the pages in use."""
    need = (_lengths(c, "len") + PAGE - 1) // PAGE
    total = max(1, int(math.ceil(need.sum() / c["live"])))
    return need, total, np.random.RandomState(c["rows"] + total).permutation(total)[:int(need.sum())]


def work(c):
    if c["op"] == "fork":
        par, lens = _parents(c), _lengths(c, "len", c["parents"])
        n = np.where(par >= 0, lens[np.maximum(par, 0)], 0)
        seen, copied = set(), 0
        for b, p in enumerate(par):
            if p >= 0 and p in seen:
                copied += int(n[b] % PAGE)
            seen.add(p)
        pages = ((lens + PAGE - 1) // PAGE).sum() + ((n + c["reserve"] + PAGE - 1) // PAGE).sum()
        return {"bytes": float(2 * copied * (c["layers"] * _entry_bytes(c) + 4) + 8 * pages + 16 * len(par)), "flops": float(pages)}
    if c["op"] == "compact":
        need, total, live = _live(c)
        moved = int((live >= len(live)).sum())
        page = PAGE * (c["layers"] * _entry_bytes(c) + 4)
        return {"bytes": float(2 * moved * page + 8 * len(live) + 8 * total), "flops": float(total)}
    new, old = _lengths(c, "new"), _lengths(c, "old")
    T, eb = float(new.sum()), 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "pack":  # q, k, v in, q out, the entries, and their values out
        return {"bytes": float(T * ((2 * c["hq"] + 4 * c["hkv"]) * c["hd"] * eb + 2 * _entry_bytes(c) + c["rot"] * 4 + 8)),
                "flops": float(T * ((c["hq"] + c["hkv"]) * c["rot"] * 3 + c["hkv"] * c["hd"] * 12))}
    w, f = c["window"] or 1 << 40, c["first"]
    lens = old + new
    low = np.maximum(np.minimum(f, lens), old - w + 1)  # entries that some query sees: the first ones, and from here on
    keys = np.where(new > 0, np.minimum(f, lens) + np.maximum(0, lens - low), 0).sum()
    pairs = 0.0
    for o, n in zip(old, new):
        e = o + np.arange(n)
        pairs += float((np.minimum(w, e + 1) + np.minimum(np.maximum(0, e + 1 - w), f)).sum())
    return {"bytes": float(keys * _entry_bytes(c) + T * c["hq"] * (2 * c["hd"] * eb + 4)), "flops": float(4 * c["hd"] * c["hq"] * pairs)}


# ----------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------

def _pages(lens, gen_case, low=None):
    """Page table of ragged rows over a shuffled pool with some spare pages: (table [rows][most], pages). With `low`: a row
    has pages for its entries below low[0] and from low[1][b] on only."""
    need = (lens + PAGE - 1) // PAGE
    most = max(1, int(need.max()))
    slot = np.arange(most)
    there = slot < need[:, None]
    if low is not None:
        there &= (slot * PAGE < low[0]) | ((slot + 1) * PAGE > low[1][:, None])
    total = int(there.sum()) + 3
    table = np.full((len(lens), most), -1, np.int32)
    table[there] = gen_case.permutation(total)[:total - 3]
    return table, total


def _rope_table(rot, max_pos, device):
    """(cos, sin) of position x frequency, base 10000, positions stretched by 2 (linear scaling), from 64 bits."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    ang = torch.arange(max_pos, dtype=torch.float64, device=device)[:, None] / 2.0 * inv
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()


def _views(pool4, hd):
    """(codes [..., 64, hd / 2] bytes, pairs [..., 64, groups, 2] bfloat16) of a 4-bit pool."""
    n = PAGE * hd // 2
    return pool4[..., :n].unflatten(-1, (PAGE, hd // 2)), pool4[..., n:].view(torch.bfloat16).unflatten(-1, (PAGE, _groups(hd), 2))


def _quantised(x):
    """Codes [..., hd / 2] and pairs [..., groups, 2] of values [..., hd] in 32 bits."""
    g = torch.nan_to_num(x, nan=0.0, posinf=LARGEST, neginf=-LARGEST).clamp(-LARGEST, LARGEST)
    g = g.unflatten(-1, (_groups(x.shape[-1]), -1))
    lo = g.amin(-1, keepdim=True).bfloat16()
    reach = (g.amax(-1, keepdim=True) - lo.float()).clamp_min(0)
    d = (reach / torch.full_like(reach, 15)).bfloat16()  # (by a tensor: by a number it would be a product with its inverse)
    n = ((g - lo.float()) / torch.where(d > 0, d, 1).float()).round().clamp(0, 15)
    n = torch.where(d > 0, n, 0).to(torch.uint8).flatten(-2)
    return n[..., 0::2] | n[..., 1::2] << 4, torch.cat([d, lo], -1)


def _values(codes, pairs):
    """What codes [..., hd / 2] and pairs [..., groups, 2] stand for, in 32 bits."""
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float().unflatten(-1, (pairs.shape[-2], -1))
    return (pairs[..., 1:].float() + pairs[..., :1].float() * n).flatten(-2)


def prepare(c, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 13)
    s = {"case": c}
    dt, hkv, hd = DTYPES[c["dtype"]], c["hkv"], c["hd"]
    rc = np.random.RandomState(c["rows"] * 101 + hd)
    i32 = lambda v: torch.tensor(np.ascontiguousarray(v, dtype=np.int32), device=dev)  # noqa: E731
    if c["op"] in ("fork", "compact"):
        if c["op"] == "fork":
            lens = _lengths(c, "len", c["parents"])
            par = _parents(c)
            n = np.where(par >= 0, lens[np.maximum(par, 0)], 0)
            room = int(((n + c["reserve"] + PAGE - 1) // PAGE - n // PAGE).sum())  # pages that the new rows may ask for
            need = (lens + PAGE - 1) // PAGE
            pages = int(need.sum()) + room + 5
            held = rc.permutation(pages)[:int(need.sum())]
            s["parents"], s["lens"] = i32(par), i32(lens)
            width = int(max(need.max(), ((n + c["reserve"] + PAGE - 1) // PAGE).max(), 1))
        else:
            need, pages, held = _live(c)
            width = max(1, int(need.max()))
        table = np.full((len(need), width), -1, np.int32)
        table[np.arange(width) < need[:, None]] = held
        refs = np.zeros(pages, np.int32)
        refs[held] = 1
        s["pool"] = torch.randn(pages, c["layers"], 2, hkv, PAGE, hd, device=dev, generator=g, dtype=dt)
        s["pos"] = torch.randint(0, 1 << 20, (pages, PAGE), dtype=torch.int32, device=dev, generator=g)
        s["page_table"], s["refs"] = i32(table), i32(refs)
        s["refs_out"] = torch.zeros_like(s["refs"])
        rows = c["rows"]
        s["table_out"] = torch.zeros(rows, width, dtype=torch.int32, device=dev)
        s["lens_out"] = torch.zeros(rows, dtype=torch.int32, device=dev)
        s["n_live"] = torch.zeros(1, dtype=torch.int32, device=dev)
        return s

    new, old = _lengths(c, "new"), _lengths(c, "old")
    lens = old + new
    w = c.get("window", 0)
    table, pages = _pages(lens, rc, (c["first"], old - w + 1) if w else None)  # what no query sees was given up long ago
    T = int(new.sum())
    s.update(T=T, most_new=max(1, int(new.max())), layers=2, layer=1, lens=i32(lens), page_table=i32(table),
             cu=i32(np.concatenate([[0], np.cumsum(new)])))
    if w:
        low = np.maximum(np.minimum(c["first"], lens), old - w + 1)  # the columns of the plain form: the first entries, the window
        s["first"], s["low"], s["most"] = c["first"], i32(low), c["first"] + max(1, int((lens - low).max()))
    else:
        s["first"], s["low"], s["most"] = 0, i32(0 * lens), max(1, int(lens.max()))
    if c["op"] == "pack" or c["kv4"]:
        size = PAGE * (hd // 2 + 4 * _groups(hd))
        s["pool"] = torch.zeros(pages, 2, 2, hkv, size, dtype=torch.uint8, device=dev)
        codes, pairs = _views(s["pool"], hd)
        for layer in range(2):
            x = torch.randn(pages, 2, hkv, PAGE, hd, device=dev, generator=g)
            codes[:, layer], pairs[:, layer] = _quantised(x)
            del x
    else:
        s["pool"] = torch.randn(pages, 2, 2, hkv, PAGE, hd, device=dev, generator=g).to(dt)
    if c["op"] == "pack":
        s["qkv"] = torch.randn(max(1, T), (c["hq"] + 2 * hkv) * hd, device=dev, generator=g).to(dt)
        # a token's position: ahead of its entry, since some tokens left none in this cache
        p = np.concatenate([o + np.arange(n) + o // 8 for o, n in zip(old, new)]) if T else np.zeros(0)
        s["positions"] = i32(p)
        s["max_pos"] = c["old_hi"] + c["new_hi"] + c["old_hi"] // 8 + 1
        s["table"] = _rope_table(c["rot"], s["max_pos"], dev)
        s["q_out"] = torch.zeros(max(1, T), c["hq"], hd, dtype=dt, device=dev)
        s["k_out"], s["v_out"] = (torch.zeros(max(1, T), hkv, hd, dtype=dt, device=dev) for _ in range(2))
        s["pos"] = torch.full((pages, PAGE), -1, dtype=torch.int32, device=dev)
        return s
    # queries that look at some keys more than at others
    s["q"] = (torch.randn(max(1, T), c["hq"], hd, device=dev, generator=g) * 1.5).to(dt)
    s["out"] = torch.zeros(max(1, T), c["hq"], hd, dtype=dt, device=dev)
    s["lse"] = torch.zeros(max(1, T), c["hq"], dtype=torch.float32, device=dev)
    return s


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    return {"pack": _pack, "attend": _attend, "fork": _fork, "compact": _compact}[s["case"]["op"]](s)


def _run_own(s):
    from paper_2609_15160_gb300 import tlf
    c = s["case"]
    stream = torch.cuda.current_stream()
    if "args" not in s:  # the buffers' descriptions and the workspace, which a program makes once and keeps with the buffers
        s["args"] = _describe(tlf, s, c)
    a = s["args"]
    if c["op"] == "pack":
        tlf.tlf_kv4_append(a[0], a[1], stream)
        tlf.tlf_kv4_read(a[0], a[2], stream)
        return s["q_out"], s["k_out"], s["v_out"], s["pos"]
    if c["op"] == "attend":
        tlf.tlf_attn_window(a[0], a[1], a[2], a[2].numel(), stream)
        return s["out"], s["lse"]
    if c["op"] == "fork":
        tlf.tlf_cache_fork(a[0], a[1], a[1].numel(), stream)
        return s["pool"], s["pos"], s["table_out"], s["lens_out"], s["refs_out"]
    tlf.tlf_cache_compact(a[0], a[1], a[1].numel(), stream)
    return s["pool"], s["pos"], s["table_out"], s["refs_out"], s["n_live"]


def _describe(tlf, s, c):
    space = lambda n: torch.empty(max(1, n), dtype=torch.uint8, device="cuda")  # noqa: E731
    if c["op"] == "fork":
        a = tlf.fork_args(s["pool"], s["page_table"], s["lens"], s["parents"], s["refs"], s["table_out"], s["lens_out"],
                          s["refs_out"], reserve=c["reserve"], window=c["window"], n_first=c["first"], entry_pos=s["pos"])
        return a, space(tlf.tlf_cache_fork_scratch_bytes(a))
    if c["op"] == "compact":
        a = tlf.compact_args(s["pool"], s["page_table"], s["refs"], s["table_out"], s["refs_out"], s["n_live"], entry_pos=s["pos"])
        return a, space(tlf.tlf_cache_compact_scratch_bytes(a))
    if c["op"] == "pack" or c["kv4"]:
        b = tlf.chunk4_args(s["pool"], s["page_table"], s["cu"], s["lens"], n_heads=c["hq"], n_tokens=s["T"], head_dim=c["hd"],
                            dtype=c["dtype"], layer=s["layer"], max_chunk=s["most_new"])
    else:
        b = tlf.chunk_args(s["pool"], s["page_table"], s["cu"], s["lens"], n_heads=c["hq"], n_tokens=s["T"], layer=s["layer"],
                           max_chunk=s["most_new"])
    if c["op"] == "pack":
        h, k = c["hq"] * c["hd"], c["hkv"] * c["hd"]
        q, kk, v = s["qkv"].split([h, k, k], 1)
        return (b, tlf.rope_args(q, kk, v, s["positions"], s["table"], s["q_out"], layout=c["layout"], entry_pos=s["pos"]),
                tlf.kv4_read_args(s["k_out"], s["v_out"]))
    a = tlf.attn_window_args(s["q"], s["out"], lse=s["lse"], window=c["window"], n_first=c["first"], kv4=c["kv4"])
    return b, a, space(tlf.tlf_attn_window_scratch_bytes(b, a))


# ---- the plain forms ----

def _token_rows(s):
    """Row, index in the row's chunk and cache entry of every new token."""
    t = torch.arange(s["T"], device="cuda")
    row = torch.searchsorted(s["cu"][1:].long().contiguous(), t, right=True)
    i = t - s["cu"].long()[row]
    return row, i, s["lens"].long()[row] - (s["cu"][1:] - s["cu"][:-1]).long()[row] + i


def _pack(s):
    c = s["case"]
    T, hq, hkv, hd, rot = s["T"], c["hq"], c["hkv"], c["hd"], c["rot"]
    row, _, e = _token_rows(s)
    page, off = s["page_table"].long()[row, e // PAGE], e % PAGE
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
    turned = torch.cat([turned, x[:, :hq + hkv, rot:]], -1).to(s["q_out"].dtype)
    s["q_out"][:T] = turned[:, :hq]
    codes, pairs = _views(s["pool"], hd)
    for i, kv in enumerate((turned[:, hq:].float(), x[:, hq + hkv:])):
        codes[page, s["layer"], i, :, off], pairs[page, s["layer"], i, :, off] = _quantised(kv)
    s["pos"][page, off] = s["positions"]
    for i, to in enumerate((s["k_out"], s["v_out"])):
        to[:T] = _values(codes[page, s["layer"], i, :, off], pairs[page, s["layer"], i, :, off]).to(to.dtype)
    return s["q_out"], s["k_out"], s["v_out"], s["pos"]


def _attend(s):
    c = s["case"]
    T, hq, hkv, hd, n, most = s["T"], c["hq"], c["hkv"], c["hd"], c["rows"], s["most"]
    G, mq, first = hq // hkv, s["most_new"], s["first"]
    if not T:
        return s["out"], s["lse"]
    row, i, e = _token_rows(s)
    col = torch.arange(most, device="cuda")
    lens = s["lens"].long()[:, None]
    keys = torch.where(col < first, col, s["low"].long()[:, None] + col - first)  # [n, most]: the entry of a column
    live = (keys < lens) & ((col >= first) | (keys < s["low"].long()[:, None]))
    slot = (keys // PAGE).clamp_max(s["page_table"].shape[1] - 1)
    page, off = s["page_table"].long().gather(1, slot).clamp_min(0), keys % PAGE
    if c["kv4"]:
        codes, pairs = _views(s["pool"], hd)
        kv = _values(codes[page, s["layer"], :, :, off], pairs[page, s["layer"], :, :, off])  # [n, most, 2, hkv, hd]
    else:
        kv = s["pool"][page, s["layer"], :, :, off].float()
    k, v = kv[:, :, 0].permute(0, 2, 3, 1), kv[:, :, 1].permute(0, 2, 1, 3)
    v = v * live[:, None, :, None]
    q = torch.zeros(n, mq, hq, hd, device="cuda")
    q[row, i] = s["q"][:T].float()
    at = torch.full((n, mq), -1, device="cuda", dtype=torch.long)  # the last entry that a query sees
    at[row, i] = e
    q = q.view(n, mq, hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * mq, hd)
    p = torch.matmul(q, k).mul_(1 / math.sqrt(hd)).view(n, hkv, G, mq, most)
    hidden = (keys[:, None] > at[:, :, None]) | ~live[:, None]
    if c["window"]:
        hidden |= (keys[:, None] <= at[:, :, None] - c["window"]) & (keys[:, None] >= first)
    p.masked_fill_(hidden[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True).clamp_min(-3e38)
    p = p.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(l > 0, l, 1.0))
    o = torch.matmul(p.view(n, hkv, G * mq, most), v).view(n, hkv, G, mq, hd).permute(0, 3, 1, 2, 4).reshape(n, mq, hq, hd)
    s["out"][:T] = o[row, i].to(s["out"].dtype)
    s["lse"][:T] = (m + l.log())[..., 0].permute(0, 3, 1, 2).reshape(n, mq, hq)[row, i]
    return s["out"], s["lse"]


def _counted(refs, out, table, by):
    """out = refs + by for every entry of the table that names a page."""
    out.copy_(refs)
    t = table.long().flatten()
    return out.index_add_(0, t.clamp_min(0), (t >= 0).int() * by)


def _fork(s):
    c = s["case"]
    par, table, refs = s["parents"].long(), s["page_table"].long(), s["refs"]
    n, width = par.shape[0], table.shape[1]
    there = par >= 0
    src = par.clamp_min(0)
    lens = torch.where(there, s["lens"].long()[src], 0)
    full, need = (lens // PAGE)[:, None], ((lens + c["reserve"] + PAGE - 1) // PAGE)[:, None]
    old = torch.where(there[:, None], table[src], -1)
    slot, b = torch.arange(width, device="cuda"), torch.arange(n, device="cuda")
    eldest = torch.full((table.shape[0],), n, device="cuda").scatter_reduce_(0, src, torch.where(there, b, n), "amin")
    mine = (there & (eldest[src] == b))[:, None] & (old >= 0) & (refs[old.clamp_min(0)] == 1)
    shared, tail = slot < full, (slot >= full) & (slot < need)
    if c["window"]:
        shared &= ~((PAGE * (slot + 1) <= lens[:, None] - c["window"] + 1) & (PAGE * slot >= c["first"]))
    fresh = tail & ~mine
    free = (refs == 0).nonzero()[:, 0]
    rank = (fresh.flatten().cumsum(0) - 1).view(n, width)
    page = free[rank.clamp(0, len(free) - 1)]  # as many as are asked for, in these cases
    out = torch.where(shared | (tail & mine), old, torch.where(fresh, page, -1))
    left = lens % PAGE
    r, o = (((fresh & (slot == full)).any(1) & (left > 0))[:, None] & (torch.arange(PAGE, device="cuda") < left[:, None])).nonzero(as_tuple=True)
    at = full[r, 0]
    to, fr = out[r, at], old[r, at]
    s["pool"][to, :, :, :, o] = s["pool"][fr, :, :, :, o]
    s["pos"][to, o] = s["pos"][fr, o]
    s["table_out"].copy_(out)
    s["lens_out"].copy_(lens)
    _counted(_counted(refs, s["refs_out"], table, -1), s["refs_out"], out, 1)
    return s["pool"], s["pos"], s["table_out"], s["lens_out"], s["refs_out"]


def _compact(s):
    used = s["refs"] > 0
    live = used.sum()
    page = torch.arange(len(used), device="cuda")
    fr, to = (used & (page >= live)).nonzero()[:, 0], (~used & (page < live)).nonzero()[:, 0]
    s["pool"][to] = s["pool"][fr]
    s["pos"][to] = s["pos"][fr]
    where = page.clone()
    where[fr] = to
    t = s["page_table"].long()
    s["table_out"].copy_(torch.where(t >= 0, where[t.clamp_min(0)], -1))
    s["refs_out"].copy_(s["refs"])
    s["refs_out"][to] = s["refs"][fr]
    s["refs_out"].masked_fill_(page >= live, 0)
    s["n_live"].copy_(live)
    return s["pool"], s["pos"], s["table_out"], s["refs_out"], s["n_live"]


# ----------------------------------------------------------------------------
# In 64 bits, row by row
# ----------------------------------------------------------------------------

def _grid64(x):
    """The values that a 4-bit cache holds in the place of x [..., hd] (in 64 bits)."""
    out = torch.empty_like(x)
    for g in range(0, x.shape[-1], 64):
        y = x[..., g:g + 64]
        lo = y.min(-1, keepdim=True).values.bfloat16().double()
        d = ((y.max(-1, keepdim=True).values - lo).clamp_min(0) / 15).bfloat16().double()
        out[..., g:g + 64] = lo + d * torch.nan_to_num((y - lo) / d, nan=0.0).round().clamp(0, 15)
    return out


def _held64(s, c, page, kv, head, off):
    """K (0) or V (1) of some entries of a head, in 64 bits."""
    hd = c["hd"]
    if not c["kv4"]:
        return s["pool"][page, s["layer"], kv, head, off].double()
    block = s["pool"][page, s["layer"], kv, head]
    byte = block[:, :PAGE * hd // 2].reshape(-1, PAGE, hd // 2)[torch.arange(len(off), device="cuda"), off].long()
    pair = block[:, PAGE * hd // 2:].contiguous().view(torch.bfloat16).reshape(len(off), PAGE, -1)[torch.arange(len(off), device="cuda"), off].double()
    n = torch.zeros(len(off), hd, dtype=torch.float64, device="cuda")
    n[:, 0::2], n[:, 1::2] = (byte % 16).double(), (byte // 16).double()
    per = hd // (pair.shape[1] // 2)
    return n * pair[:, 0::2].repeat_interleave(per, 1) + pair[:, 1::2].repeat_interleave(per, 1)


def exact(c, seed):
    s = prepare(c, seed)
    pt = s["page_table"].long()
    if c["op"] == "compact":
        pool = s["pool"].double()
        refs = s["refs"].tolist()
        live = sum(r > 0 for r in refs)
        holes = [p for p in range(live) if refs[p] == 0]
        for hole, p in zip(holes, [p for p in range(live, len(refs)) if refs[p] > 0]):
            pool[hole] = s["pool"][p].double()
        return pool, None, None, None, None
    if c["op"] == "fork":
        pool, lens, par = s["pool"].double(), s["lens"].tolist(), s["parents"].tolist()
        free = iter([p for p, r in enumerate(s["refs"].tolist()) if r == 0])
        seen = set()
        for p in par:
            n = lens[p] if p >= 0 else 0
            for slot in range(n // PAGE, (n + c["reserve"] + PAGE - 1) // PAGE):
                if p in seen or p < 0 or slot * PAGE >= n:  # a new page (the first child keeps a partly filled one)
                    page = next(free)
                    k = max(0, n - slot * PAGE)
                    if k:
                        pool[page, :, :, :, :k] = s["pool"][pt[p, slot], :, :, :, :k].double()
            if p >= 0:
                seen.add(p)
        return pool, None, None, None, None

    cu, lens = s["cu"].tolist(), s["lens"].tolist()
    if c["op"] == "pack":
        hq, hkv, hd, rot = c["hq"], c["hkv"], c["hd"], c["rot"]
        q_out, k_out, v_out = (s[x].double() for x in ("q_out", "k_out", "v_out"))
        for t0, t1 in zip(cu[:-1], cu[1:]):
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
            k_out[t0:t1] = _grid64(y[:, hq:].to(s["k_out"].dtype).double())  # of the keys as a plain cache holds them
            v_out[t0:t1] = _grid64(x[:, hq + hkv:])
        # in float32 a turned key next to a border between two codes is no number that 64 bits could settle
        return q_out, k_out if c["dtype"] == "bf16" else None, v_out, None

    hq, hkv, hd = c["hq"], c["hkv"], c["hd"]
    if work(c)["flops"] > 2e12:
        return None
    out, lse = s["out"].double(), s["lse"].double()
    for b, n in enumerate(lens):
        t0, t1 = cu[b], cu[b + 1]
        if t1 == t0:
            continue
        q_at = (n - (t1 - t0) + torch.arange(t1 - t0, device="cuda"))[:, None]
        e = torch.arange(n, device="cuda")
        if c["window"]:
            e = e[(e < c["first"]) | (e > n - (t1 - t0) - c["window"])]
        page, off = pt[b, e // PAGE], e % PAGE
        sees = e[None] <= q_at
        if c["window"]:
            sees &= (e[None] > q_at - c["window"]) | (e[None] < c["first"])
        for h in range(hkv):
            k, v = _held64(s, c, page, 0, h, off), _held64(s, c, page, 1, h, off)
            for j in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                sc = (s["q"][t0:t1, j].double() @ k.T / math.sqrt(hd)).masked_fill(~sees, -math.inf)
                lse[t0:t1, j] = torch.logsumexp(sc, 1)
                out[t0:t1, j] = torch.exp(sc - lse[t0:t1, j, None]) @ v
    return out, lse
