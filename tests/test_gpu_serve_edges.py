"""Where the operators on paged caches and logits could go wrong for one row because of another, at the ends of their types, and
in the paths that only large calls take. Bounds as in test_gpu_serve_ops."""
import numpy as np
import pytest

import _serve_ref as R
from test_gpu_serve_ops import RB, T, U, _attend, _draw, _hold  # noqa: F401

pytestmark = pytest.mark.gpu


def _hold_tokens(c, out, ref, tokens):
    """The outputs of some tokens within their bounds."""
    r = RB if c.dtype == "bf16" else 0.0
    p_rel = 2 * (c.hd + 4) * U * ref[3] + 2.0 ** -20
    bound = ((p_rel[..., None] + r) * ref[2] + (r + 4 * U) * np.abs(ref[0]) * (1 + r) + 1e-30)[tokens]
    got = out.float().cpu().numpy().astype(np.float64)[tokens]
    assert np.isfinite(got).all() and (np.abs(got - ref[0][tokens]) <= bound).all(), np.max(np.abs(got - ref[0][tokens]) / bound)


# ---- one row's values and the others ----

def test_rows_without_a_number_leave_the_others_alone(T):
    """Many short items of two tiles and two blocks to a CTA; the queries of some rows' first tiles are NaN. Every other row is
    right, and no wait runs out."""
    rng = np.random.default_rng(0)
    new = rng.integers(66, 73, 64)
    c = R.Cache(np.zeros(64, int), new, 16, 8, 64, "bf16", layers=1, layer=0, seed=21)
    ref = R.attention(c)
    bad = [3, 4, 20, 41, 63]
    for b in bad:
        c.q[c.cu[b]:c.cu[b] + 64] = np.nan
    d = c.device()
    out, _, _ = _attend(T, c, d)
    assert int(d["err"][0].item()) == 0
    _hold_tokens(c, out, ref, np.concatenate([np.arange(c.cu[b], c.cu[b + 1]) for b in range(64) if b not in bad]))
    for b in bad:
        assert not np.isfinite(out[c.cu[b]:c.cu[b] + 64].float().cpu().numpy()).any()
        _hold_tokens(c, out, ref, np.arange(c.cu[b] + 64, c.cu[b + 1]))


def _without(c, gone):
    """R.attention with the entries of pages `gone` (row, page of the row) left out: out, lse, spread, terms, weights."""
    out, spread = np.zeros((c.T, c.hq, c.hd)), np.zeros((c.T, c.hq, c.hd))
    lse, terms = np.full((c.T, c.hq), -np.inf), np.zeros((c.T, c.hq))
    weights, G = [np.zeros(n) for n in c.lens], c.hq // c.hkv
    for b in range(c.n):
        k, v = (x.astype(np.float64) for x in c.kv(b))
        there = np.array([(b, e // 64) not in gone for e in range(c.lens[b])])
        for i in range(c.new[b]):
            t = c.cu[b] + i
            e = np.nonzero(there[:c.old[b] + i + 1])[0]
            if len(e) == 0:
                continue
            for h in range(c.hq):
                q = c.q[t, h].astype(np.float64)
                s = k[e, h // G] @ q / np.sqrt(c.hd)
                terms[t, h] = (np.abs(k[e, h // G]) @ np.abs(q)).max() / np.sqrt(c.hd)
                lse[t, h] = s.max() + np.log(np.exp(s - s.max()).sum())
                p = np.exp(s - lse[t, h])
                out[t, h], spread[t, h] = p @ v[e, h // G], p @ np.abs(v[e, h // G])
                weights[b][e] += p
    return out, lse, spread, terms, weights


@pytest.mark.parametrize("new", [[1, 1, 1], [1, 6, 3], [1, 90, 150], [1, 20, 257]], ids=["one", "few", "many", "mixed"])
@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("bf16", 64), ("bf16", 128)])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_page_that_is_not_there_is_left_out(T, new, dtype, hd, bad):
    """Page ids outside the pool, in rows of one token beside longer ones, while page 0 holds no number at all. The long rows
    put several blocks into a CTA's share, missing ones among them."""
    import torch
    c = R.Cache([300, 200, 0] + [5000] * 8, new + [1] * 8, 4, 2, hd, dtype, seed=31)
    spare = np.setdiff1d(np.arange(c.pages), c.table)[0]
    if 0 in c.table:  # page 0 is nobody's
        c.pool[spare] = c.pool[0]
        c.table[c.table == 0] = spare
    c.pool[0] = bad
    gone = {(0, 1): c.pages + 7, (0, 3): -1, (1, 0): 1 << 30, (1, 2): -9, (2, 0): c.pages}
    gone.update({(b, p): -1 for b in range(3, 11) for p in range(b, 79, 5)})
    ref = _without(c, gone)
    d = c.device()
    for (b, p), page in gone.items():
        d["table"][b, p] = page
    w_in = torch.rand(c.pages, 64, device="cuda")
    out, lse, w = _attend(T, c, d, weights=True, weight_in=w_in)
    plain = _attend(T, c, d, max_chunk=max(new))  # (a tighter bound may take another kernel)
    assert int(d["err"][0].item()) == 2
    d["err"].zero_()
    _hold(c, d, (out, lse), ref)
    _hold(c, d, plain, ref)
    w, before = w.cpu().numpy().astype(np.float64), w_in.cpu().numpy()
    for b in range(c.n):
        e = np.array([e for e in range(c.lens[b]) if (b, e // 64) not in gone], int)
        want = before[c.at(b, e)] + ref[4][b][e]
        assert (np.abs(w[c.at(b, e)] - want) <= 2.0 ** -11 * ref[4][b][e] + 4 * U * want).all()
        lost = np.setdiff1d(np.arange(c.lens[b]), e)
        assert (w[c.at(b, lost)] == -7).all()


SPOILT = [  # old, new, hq, hkv, hd
    ([70, 300], [9, 12], 4, 2, 128), ([70, 0], [20, 31], 2, 2, 64), ([10, 500], [60, 64], 2, 2, 32), ([0, 64], [20, 33], 6, 2, 64),
    ([70, 3000], [33, 130], 4, 2, 128), ([0, 1000], [300, 80], 2, 2, 64), ([4000], [257], 4, 2, 64), ([5, 63], [64, 40], 16, 1, 128)]


@pytest.mark.parametrize("old,new,hq,hkv,hd", SPOILT, ids=lambda v: str(v))
def test_a_new_tokens_infinite_value_reaches_those_that_see_it_and_nobody_else(T, old, new, hq, hkv, hd):
    """Values of tokens amid the chunks hold infinities and NaN in a few dims: earlier queries do not see them at all, later ones
    in those dims only; infinities of both signs meet as NaN."""
    c = R.Cache(old, new, hq, hkv, hd, "bf16", seed=hd + hq)
    ref = R.attention(c)  # of the finite values
    want = ref[0].copy()
    for b in range(c.n):
        for i, dim, x in ((c.new[b] // 3, 5, np.inf), (c.new[b] // 3, 9, -np.inf), (c.new[b] // 2, 30, np.nan), (c.new[b] - 2, 9, np.inf)):
            p, o = c.at(b, np.array([c.old[b] + i]))
            c.pool[p, c.layer, 1, :, o, dim] = x
            with np.errstate(invalid="ignore"):
                want[c.cu[b] + i:c.cu[b + 1], :, dim] += x
    d = c.device()
    out, lse, _ = _attend(T, c, d)
    got, fin = out.float().cpu().numpy().astype(np.float64), np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True)
    r = RB
    p_rel = 2 * (c.hd + 4) * U * ref[3] + 2.0 ** -20
    bound = (p_rel[..., None] + r) * ref[2] + (r + 4 * U) * np.abs(ref[0]) * (1 + r) + 1e-30
    # (the values that were replaced are part of ref in the dims that are not looked at)
    assert (np.abs(got[fin] - want[fin]) <= bound[fin]).all()
    clean = _attend(T, c, d)[1]
    assert np.abs(clean.cpu().numpy() - ref[1]).max() < 1e-4 and int(d["err"][0].item()) == 0


def _time(T, c, d, **kw):
    """Milliseconds of a call, the best of five."""
    import torch
    out = torch.empty(c.T, c.hq, c.hd, dtype=d["q"].dtype, device="cuda")
    b = T.chunk_args(d["pool"], d["table"], d["cu"], d["lens"], c.hq, c.T, layer=c.layer, err=d["err"], **kw)
    a = T.attn_chunk_args(d["q"], out)
    n = T.tlf_attn_chunk_scratch_bytes(b, a)
    scratch = torch.empty(n, dtype=torch.uint8, device="cuda")
    best = np.inf
    for _ in range(6):
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record()
        T.tlf_attn_chunk(b, a, scratch, n, torch.cuda.current_stream())
        e1.record()
        torch.cuda.synchronize()
        best = min(best, e0.elapsed_time(e1))
    return best


@pytest.mark.parametrize("new,hq,hd", [([8, 5], 4, 128), ([20, 17], 4, 64), ([200, 300], 4, 64), ([200, 300], 4, 128)])
def test_values_that_are_not_finite_cost_little_time(T, new, hq, hd):
    """An infinite value early in a long cache, a query that is NaN, and a chunk whose values all are: no more than a few times
    the usual time (and 0.2 ms for what is done once an item)."""
    c = R.Cache([8000, 6000], new, hq, 2, hd, "bf16", seed=3)
    usual = _time(T, c, c.device())
    pool, q = c.pool.copy(), c.q.copy()
    c.pool[c.table[:, 0], c.layer, 1, :, 5] = np.inf
    early = _time(T, c, c.device())
    c.pool[:] = pool
    c.q[c.cu[1] // 2] = np.nan
    query = _time(T, c, c.device())
    c.q[:] = q
    for b in range(2):
        p, o = c.at(b, np.arange(c.old[b], c.lens[b]))
        c.pool[p, c.layer, 1, :, o] = np.nan
    chunk = _time(T, c, c.device())
    assert max(early, query, chunk) <= 4 * usual + 0.2, (usual, early, query, chunk)


# ---- the ends of the types ----

@pytest.mark.parametrize("scale", [1.6e-38, 1e-38, 1e-41, 1e-45])
@pytest.mark.parametrize("old,new,hq,hkv,hd", [([70, 300], [20, 33], 4, 2, 64), ([70, 300], [130, 64], 4, 2, 128), ([7000], [65], 2, 1, 64),
                                               ([7000], [65], 2, 1, 128), ([100, 30], [5, 1], 4, 2, 64)])
def test_a_tiny_scale_without_accounts(T, scale, old, new, hq, hkv, hd):
    """All scores alike, in items of one CTA and in shared ones: means over what is seen, lse the logarithm of its number."""
    c = R.Cache(old, new, hq, hkv, hd, "bf16", seed=hd)
    d = c.device()
    _hold(c, d, _attend(T, c, d, scale=scale), R.attention(c, scale=scale), scale=scale)


def test_eviction_takes_the_two_zeros_for_equal(T):
    """Weights 0 and -0: the lower index stays, whichever zero it has."""
    import torch
    rng = np.random.default_rng(5)
    lens = [100, 300, 3000]
    c = R.Cache(lens, [0] * 3, 1, 1, 64, "bf16", layers=1, layer=0, seed=2)
    w = np.where(rng.random((c.pages, 64)) < 0.5, np.float32(-0.0), np.float32(0.0))
    w[rng.random(w.shape) < 0.1] = 1
    w[rng.random(w.shape) < 0.1] = -1
    pos = np.zeros((c.pages, 64), np.int32)
    for b, n in enumerate(lens):
        pos[c.at(b, np.arange(n))] = np.arange(n)
    d = c.device(w=w, pos=pos, nxt=np.asarray(lens, np.int32))
    wo, po, lo = torch.zeros_like(d["w"]), torch.zeros_like(d["pos"]), torch.zeros_like(d["lens"])
    a = T.evict_args(d["pool"], d["table"], d["lens"], d["nxt"], d["pos"], po, d["w"], wo, lo, budget=60, n_first=2, n_recent=8)
    n = T.tlf_cache_evict_scratch_bytes(a)
    T.tlf_cache_evict(a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    for b, n in enumerate(lens):
        e = np.arange(n)
        src = R.evict(w[c.at(b, e)], pos[c.at(b, e)], n, 60, 2, 8)
        assert np.array_equal(po.cpu().numpy()[c.at(b, np.arange(60))], src)


def test_eviction_with_a_budget_that_nothing_reaches(T):
    """The workspace goes by the entries that a row can have, and nothing changes."""
    import torch
    c = R.Cache([200, 64, 0], [0] * 3, 1, 1, 64, "bf16", layers=1, layer=0, seed=2)
    rng = np.random.default_rng(1)
    w, pos = rng.random((c.pages, 64)).astype(np.float32), rng.integers(0, 99, (c.pages, 64)).astype(np.int32)
    d = c.device(w=w, pos=pos, nxt=np.asarray([200, 64, 0], np.int32))
    a = T.evict_args(d["pool"], d["table"], d["lens"], d["nxt"], d["pos"], d["pos"], d["w"], d["w"], d["lens"], budget=2 ** 31 - 1,
                     n_recent=5)
    n = T.tlf_cache_evict_scratch_bytes(a)
    assert 0 < n < 1 << 16
    T.tlf_cache_evict(a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    assert d["lens"].tolist() == [200, 64, 0] and np.array_equal(d["w"].cpu().numpy(), w) and np.array_equal(d["pos"].cpu().numpy(), pos)
    assert np.array_equal(d["pool"].float().cpu().numpy(), c.pool)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("hq,hkv", [(16, 16), (1024, 1024), (64, 2)])
def test_the_largest_arguments_have_a_workspace(T, weights, hq, hkv):
    """Tokens x heads x pages pass 64 bits: the size is that of the kernels' parts and of lse. (Nothing is launched.)"""
    import ctypes as C
    P = 1 << 20
    c = T.TlfChunk(n=2, n_tokens=1 << 26, max_chunk=0, n_heads=hq, n_kv_heads=hkv, head_dim=32, n_layers=1, page_size=64, dtype=1,
                   max_pages=(1 << 25) - 65, n_pages=9, pool=P, page_table=P, cu_tokens=P, lens=P)
    n = T.load_library().tlf_attn_chunk_scratch_bytes(C.byref(c), C.byref(T.TlfAttnChunkArgs(q=P, out=P, weight_out=P if weights else None)))
    lse = (1 << 26) * hq * 4 if weights else 0
    sms = __import__("torch").cuda.get_device_properties(0).multi_processor_count
    part = 2 * 2 * sms * 64 * (32 * 4 + 8)  # two parts a CTA, of 64 rows
    assert lse + part <= n <= lse + 2 * part


# ---- paths that only large calls take ----

def _evict_rows(T, lens, budget, first, recent, in_place, seed):
    import torch
    c = R.Cache(lens, [0] * len(lens), 1, 1, 16, "f32", layers=1, layer=0, seed=seed)
    rng = np.random.default_rng(seed)
    w = np.round(rng.exponential(1, (c.pages, 64)), 3).astype(np.float32)  # ties
    w[rng.random(w.shape) < 0.05] = np.nan
    pos = np.zeros((c.pages, 64), np.int32)
    for b, n in enumerate(lens):
        pos[c.at(b, np.arange(n))] = np.arange(n)
    d = c.device(w=w, pos=pos, nxt=np.asarray(lens, np.int32))
    wo = d["w"] if in_place else torch.full((c.pages, 64), -7.0, device="cuda")
    po = d["pos"] if in_place else torch.full((c.pages, 64), -7, dtype=torch.int32, device="cuda")
    lo = torch.zeros_like(d["lens"])
    a = T.evict_args(d["pool"], d["table"], d["lens"], d["nxt"], d["pos"], po, d["w"], wo, lo, budget=budget, n_first=first,
                     n_recent=recent, err=d["err"])
    n = T.tlf_cache_evict_scratch_bytes(a)
    T.tlf_cache_evict(a, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n)
    assert int(d["err"][0].item()) == 0 and lo.tolist() == [min(n, budget) for n in lens]
    pool, wx, px = d["pool"].cpu().numpy(), wo.cpu().numpy(), po.cpu().numpy()
    for b, n in enumerate(lens):
        e = np.arange(n)
        src = R.evict(w[c.at(b, e)], pos[c.at(b, e)], n, budget, first, recent)
        to, fr = c.at(b, np.arange(len(src))), c.at(b, src)
        assert np.array_equal(px[to], pos[fr]) and np.array_equal(wx[to], w[fr], equal_nan=True)
        assert np.array_equal(pool[to[0], 0, :, :, to[1]], c.pool[fr[0], 0, :, :, fr[1]])
        if not in_place:
            rest = c.at(b, np.arange(len(src), n))
            assert (wx[rest] == -7).all() and (px[rest] == -7).all()


@pytest.mark.parametrize("in_place", [False, True])
def test_eviction_of_rows_that_clusters_share(T, in_place):
    """Several rows, each split over CTAs, of unlike lengths."""
    _evict_rows(T, [20000, 5, 9999, 8192, 0, 16001], 8192, 4, 100, in_place, 11)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lens", [[340000], [45000] + [70] * 80], ids=["cluster", "one-cta"])
def test_eviction_of_rows_that_shared_memory_does_not_hold(T, lens, in_place):
    """More keys a CTA than it keeps: they are read again in every level."""
    _evict_rows(T, lens, lens[0] // 3, 4, 64, in_place, 12)


@pytest.mark.parametrize("rows,V", [(1, 64000), (1, 128256), (1, 262144), (3, 262144), (9, 128256), (9, 262144), (40, 64000), (40, 128256)])
def test_sampling_from_large_vocabularies(T, rows, V):
    """Rows split over two to eight CTAs, all limits among them."""
    import torch
    rng = np.random.default_rng(V + rows)
    l = (rng.standard_normal((rows, V)) * 3).astype(np.float32)
    l[rng.random((rows, V)) < 0.01] = -np.inf
    u = rng.random((rows, V), dtype=np.float32)
    for kw in (dict(), dict(temperature=0.0), dict(temperature=0.7, top_k=50), dict(top_p=0.95), dict(min_p=0.05),
               dict(temperature=1.3, top_k=5000, top_p=0.9, min_p=0.001), dict(temperature=6.0, top_p=0.8)):
        tok, lp = _draw(T, torch.tensor(l).cuda(), torch.tensor(u).cuda(), **kw)
        names = dict(temperature="T")
        for b in range(rows):
            par = {names.get(k, k): v for k, v in kw.items()}
            _, wlp, _ = R.sample(l[b], u[b], **par)
            # limits that float32 does not tell apart: the winner among a few tokens less, or a few more
            top_p, min_p = par.pop("top_p", 1.0), par.pop("min_p", 0.0)
            less = R.sample(l[b], u[b], top_p=top_p - 1e-5 if top_p < 1 else 1.0, min_p=min_p * (1 + 1e-5), **par)
            more = R.sample(l[b], u[b], top_p=top_p + 1e-5 if top_p < 1 else 1.0, min_p=min_p * (1 - 1e-5), **par)
            assert tok[b] in (less[0], more[0]), (kw, b, tok[b], less, more)
            if less[0] == more[0]:
                z = abs(l[b][tok[b]] - l[b].max()) / (kw.get("temperature") or 1.0)
                assert abs(lp[b] - wlp) <= 4 * U * z + 2.0 ** -19 + 2 * U * abs(wlp), (kw, b, lp[b], wlp)
