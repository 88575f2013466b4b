"""The operators on a caller's paged caches and logits against plain 64-bit forms.

Bounds (u = 2^-24, half a float32 step; r = 2^-8, half a step of bfloat16's 8 significant bits): a score is a float32 sum of head_dim products and
is off by at most D = head_dim u sum |q k| (plus the scale's rounding); probabilities are then off by a factor of at most
1 + 2 D + 2^-20 (exponential, sum), rounded to bfloat16 by r in bfloat16 caches, and so is the result once.
"""
import math

import numpy as np
import pytest

import _serve_ref as R

pytestmark = pytest.mark.gpu
U, RB = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def T():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2609_15160_gb300 import build, tlf
    build.build()
    tlf.load_library()
    return tlf


def _attend(T, c, d, weights=False, scale=0.0, max_chunk=0, stream=None, out=None, lse=True, weight_in=None, in_place=False):
    import torch
    out = torch.full((max(1, c.T), c.hq, c.hd), float("nan"), dtype=d["q"].dtype, device="cuda") if out is None else out
    l = torch.full((max(1, c.T), c.hq), float("nan"), device="cuda") if lse else None
    w = (weight_in if in_place else torch.full((c.pages, 64), -7.0, device="cuda")) if weights else None
    b = T.chunk_args(d["pool"], d["table"], d["cu"], d["lens"], c.hq, c.T, layer=c.layer, max_chunk=max_chunk, err=d["err"])
    a = T.attn_chunk_args(d["q"], out, lse=l, weight_in=weight_in, weight_out=w, scale=scale)
    n = T.tlf_attn_chunk_scratch_bytes(b, a)
    assert n > 0
    scratch = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN wherever it is read before it is written
    T.tlf_attn_chunk(b, a, scratch, n, stream)
    torch.cuda.synchronize()
    return out, l, w


def _hold(c, d, got, ref, scale=None):
    """out and lse within their bounds; returns the bound of a score."""
    out, lse, spread, terms, _ = ref
    D = (c.hd + 4) * U * terms
    p_rel = 2 * D + 2.0 ** -20
    r = RB if c.dtype == "bf16" else 0.0
    o, l = (x[:c.T].float().cpu().numpy().astype(np.float64) for x in got[:2])
    bound = (p_rel[..., None] + r) * spread + (r + 4 * U) * np.abs(out) * (1 + r) + 1e-30
    assert np.isfinite(o).all() and (np.abs(o - out) <= bound).all(), np.max(np.abs(o - out) / bound)
    none = np.isneginf(lse)
    assert np.isneginf(l[none]).all() and (o[none] == 0).all()
    lb = D + 2.0 ** -20 + 2 * U * np.abs(np.where(none, 0, lse))
    off = np.abs(l[~none] - lse[~none])
    assert (off <= lb[~none]).all(), np.max(off / lb[~none])
    assert int(d["err"][0].item()) == 0
    return p_rel


def _hold_weights(c, w, w_in, ref, p_rel):
    weights = ref[4]
    w = w.cpu().numpy().astype(np.float64)
    seen = np.zeros((c.pages, 64), bool)
    rel = (p_rel.max() if p_rel.size else 0) + 2.0 ** -19
    for b in range(c.n):
        e = np.arange(max(0, c.lens[b]))
        want = w_in[c.at(b, e)].astype(np.float64) + weights[b]
        seen[c.at(b, e)] = True
        # sums of up to heads x queries positive float32 terms, in runs
        bound = (rel + 256 * U) * weights[b] + 4 * U * want + 1e-30
        assert (np.abs(w[c.at(b, e)] - want) <= bound).all(), (b, np.max(np.abs(w[c.at(b, e)] - want) / bound))
    return seen


ATTEND = {
    # old, new, hq, hkv, hd, dtype
    "ones": ([0, 1, 63, 64, 65, 127, 128, 3000], [1] * 8, 16, 8, 128, "bf16"),
    "ones-mha": ([0, 5, 62, 63, 64, 700], [1] * 6, 8, 8, 64, "bf16"),
    "few": ([0, 1, 60, 64, 200, 1000], [3, 16, 5, 1, 7, 2], 8, 2, 128, "bf16"),
    "few-g3": ([0, 100, 63], [20, 1, 9], 12, 4, 64, "bf16"),
    "none-new": ([10, 0, 64, 130], [0, 4, 0, 2], 4, 2, 32, "bf16"),
    "mqa": ([0, 77], [5, 11], 24, 1, 64, "bf16"),
    "g64": ([3, 150], [2, 1], 64, 1, 64, "bf16"),
    "many": ([0, 64, 100], [130, 257, 64], 4, 2, 128, "bf16"),
    "many-mha": ([0, 1, 500], [300, 127, 128], 2, 2, 64, "bf16"),
    "many-g5": ([17, 200], [140, 33], 5, 1, 64, "bf16"),
    "many-32": ([0, 99], [200, 70], 4, 2, 32, "bf16"),
    "many-short": ([3], [66], 2, 2, 64, "bf16"),
    "many-g16": ([40, 0], [9, 30], 32, 2, 128, "bf16"),
    "many-far": ([3000], [70], 2, 1, 128, "bf16"),
    "one-row": ([4000], [40], 4, 1, 128, "bf16"),
    "f32-16": ([0, 1, 64, 90], [1, 5, 64, 3], 4, 4, 16, "f32"),
    "f32-64": ([0, 300], [70, 1], 4, 2, 64, "f32"),
    "f32-128": ([5, 129], [9, 1], 6, 2, 128, "f32"),
    "f32-32-one": ([2000, 0], [1, 1], 2, 1, 32, "f32"),
}


@pytest.mark.parametrize("name", ATTEND)
def test_attention_of_a_chunk(T, name):
    import torch
    old, new, hq, hkv, hd, dtype = ATTEND[name]
    c = R.Cache(old, new, hq, hkv, hd, dtype, seed=len(name))
    d = c.device()
    ref = R.attention(c)
    got = _attend(T, c, d)
    _hold(c, d, got, ref)
    # the same with weights, on a prior account
    w_in = torch.rand(c.pages, 64, device="cuda")
    got = _attend(T, c, d, weights=True, weight_in=w_in)
    p_rel = _hold(c, d, got, ref)
    seen = _hold_weights(c, got[2], w_in.cpu().numpy(), ref, p_rel)
    assert (got[2].cpu().numpy()[~seen] == -7).all()  # nothing but the rows' entries is written
    # the same inputs give the same bits
    again = _attend(T, c, d, weights=True, weight_in=w_in)
    assert all(torch.equal(x[:c.T] if i < 2 else x, y[:c.T] if i < 2 else y) for i, (x, y) in enumerate(zip(got, again)))


MIDDLE = {
    # old, new, hq, hkv, hd: where one kernel takes over from the other, and rows shared by many CTAs
    "128-16": ([500, 0, 63, 64], [8, 1, 8, 3], 4, 2, 128),
    "128-17": ([500, 0, 63, 64], [17, 1, 8, 0], 2, 2, 128),
    "128-g3": ([500, 10], [11, 20], 3, 1, 128),
    "64-32": ([130, 4000], [8, 5], 8, 2, 64),
    "64-33": ([130, 4000, 0], [33, 5, 30], 2, 2, 64),
    "64-64": ([0, 63, 700], [16, 16, 15], 4, 1, 64),
    "64-g64": ([1, 190], [1, 1], 64, 1, 64),
    "short": ([0] * 40, [40, 1, 20, 33] * 10, 2, 2, 64),
    "shared": ([7000], [65], 2, 1, 64),
}


@pytest.mark.parametrize("name", MIDDLE)
def test_attention_between_few_and_many_rows(T, name):
    import torch
    old, new, hq, hkv, hd = MIDDLE[name]
    c = R.Cache(old, new, hq, hkv, hd, "bf16", seed=len(name) + 100)
    d = c.device()
    ref = R.attention(c)
    _hold(c, d, _attend(T, c, d), ref)
    w_in = torch.rand(c.pages, 64, device="cuda")
    got = _attend(T, c, d, weights=True, weight_in=w_in)
    seen = _hold_weights(c, got[2], w_in.cpu().numpy(), ref, _hold(c, d, got, ref))
    assert (got[2].cpu().numpy()[~seen] == -7).all()


@pytest.mark.parametrize("new", [[1, 1], [20, 9], [130, 64]], ids=["one", "few", "many"])
@pytest.mark.parametrize("hd", [64, 128])
def test_accounts_at_a_tiny_scale(T, new, hd):
    """All scores alike: every visible entry gets the same weight, and lse over the scale is far outside of float32."""
    import torch
    c = R.Cache([70, 300], new, 4, 2, hd, "bf16", seed=hd)
    d = c.device()
    ref = R.attention(c, scale=1e-38)
    w_in = torch.rand(c.pages, 64, device="cuda")
    got = _attend(T, c, d, weights=True, weight_in=w_in, scale=1e-38)
    p_rel = _hold(c, d, got, ref, scale=1e-38)
    _hold_weights(c, got[2], w_in.cpu().numpy(), ref, p_rel)


@pytest.mark.parametrize("new,max_chunk", [([1, 1, 1], 1), ([3, 1, 0], 3), ([90, 150, 1], 150)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing_and_rows_without_entries(T, new, max_chunk, dtype):
    """lens smaller than the new tokens: the first queries see nothing."""
    c = R.Cache([5, 100, 0], new, 4, 2, 64, dtype, seed=3)
    c.lens = np.array([0, max(0, new[1] - 2), c.lens[2]])
    d = c.device()
    ref = R.attention(c)
    w_in = np.zeros((c.pages, 64), np.float32)
    got = _attend(T, c, d, weights=True, max_chunk=max_chunk)
    _hold_weights(c, got[2], w_in, ref, _hold(c, d, got, ref))


@pytest.mark.parametrize("new", [[1, 1], [6, 2], [140, 70]], ids=["one", "few", "many"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_a_query_may_not_see_does_not_reach_it(T, new, dtype, bad):
    """Entries behind a row's cache, entries of later tokens and pages of nobody hold NaN or infinities."""
    c = R.Cache([70, 30], new, 4, 2, 64, dtype, seed=11)
    ref = R.attention(c)
    keep = np.ones((c.pages, 64), bool)
    for b in range(c.n):
        keep[c.at(b, np.arange(c.lens[b]))] = False
    mask = keep[:, None, None, None, :, None]
    c.pool = np.where(mask, np.float32(bad), c.pool)
    d = c.device()
    _hold(c, d, _attend(T, c, d), ref)
    # the last new token's key and value: only its own query may see them
    for b in range(c.n):
        p, o = c.at(b, np.array([c.lens[b] - 1]))
        c.pool[p, c.layer, :, :, o] = bad
    d = c.device()
    out, lse, _ = _attend(T, c, d)
    last = c.cu[1:] - 1
    others = np.setdiff1d(np.arange(c.T), last)
    r = RB if dtype == "bf16" else 0.0
    p_rel = 2 * (c.hd + 4) * U * ref[3] + 2.0 ** -20
    o = out.float().cpu().numpy()[others]
    bound = ((p_rel[..., None] + r) * ref[2] + (r + 4 * U) * np.abs(ref[0]) * (1 + r) + 1e-30)[others]
    assert (np.abs(o - ref[0][others]) <= bound).all()
    assert not np.isfinite(out.float().cpu().numpy()[last]).all()


@pytest.mark.parametrize("new,hq,hd", [([9, 12], 4, 128), ([20, 1], 2, 128), ([40, 33], 2, 64), ([130, 64], 4, 128)])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_what_a_query_may_not_see_does_not_reach_the_accounts(T, new, hq, hd, bad):
    """The same where tiles are mostly padding, and for the weights: entries behind the caches and pages of nobody."""
    import torch
    c = R.Cache([70, 300], new, hq, 2, hd, "bf16", seed=13)
    ref = R.attention(c)
    keep = np.ones((c.pages, 64), bool)
    for b in range(c.n):
        keep[c.at(b, np.arange(c.lens[b]))] = False
    c.pool = np.where(keep[:, None, None, None, :, None], np.float32(bad), c.pool)
    d = c.device()
    w_in = torch.rand(c.pages, 64, device="cuda")
    got = _attend(T, c, d, weights=True, weight_in=w_in)
    seen = _hold_weights(c, got[2], w_in.cpu().numpy(), ref, _hold(c, d, got, ref))
    assert (got[2].cpu().numpy()[~seen] == -7).all()
    # the last new token's key: earlier queries' output and lse are as before
    for b in range(c.n):
        p, o = c.at(b, np.array([c.lens[b] - 1]))
        c.pool[p, c.layer, :, :, o] = bad
    again = _attend(T, c, c.device())
    others = torch.as_tensor(np.setdiff1d(np.arange(c.T), c.cu[1:] - 1), device="cuda")
    assert torch.isfinite(again[0][others].float()).all()
    assert (again[0][others].float() - got[0][others].float()).abs().max().item() <= 2 * RB * got[0].float().abs().max().item()


def test_a_value_that_is_infinite_reaches_those_that_see_it(T):
    for new in ([1], [5], [130]):
        c = R.Cache([100], new, 2, 1, 64, "bf16", seed=5)
        c.pool[c.table[0, 0], c.layer, 1, 0, 3, 7] = np.inf
        d = c.device()
        out = _attend(T, c, d)[0].float().cpu().numpy()
        assert np.isposinf(out[:, :, 7]).all() and np.isfinite(np.delete(out, 7, 2)).all()


def test_strides_scale_stream_and_accounts_in_place(T):
    import torch
    for new in ([4, 1], [100, 40]):
        c = R.Cache([64, 33], new, 4, 2, 64, "bf16", seed=8)
        d = c.device()
        wide = torch.zeros(c.T, 7, c.hq * c.hd + 24, dtype=torch.bfloat16, device="cuda")
        q = wide[:, 2, 8:8 + c.hq * c.hd].unflatten(1, (c.hq, c.hd))
        q.copy_(d["q"][:c.T])
        out = torch.full((c.T, c.hq * c.hd + 8), 3.0, dtype=torch.bfloat16, device="cuda")
        w = torch.rand(c.pages, 64, device="cuda")
        w_in = w.cpu().numpy()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = _attend(T, c, dict(d, q=q), weights=True, weight_in=w, in_place=True, scale=0.3, stream=s,
                      out=out[:, :c.hq * c.hd].unflatten(1, (c.hq, c.hd)))
        ref = R.attention(c, 0.3)
        _hold_weights(c, got[2], w_in, ref, _hold(c, d, got, ref))
        assert (out[:, c.hq * c.hd:] == 3).all()
        # odd strides and offsets that are not multiples of 16 bytes
        odd = torch.zeros(c.T, c.hq * c.hd + 3, dtype=torch.bfloat16, device="cuda")
        q = odd[:, 1:1 + c.hq * c.hd].unflatten(1, (c.hq, c.hd))
        q.copy_(d["q"][:c.T])
        o = torch.zeros(c.T, c.hq * c.hd + 1, dtype=torch.bfloat16, device="cuda")
        got = _attend(T, c, dict(d, q=q), out=o[:, 1:].unflatten(1, (c.hq, c.hd)), scale=0.3)
        _hold(c, d, got, ref)


def test_scores_far_from_zero(T):
    """Scores of thousands: the maximum has to be taken out before the exponential."""
    for new in ([1], [9], [200]):
        c = R.Cache([150], new, 4, 2, 64, "bf16", seed=2)
        c.q = R.bf16(c.q * 64)
        d = c.device()
        ref = R.attention(c)
        _hold(c, d, _attend(T, c, d), ref)


def test_bad_indices_are_reported_and_skipped(T):
    """Page ids outside the pool, offsets and lengths out of range: reported, and the other rows are right."""
    import torch
    for new in ([2, 3, 1], [70, 90, 80]):
        c = R.Cache([70, 64, 130], new, 4, 2, 64, "bf16", seed=4)
        ref = R.attention(c)
        for what in ("page", "length", "offsets"):
            d = c.device()
            if what == "page":
                d["table"][0, 0], d["table"][2, 1] = c.pages + 5, -3
                rows = [1]
            elif what == "length":
                d["lens"][0] = 64 * c.table.shape[1] + 1000
                d["lens"][2] = -5
                rows = [1]
            else:
                d["cu"][3] = c.T + 50
                rows = [0, 1]
            out = _attend(T, c, d)[0].float().cpu().numpy()
            assert int(d["err"][0].item()) & 2
            for b in rows:
                t = slice(c.cu[b], c.cu[b + 1])
                assert np.abs(out[t] - ref[0][t]).max() < 0.1
            torch.cuda.synchronize()


def test_no_tokens(T):
    c = R.Cache([64, 10], [0, 0], 4, 2, 64, "bf16")
    d = c.device()
    w = np.random.rand(c.pages, 64).astype(np.float32)
    import torch
    got = _attend(T, c, d, weights=True, weight_in=torch.tensor(w).cuda())
    _hold_weights(c, got[2], w, R.attention(c), np.zeros(0))


# ---- rotary positions ----

@pytest.mark.parametrize("dtype,hq,hkv,hd,rot", [("bf16", 4, 2, 128, 128), ("bf16", 3, 1, 64, 32), ("bf16", 2, 2, 32, 6),
                                                 ("f32", 4, 4, 16, 16), ("f32", 2, 1, 64, 10), ("bf16", 8, 8, 64, 64)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("q32", [False, True])
def test_rotary_append(T, dtype, hq, hkv, hd, rot, layout, q32):
    import torch
    c = R.Cache([0, 63, 64, 10, 200], [1, 3, 0, 70, 9], hq, hkv, hd, dtype, seed=hd + rot)
    pos = np.concatenate([o + o // 3 + np.arange(n) for o, n in zip(c.old, c.new)]).astype(np.int32)
    for pad in (0, 3):  # packed q, k, v with aligned and with odd rows
        qkv = c.round(c.rng.standard_normal((c.T, (hq + 2 * hkv) * hd + pad)).astype(np.float32))
        d = c.device(qkv=qkv, pos=pos)
        dt = d["pool"].dtype
        table = torch.empty(512, rot // 2, 2, device="cuda")
        T.tlf_rope_table(T.rope_config(rot), 512, table)
        qo = torch.full((c.T, hq, hd), 9.0, dtype=torch.float32 if q32 else dt, device="cuda")
        epos, ew = torch.full((c.pages, 64), -9, dtype=torch.int32, device="cuda"), torch.full((c.pages, 64), 5.0, device="cuda")
        x = d["qkv"].to(dt)
        q, k, v = (x[:, a:b] for a, b in ((0, hq * hd), (hq * hd, (hq + hkv) * hd), ((hq + hkv) * hd, (hq + 2 * hkv) * hd)))
        b = T.chunk_args(d["pool"], d["table"], d["cu"], d["lens"], hq, c.T, layer=c.layer, err=d["err"])
        T.tlf_rope_append(b, T.rope_args(q, k, v, d["pos"], table, qo, layout=layout, entry_pos=epos, entry_weight=ew))
        torch.cuda.synchronize()
        assert int(d["err"][0].item()) == 0
        xs = qkv[:, :(hq + 2 * hkv) * hd].reshape(c.T, hq + 2 * hkv, hd)
        cs = table.cpu().numpy()[pos]
        want = R.turn(xs[:, :hq + hkv], cs, rot, layout)
        size = np.abs(xs[:, :hq + hkv]).astype(np.float64)
        size[..., :rot] = np.abs(xs[:, :hq + hkv, :rot]).max(-1, keepdims=True) * 2
        err_q = 3 * U * size[:, :hq] + (RB * np.abs(want[:, :hq]) * 1.01 if dtype == "bf16" and not q32 else 0)
        assert (np.abs(qo.float().cpu().numpy() - want[:, :hq]) <= err_q).all()
        pool = c.pool.copy()
        got = d["pool"].float().cpu().numpy()
        expos, exw = np.full((c.pages, 64), -9), np.full((c.pages, 64), 5.0)
        for row in range(c.n):
            t = np.arange(c.cu[row], c.cu[row + 1])
            p, o = c.at(row, c.lens[row] - c.new[row] + np.arange(len(t)))
            err_k = 3 * U * size[t, hq:] + (RB * np.abs(want[t, hq:]) * 1.01 if dtype == "bf16" else 0)
            assert (np.abs(got[p, c.layer, 0, :, o] - want[t, hq:]) <= err_k).all()
            pool[p, c.layer, 0, :, o] = got[p, c.layer, 0, :, o]
            pool[p, c.layer, 1, :, o] = xs[t, hq + hkv:]
            expos[p, o], exw[p, o] = pos[t], 0
        assert np.array_equal(got, pool) and np.array_equal(epos.cpu().numpy(), expos) and np.array_equal(ew.cpu().numpy(), exw)


def test_rotary_append_reports_what_it_cannot_place(T):
    """A position out of range: a zero query and no entry. A row with fewer entries than tokens: queries only."""
    import torch
    c = R.Cache([10, 0], [3, 2], 2, 1, 64, "bf16", seed=1)
    d = c.device()
    d["lens"][1] = 1
    x = torch.randn(c.T, 4 * 64, device="cuda").bfloat16()
    pos = torch.tensor([0, -1, 64, 3, 4], dtype=torch.int32, device="cuda")
    table = torch.empty(64, 32, 2, device="cuda")
    T.tlf_rope_table(T.rope_config(64), 64, table)
    qo = torch.full((c.T, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    before = d["pool"].clone()
    b = T.chunk_args(d["pool"], d["table"], d["cu"], d["lens"], 2, c.T, layer=c.layer, err=d["err"])
    T.tlf_rope_append(b, T.rope_args(x[:, :128], x[:, 128:192], x[:, 192:], pos, table, qo))
    torch.cuda.synchronize()
    assert int(d["err"][0].item()) & 2
    assert (qo[1:3] == 0).all() and not (qo[3:] == 9).any() and not (qo[0] == 9).any()
    changed = (d["pool"] != before).any(-1).any(2).any(2).any(1).nonzero().tolist()  # [page, offset]
    assert sorted(changed) == sorted([[int(c.table[0, 0]), 10], [int(c.table[1, 0]), 0]])


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0, base=5e5),
                                dict(scaling="ramp", factor=16.0, original_len=4096, magnitude=1.2772588722239782)])
@pytest.mark.parametrize("rot,max_pos", [(64, 131072), (6, 1000), (128, 33)])
def test_rotary_table(T, kw, rot, max_pos):
    import torch
    table = torch.empty(max_pos, rot // 2, 2, device="cuda")
    T.tlf_rope_table(T.rope_config(rot, **kw), max_pos, table)
    k = np.arange(rot // 2)
    base, s = kw.get("base", 1e4), kw.get("factor", 1.0)
    if kw.get("scaling") == "ntk":
        base *= s ** (rot / (rot - 2))
    f = base ** (-2.0 * k / rot)
    if kw.get("scaling") == "linear":
        f = f / s
    if kw.get("scaling") == "ramp":
        r = np.clip((4096 * f / (2 * math.pi) - 1) / 31, 0, 1)
        f = f / s * (1 - r) + f * r
    ang, mag = np.arange(max_pos)[:, None] * f, kw.get("magnitude", 1.0)
    want = np.stack([np.cos(ang), np.sin(ang)], -1) * mag
    # float32 rounding, and the angle's: a few steps of 2^-53 of it
    bound = U * mag * 1.01 + 8 * 2.0 ** -53 * (ang[..., None] + 1) * mag
    assert (np.abs(table.cpu().numpy() - want) <= bound).all()


# ---- eviction ----

@pytest.mark.parametrize("dtype,hkv,hd,layers", [("bf16", 2, 64, 3), ("f32", 1, 16, 1), ("bf16", 1, 128, 2)])
@pytest.mark.parametrize("budget,first,recent", [(64, 4, 16), (200, 0, 0), (1, 0, 0), (5, 2, 3), (1000, 8, 100)])
@pytest.mark.parametrize("in_place", [False, True])
def test_eviction(T, dtype, hkv, hd, layers, budget, first, recent, in_place):
    import torch
    lens = [0, 1, 63, 64, 65, 200, 201, 1500, 5]
    c = R.Cache(lens, [0] * len(lens), hkv, hkv, hd, dtype, layers=layers, layer=0, seed=budget + layers)
    rng = np.random.default_rng(budget)
    w = rng.exponential(1, (c.pages, 64)).astype(np.float32)
    w[rng.random(w.shape) < 0.3] = 0  # ties
    w[rng.random(w.shape) < 0.05] = np.nan
    w[rng.random(w.shape) < 0.05] = np.inf
    w[rng.random(w.shape) < 0.05] = -1
    pos, nxt = np.full((c.pages, 64), -1, np.int32), []
    for b, n in enumerate(lens):
        p = np.cumsum(rng.integers(1, 3, n)) - 1 if n else np.zeros(0, int)
        pos[c.at(b, np.arange(n))] = rng.permutation(p) if b % 2 else p  # moved entries are not in order
        nxt.append(int(p[-1]) + 1 if n else 0)
    d = c.device(w=w, pos=pos, nxt=np.asarray(nxt, np.int32))
    wo = d["w"] if in_place else torch.full((c.pages, 64), -7.0, device="cuda")
    po = d["pos"] if in_place else torch.full((c.pages, 64), -7, dtype=torch.int32, device="cuda")
    lo = d["lens"] if in_place else torch.full((c.n,), -7, dtype=torch.int32, device="cuda")
    a = T.evict_args(d["pool"], d["table"], d["lens"], d["nxt"], d["pos"], po, d["w"], wo, lo, budget=budget, n_first=first,
                     n_recent=recent, err=d["err"])
    n = T.tlf_cache_evict_scratch_bytes(a)
    T.tlf_cache_evict(a, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n)
    torch.cuda.synchronize()
    assert int(d["err"][0].item()) == 0
    pool, wx, px = c.pool.copy(), np.full_like(w, -7), np.full_like(pos, -7)
    if in_place:
        wx, px = w.copy(), pos.copy()
    for b, n in enumerate(lens):
        e = np.arange(n)
        src = R.evict(w[c.at(b, e)], pos[c.at(b, e)], nxt[b], budget, first, recent)
        to, fr = c.at(b, np.arange(len(src))), c.at(b, src)
        pool[to[0], :, :, :, to[1]] = c.pool[fr[0], :, :, :, fr[1]]
        wx[to], px[to] = w[fr], pos[fr]
    assert np.array_equal(lo.cpu().numpy(), np.minimum(lens, budget))
    assert np.array_equal(d["pool"].float().cpu().numpy(), pool)
    assert np.array_equal(wo.cpu().numpy(), wx, equal_nan=True) and np.array_equal(po.cpu().numpy(), px)


def test_eviction_of_a_long_row(T):
    """More entries than a CTA keeps in shared memory."""
    import torch
    L = 50000
    c = R.Cache([L], [0], 1, 1, 16, "f32", layers=1, layer=0)
    rng = np.random.default_rng(0)
    w = np.round(rng.exponential(1, (c.pages, 64)), 2).astype(np.float32)
    pos = np.zeros((c.pages, 64), np.int32)
    e = np.arange(L)
    pos[c.at(0, e)] = e
    for budget in (1000, 30000, 49990):
        d = c.device(w=w, pos=pos, nxt=np.array([L], np.int32))
        wo, po, lo = torch.zeros_like(d["w"]), torch.zeros_like(d["pos"]), torch.zeros_like(d["lens"])
        a = T.evict_args(d["pool"], d["table"], d["lens"], d["nxt"], d["pos"], po, d["w"], wo, lo, budget=budget, n_first=4,
                         n_recent=64)
        n = T.tlf_cache_evict_scratch_bytes(a)
        T.tlf_cache_evict(a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
        src = R.evict(w[c.at(0, e)], pos[c.at(0, e)], L, budget, 4, 64)
        to, fr = c.at(0, np.arange(budget)), c.at(0, src)
        assert np.array_equal(po.cpu().numpy()[to], pos[fr]) and np.array_equal(wo.cpu().numpy()[to], w[fr])
        assert np.array_equal(d["pool"].cpu().numpy()[to[0], 0, :, :, to[1]], c.pool[fr[0], 0, :, :, fr[1]])


def test_eviction_reports_bad_pages(T):
    import torch
    c = R.Cache([200, 100], [0, 0], 1, 1, 64, "bf16", layers=1, layer=0)
    d = c.device(w=np.ones((c.pages, 64), np.float32), pos=np.zeros((c.pages, 64), np.int32), nxt=np.array([300, 300], np.int32))
    d["table"][0, 1] = c.pages
    before = d["pool"].clone()
    a = T.evict_args(d["pool"], d["table"], d["lens"], d["nxt"], d["pos"], d["pos"], d["w"], d["w"], d["lens"], budget=50,
                     err=d["err"])
    n = T.tlf_cache_evict_scratch_bytes(a)
    T.tlf_cache_evict(a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    assert int(d["err"][0].item()) & 2 and d["lens"].tolist() == [50, 50]
    other = torch.ones(c.pages, dtype=torch.bool, device="cuda")
    other[torch.tensor(c.table[:, 0].astype(np.int64)).cuda()] = False
    assert torch.equal(d["pool"][other], before[other])


# ---- sampling ----

def _draw(T, l, u, **kw):
    import torch
    n = l.shape[0]
    tok, lp = torch.full((n,), -5, dtype=torch.int32, device="cuda"), torch.full((n,), 5.0, device="cuda")
    par = {k: torch.tensor(np.broadcast_to(np.asarray(v, np.int32 if k == "top_k" else np.float32), (n,)).copy()).cuda()
           for k, v in kw.items()}
    T.tlf_sample(T.sample_args(l, u, tok, lp, **par))
    torch.cuda.synchronize()
    return tok.cpu().numpy(), lp.cpu().numpy()


PARAMS = [dict(), dict(temperature=0.0), dict(temperature=0.7, top_k=50), dict(top_p=0.9), dict(min_p=0.05),
          dict(temperature=1.3, top_k=200, top_p=0.95, min_p=0.01), dict(top_k=1), dict(top_p=0.0), dict(top_p=1e-6),
          dict(min_p=1.0), dict(min_p=2.0), dict(top_k=3000, top_p=0.7), dict(top_k=1 << 30, top_p=0.999), dict(temperature=8.0, top_p=0.8)]


@pytest.mark.parametrize("V", [1, 2, 31, 1000, 1024, 1025, 5003, 50304])
@pytest.mark.parametrize("kw", PARAMS, ids=lambda k: "-".join(f"{a}{b}" for a, b in k.items()) or "plain")
def test_sampling(T, V, kw):
    import torch
    rng = np.random.default_rng(V)
    rows = 6
    l = (rng.standard_normal((rows, V)) * 4).astype(np.float32)
    l[1] = np.round(l[1])  # ties
    l[2] = 0               # all alike
    l[3][rng.random(V) < 0.9] = -np.inf
    l[4] *= 30
    u = rng.random((rows, V), dtype=np.float32)
    tok, lp = _draw(T, torch.tensor(l).cuda(), torch.tensor(u).cuda(), **kw)
    names = dict(temperature="T")
    for b in range(rows):
        want, wlp, gap = R.sample(l[b], u[b], **{names.get(k, k): v for k, v in kw.items()})
        # a draw that another token misses by less than float32 tells apart is not held to the token
        if gap > 1e-5:
            assert tok[b] == want, (b, tok[b], want, gap)
            z = abs(l[b][want] - l[b].max()) / (kw.get("temperature") or 1.0) if want >= 0 else 0
            assert (lp[b] == wlp) or abs(lp[b] - wlp) <= 4 * U * z + 2.0 ** -19 + 2 * U * abs(wlp), (b, lp[b], wlp)


def test_sampling_rows_with_nothing_to_draw_and_odd_values(T):
    import torch
    V = 300
    l = np.full((8, V), -np.inf, np.float32)
    u = np.full((8, V), 0.5, np.float32)
    l[1] = np.nan
    l[2, 7] = -3e38
    l[3, [4, 9]] = np.inf
    l[4, :] = np.nan
    l[4, 11] = 1.0
    l[5, :] = np.linspace(-3e38, 3e38, V)
    l[6, :] = 0
    u[6, :] = 0            # every number 0: the lowest index
    l[7, :3] = 1
    u[7, :3] = [np.nan, 0.0, 1.0]
    tok, lp = _draw(T, torch.tensor(l).cuda(), torch.tensor(u).cuda())
    assert tok.tolist() == [-1, -1, 7, 4, 11, V - 1, 0, 2]
    assert np.isneginf(lp[:2]).all() and np.allclose(lp[[2, 4, 5]], 0) and abs(lp[3] + math.log(2)) < 1e-6


def test_sampling_follows_the_probabilities(T):
    """Over many rows with the same logits the tokens come with the kept tokens' probabilities."""
    import torch
    n, V = 40000, 40
    g = torch.Generator(device="cuda").manual_seed(3)
    l = torch.randn(V, device="cuda", generator=g)
    u = torch.rand(n, V, device="cuda", generator=g)
    tok, _ = _draw(T, l.expand(n, V).contiguous(), u, top_k=10, temperature=0.8)
    p = torch.softmax(l.double() / 0.8, 0).cpu().numpy()
    kept = np.argsort(-p, kind="stable")[:10]
    q = np.zeros(V)
    q[kept] = p[kept] / p[kept].sum()
    f = np.bincount(tok, minlength=V) / n
    assert (f[q == 0] == 0).all() and (np.abs(f - q) <= 6 * np.sqrt(q * (1 - q) / n) + 1e-9).all()


def test_sampling_strides_and_defaults(T):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    l, u = (torch.randn(5, 777, device="cuda", generator=g) * 3, torch.rand(5, 1001, device="cuda", generator=g))
    a, _ = _draw(T, l[:, 3:603], u[:, 1:601], top_k=20)
    b, _ = _draw(T, l[:, 3:603].contiguous(), u[:, 1:601].contiguous(), top_k=20)
    assert np.array_equal(a, b)
    tok = torch.zeros(5, dtype=torch.int32, device="cuda")
    T.tlf_sample(T.sample_args(l[:, :600], u[:, :600], tok))
    c, _ = _draw(T, l[:, :600], u[:, :600], temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    assert np.array_equal(tok.cpu().numpy(), c)


# ---- together ----

def test_operators_in_a_cuda_graph(T):
    """append, attend with weights and sample captured once and replayed with other inputs."""
    import torch
    c = R.Cache([64, 100, 3], [1, 1, 1], 4, 2, 64, "bf16", seed=6)
    d = c.device()
    x = torch.randn(3, 8 * 64, device="cuda").bfloat16()
    pos = torch.tensor(c.old.astype(np.int32)).cuda()
    table = torch.empty(256, 32, 2, device="cuda")
    T.tlf_rope_table(T.rope_config(64), 256, table)
    q, out = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(c.pages, 64, device="cuda")
    l, u, tok = torch.randn(3, 500, device="cuda"), torch.rand(3, 500, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    b = T.chunk_args(d["pool"], d["table"], d["cu"], d["lens"], 4, 3, layer=c.layer, max_chunk=1, err=d["err"])
    ra = T.rope_args(x[:, :256], x[:, 256:384], x[:, 384:], pos, table, q)
    aa = T.attn_chunk_args(q, out, weight_in=w, weight_out=w)
    n = T.tlf_attn_chunk_scratch_bytes(b, aa)
    scratch = torch.empty(n, dtype=torch.uint8, device="cuda")
    sa = T.sample_args(l, u, tok)

    def step(stream):
        T.tlf_rope_append(b, ra, stream)
        T.tlf_attn_chunk(b, aa, scratch, n, stream)
        T.tlf_sample(sa, stream)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(torch.cuda.current_stream())
    x.copy_(torch.randn(3, 8 * 64, device="cuda").bfloat16())
    l.copy_(torch.randn(3, 500, device="cuda"))
    w.zero_()
    g.replay()
    torch.cuda.synchronize()
    once = out.clone(), tok.clone(), w.clone()
    w.zero_()
    step(torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(once[0], out) and torch.equal(once[1], tok) and torch.equal(once[2], w)
    assert abs(float(w.sum()) - 12) < 1e-3  # every query head of every row gives away 1
    assert int(d["err"][0].item()) == 0


# ---- sizes at the edges of the types ----

def test_a_thousand_rows(T):
    """The most rows of a call; with one long row among them every kernel's tables are at their largest."""
    rng = np.random.default_rng(0)
    for new in (np.ones(1024, np.int64), np.where(np.arange(1024) == 700, 90, 1)):
        c = R.Cache(rng.integers(0, 130, 1024), new, 2, 1, 64, "bf16", layers=1, layer=0, seed=9)
        d = c.device()
        ref = R.attention(c)
        w_in = np.zeros((c.pages, 64), np.float32)
        got = _attend(T, c, d, weights=True)
        _hold_weights(c, got[2], w_in, ref, _hold(c, d, got, ref))


@pytest.mark.parametrize("new", [1, 5, 100])
def test_pages_beyond_32_bit_offsets(T, new):
    """Pages whose elements lie past 2^32: append, attention with weights and eviction there."""
    import torch
    c = R.Cache([90, 200], [new, new], 4, 2, 128, "bf16", layers=2, layer=1, seed=7)
    page = 2 * 2 * 2 * 64 * 128
    far = (1 << 32) // page + 10
    if torch.cuda.mem_get_info()[0] < (far + c.pages) * page * 2 + (4 << 30):
        pytest.skip("needs 13 GB of the GPU's memory")
    pool = torch.empty(far + c.pages, 2, 2, 2, 64, 128, dtype=torch.bfloat16, device="cuda")
    pool[far:] = torch.tensor(c.pool).bfloat16().cuda()
    side = lambda fill, dt: torch.full((far + c.pages, 64), fill, dtype=dt, device="cuda")  # noqa: E731
    table = torch.tensor(np.where(c.table >= 0, c.table + far, -1)).cuda()
    d = c.device()
    # the new entries again, from the rows' own keys and values, unturned
    kv = [c.kv(b) for b in range(2)]
    k, v = (torch.tensor(np.concatenate([x[i][o:] for x, o in zip(kv, c.old)])).bfloat16().cuda() for i in (0, 1))
    for b in range(2):
        p, o = c.at(b, np.arange(c.old[b], c.lens[b]))
        pool[torch.tensor(p + far).cuda().long(), 1, :, :, torch.tensor(o).cuda()] = 9
    cs = torch.zeros(8, 64, 2, device="cuda")
    cs[..., 0] = 1
    qo, pos, w = torch.empty_like(d["q"]), side(-1, torch.int32), side(3.0, torch.float32)
    b = T.chunk_args(pool, table, d["cu"], d["lens"], 4, c.T, layer=1, err=d["err"])
    zero = torch.zeros(c.T, dtype=torch.int32, device="cuda")
    T.tlf_rope_append(b, T.rope_args(d["q"], k, v, zero, cs, qo, entry_pos=pos, entry_weight=w))
    got = _attend(T, c, dict(d, pool=pool, table=table), weights=False)
    ref = R.attention(c)
    _hold(c, d, got, ref)
    out, lse = torch.empty_like(d["q"]), torch.empty(c.T, 4, device="cuda")
    w_out = torch.zeros_like(w)
    a = T.attn_chunk_args(d["q"], out, lse=lse, weight_in=w, weight_out=w_out)
    n = T.tlf_attn_chunk_scratch_bytes(b, a)
    T.tlf_attn_chunk(b, a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    for row in range(2):
        p, o = c.at(row, np.arange(c.lens[row]))
        seen = w_out[torch.tensor(p + far).cuda().long(), torch.tensor(o).cuda()].cpu().numpy()
        prior = np.where(np.arange(c.lens[row]) < c.old[row], 3.0, 0.0)
        assert np.abs(seen - prior - ref[4][row]).max() < 1e-3
    nxt = torch.tensor([1000, 1000], dtype=torch.int32, device="cuda")
    before = pool[far:].clone()
    e = T.evict_args(pool, table, d["lens"], nxt, pos, pos, w_out, w_out, torch.empty_like(d["lens"]), budget=70, err=d["err"])
    n = T.tlf_cache_evict_scratch_bytes(e)
    T.tlf_cache_evict(e, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    torch.cuda.synchronize()
    assert int(d["err"][0].item()) == 0
    after = pool[far:]
    for row in range(2):
        p, o = c.at(row, np.arange(c.lens[row]))
        p, o = torch.tensor(p).cuda().long(), torch.tensor(o).cuda()
        held = {x.tobytes() for x in before[p, :, :, :, o].float().cpu().numpy()}
        assert all(x.tobytes() in held for x in after[p[:70], :, :, :, o[:70]].float().cpu().numpy())
