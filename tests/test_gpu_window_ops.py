"""The 4-bit cache, windowed attention and the page operators against plain 64-bit forms.

Bounds (u = 2^-24, half a float32 step; r = 2^-8, half a step of bfloat16's 8 significant bits). A score is a sum of head_dim
products and, in 4 bits, of the groups' lo times the sums of q beside d times the sums of q n; tensor cores may cut a partial sum
where float32 rounds it, so each of the head_dim + 8 additions is off by at most a step, 2 u, of the sum of the terms' magnitudes:
D = 2 (head_dim + 8) u sum(|q| (|lo| + d n)), in plain caches sum |q k|. Probabilities are then off by a factor of at most
1 + 2 D + 2^-19 (exponential, sum), rounded to 8 bits or more in bfloat16 calls, and so is the result once; values rounded to 11
bits for the tensor cores (2^-11) stay within the latter's slack of r for the probabilities, which are rounded to 11 bits there too.
"""
import numpy as np
import pytest

import _serve_ref as R
import _window_ref as W

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


def _batch(T, c, d, max_chunk=0):
    if isinstance(c, W.Cache4):
        return T.chunk4_args(d["pool"], d["table"], d["cu"], d["lens"], c.hq, c.T, c.hd, c.dtype, layer=c.layer, max_chunk=max_chunk, err=d["err"])
    return T.chunk_args(d["pool"], d["table"], d["cu"], d["lens"], c.hq, c.T, layer=c.layer, max_chunk=max_chunk, err=d["err"])


def _attend(T, c, d, window=0, first=0, scale=0.0, max_chunk=0, stream=None, out=None, lse=True):
    import torch
    out = torch.full((max(1, c.T), c.hq, c.hd), float("nan"), dtype=d["q"].dtype, device="cuda") if out is None else out
    l = torch.full((max(1, c.T), c.hq), float("nan"), device="cuda") if lse else None
    b = _batch(T, c, d, max_chunk)
    a = T.attn_window_args(d["q"], out, lse=l, window=window, n_first=first, kv4=isinstance(c, W.Cache4), scale=scale)
    n = T.tlf_attn_window_scratch_bytes(b, a)
    assert n > 0
    scratch = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN wherever it is read before it is written
    T.tlf_attn_window(b, a, scratch, n, stream)
    torch.cuda.synchronize()
    return out, l


def _hold(c, d, got, ref, tokens=None, err=0):
    """out and lse within their bounds, for all tokens or some."""
    out, lse, spread, terms = (x if tokens is None else x[tokens] for x in ref)
    D = 2 * (c.hd + 8) * U * terms
    p_rel = 2 * D + 2.0 ** -19
    r = RB if c.dtype == "bf16" else 0.0
    o, l = (x[:c.T].float().cpu().numpy().astype(np.float64) for x in got[:2])
    if tokens is not None:
        o, l = o[tokens], l[tokens]
    bound = (p_rel[..., None] + r) * spread + (r + 4 * U) * np.abs(out) * (1 + r) + 1e-30
    assert np.isfinite(o).all() and (np.abs(o - out) <= bound).all(), np.nanmax(np.abs(o - out) / bound)
    none = np.isneginf(lse)
    assert np.isneginf(l[none]).all() and (o[none] == 0).all()
    lb = D + 2.0 ** -19 + 2 * U * np.abs(np.where(none, 0, lse))
    off = np.abs(l[~none] - lse[~none])
    assert (off <= lb[~none]).all(), np.max(off / lb[~none])
    assert int(d["err"][0].item()) == err


def _cache(kind, *a, **kw):
    return W.Cache4(*a, **kw) if kind == "4bit" else R.Cache(*a, **kw)


SHAPES = {
    # old, new, hq, hkv, hd, dtype
    "ones": ([0, 1, 63, 64, 65, 127, 128, 3000], [1] * 8, 16, 8, 128, "bf16"),
    "ones-mha": ([0, 5, 62, 63, 64, 700], [1] * 6, 8, 8, 64, "bf16"),
    "few": ([0, 1, 60, 64, 200, 1000], [3, 8, 5, 1, 7, 2], 8, 2, 128, "bf16"),
    "few-16": ([130, 500], [16, 9], 4, 4, 64, "bf16"),
    "few-17": ([130, 500, 0], [17, 9, 30], 4, 4, 64, "bf16"),
    "few-g3": ([0, 100, 63], [20, 1, 9], 12, 4, 64, "bf16"),
    "g3-ones": ([400, 63], [1, 2], 6, 2, 128, "bf16"),
    "none-new": ([10, 0, 64, 130], [0, 4, 0, 2], 4, 2, 32, "bf16"),
    "mqa": ([0, 77], [5, 11], 24, 1, 64, "bf16"),
    "g64": ([3, 150], [2, 1], 64, 1, 64, "bf16"),
    "g32-ones": ([200, 0, 63], [1, 1, 1], 32, 1, 64, "bf16"),
    "few-48": ([0, 300], [48, 40], 2, 2, 64, "bf16"),
    "many-49": ([0, 300], [49, 40], 2, 2, 64, "bf16"),
    "many": ([0, 64, 100], [130, 257, 64], 4, 2, 128, "bf16"),
    "many-mha": ([0, 1, 500], [300, 127, 128], 2, 2, 64, "bf16"),
    "many-g5": ([17, 200], [140, 33], 5, 1, 64, "bf16"),
    "many-32": ([0, 99], [200, 70], 4, 2, 32, "bf16"),
    "many-g16": ([40, 0], [9, 30], 32, 2, 128, "bf16"),
    "many-far": ([3000], [70], 2, 1, 128, "bf16"),
    "one-row": ([4000], [40], 4, 1, 128, "bf16"),
    "short": ([0] * 40, [40, 1, 20, 33] * 10, 2, 2, 64, "bf16"),
    "f32-16": ([0, 1, 64, 90], [1, 5, 64, 3], 4, 4, 16, "f32"),
    "f32-64": ([0, 300], [70, 1], 4, 2, 64, "f32"),
    "f32-128": ([5, 129], [9, 1], 6, 2, 128, "f32"),
    "f32-32-one": ([2000, 0], [1, 1], 2, 1, 32, "f32"),
}
WINDOWS = [(0, 0), (1, 0), (1, 1), (7, 3), (64, 4), (100, 0), (65, 130), (1000, 64), (1 << 30, 5), (90, 1 << 30)]


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("kind", ["plain", "4bit"])
def test_windows_over_both_formats(T, name, kind):
    import torch
    old, new, hq, hkv, hd, dtype = SHAPES[name]
    c = _cache(kind, old, new, hq, hkv, hd, dtype, seed=len(name))
    d = c.device()
    for window, first in WINDOWS:
        ref = W.attention(c, window, first)
        got = _attend(T, c, d, window, first)
        try:
            _hold(c, d, got, ref)
        except AssertionError as e:
            raise AssertionError(f"window {window}, first {first}: {e}") from e
    # the same inputs give the same bits
    again = _attend(T, c, d, window, first)
    assert all(torch.equal(x[:c.T], y[:c.T]) for x, y in zip(got, again))


def test_without_a_window_a_plain_cache_is_the_chunk_attention(T):
    import torch
    from test_gpu_serve_ops import _attend as chunk
    c = R.Cache([70, 0, 300], [1, 90, 7], 4, 2, 128, "bf16", seed=2)
    d = c.device()
    a, b = _attend(T, c, d, 0, 9), chunk(T, c, d)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("kind", ["plain", "4bit"])
@pytest.mark.parametrize("new,max_chunk", [([1, 1, 1], 1), ([3, 1, 0], 3), ([90, 150, 1], 150)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing_and_rows_without_entries(T, kind, new, max_chunk, dtype):
    """lens smaller than the new tokens: the first queries see nothing."""
    c = _cache(kind, [5, 100, 0], new, 4, 2, 64, dtype, seed=3)
    c.lens = np.array([0, max(0, new[1] - 2), c.lens[2]])
    d = c.device()
    for window, first in ((0, 0), (5, 0), (30, 2)):
        _hold(c, d, _attend(T, c, d, window, first, max_chunk=max_chunk), W.attention(c, window, first))


@pytest.mark.parametrize("kind", ["plain", "4bit"])
@pytest.mark.parametrize("new", [[1, 1], [6, 2], [140, 70]], ids=["one", "few", "many"])
@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "bf16"), (64, "f32")])
@pytest.mark.parametrize("window,first", [(0, 0), (40, 3), (100, 70)])
def test_what_no_query_sees_does_not_reach_any(T, kind, new, hd, dtype, window, first):
    """Entries behind the caches, between the first ones and the window, and pages of nobody hold NaN, infinities or bits at
    random; places of the page table whose pages no query sees name no page, and nothing is reported."""
    for bad in (np.nan, np.inf, -np.inf):
        c = _cache(kind, [700, 30], new, 4, 2, hd, dtype, seed=11)
        ref = W.attention(c, window, first)
        keep = np.zeros((c.pages, 64), bool)
        for b in range(c.n):
            m = np.any([W.sees(c, b, i, window, first) for i in range(c.new[b])], 0)
            keep[c.at(b, np.nonzero(m)[0])] = True
            m = np.pad(m, (0, c.table.shape[1] * 64 - len(m)))
            for p in np.nonzero(~m.reshape(-1, 64).any(1))[0]:
                c.table[b, p] = [-1, 1 << 30, -(1 << 31), c.pages][p % 4]
        if kind == "plain":
            c.pool = np.where(~keep[:, None, None, None, :, None], np.float32(bad), c.pool)
        else:
            codes, pairs = W.parts(c.pool4, hd)
            hide = ~keep[:, None, None, None, :, None]
            pairs = np.where(hide[..., None], W.bits(np.float32(bad))[()], pairs)
            c.pool4 = W.blocks(np.where(hide, np.uint8(255), codes), pairs)
        d = c.device()
        _hold(c, d, _attend(T, c, d, window, first), ref)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("new", [[5, 3], [40, 33], [200, 140]], ids=["few", "middle", "many"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("window,first", [(30, 0), (64, 2), (150, 70), (3, 400)])
def test_values_without_a_number_reach_those_that_see_them(T, bad, new, hd, window, first):
    """Values of entries that some queries see and others do not, at the window's edge, among the first entries and in the chunk."""
    c = R.Cache([100, 333], new, 4, 2, hd, "bf16", seed=hd + window)
    ref = W.attention(c, window, first)
    want = ref[0].copy()
    for b in range(c.n):
        for e, dim in ((c.lens[b] - 2, 5), (c.old[b] + 1, 9), (c.old[b] - 20, 30), (max(0, c.old[b] - window + 2), 9), (1, 63)):
            p, o = c.at(b, np.array([e]))
            c.pool[p, c.layer, 1, :, o, dim] = bad
            for i in range(c.new[b]):
                if W.sees(c, b, i, window, first)[e]:
                    want[c.cu[b] + i, :, dim] = bad
    d = c.device()
    out, lse = _attend(T, c, d, window, first)
    o = out.float().cpu().numpy().astype(np.float64)
    odd = ~np.isfinite(want)
    assert np.array_equal(np.isnan(o[odd]), np.isnan(want[odd])) and np.array_equal(o[odd & ~np.isnan(want)], want[odd & ~np.isnan(want)])
    p_rel = 4 * (hd + 8) * U * ref[3] + 2.0 ** -19
    bound = (p_rel[..., None] + RB) * ref[2] + (RB + 4 * U) * np.abs(ref[0]) * (1 + RB) + 1e-30
    assert (np.abs(o - ref[0])[~odd] <= bound[~odd]).all()
    assert int(d["err"][0].item()) == 0


@pytest.mark.parametrize("kind", ["plain", "4bit"])
@pytest.mark.parametrize("new", [[1, 1], [5, 2], [90, 150]], ids=["one", "few", "many"])
@pytest.mark.parametrize("dtype,hd", [("f32", 64), ("bf16", 64), ("bf16", 128)])
def test_a_page_that_is_not_there_is_left_out(T, kind, new, dtype, hd):
    """Page ids outside the pool where queries do look."""
    c = _cache(kind, [300, 2000], new, 4, 2, hd, dtype, seed=31)
    full = W.sees
    gone = [(0, 1), (0, 3), (1, 0), (1, 30), (1, int(c.lens[1] - 1) // 64)]

    def without(c, b, i, window, first):
        m = full(c, b, i, window, first)
        for r, p in gone:
            if r == b:
                m[p * 64:p * 64 + 64] = False
        return m
    d = c.device()
    for k, (b, p) in enumerate(gone):
        d["table"][b, p] = [-1, c.pages, 1 << 30][k % 3]
    for window, first in ((0, 0), (400, 10)):
        W.sees = without
        try:
            ref = W.attention(c, window, first)
        finally:
            W.sees = full
        d["err"].zero_()
        got = _attend(T, c, d, window, first)
        err = int(d["err"][0].item())
        assert err in (0, 2) and (window or err == 2)
        _hold(c, d, got, ref, err=err)


@pytest.mark.parametrize("kind", ["plain", "4bit"])
def test_strides_scale_and_stream(T, kind):
    import torch
    for new in ([4, 1], [100, 40]):
        c = _cache(kind, [64, 33], new, 4, 2, 64, "bf16", seed=8)
        d = c.device()
        wide = torch.zeros(c.T, 7, c.hq * c.hd + 24, dtype=torch.bfloat16, device="cuda")
        ref = W.attention(c, 50, 2, 0.3)
        s = torch.cuda.Stream()
        for pad, at in ((8, 8), (3, 1)):  # rows at multiples of 16 bytes, and not
            odd = torch.zeros(c.T, c.hq * c.hd + pad, dtype=torch.bfloat16, device="cuda")
            q = (wide[:, 2, at:at + c.hq * c.hd] if pad == 8 else odd[:, :c.hq * c.hd]).unflatten(1, (c.hq, c.hd))
            q.copy_(d["q"][:c.T])
            out = torch.full((c.T, c.hq * c.hd + pad), 3.0, dtype=torch.bfloat16, device="cuda")
            s.wait_stream(torch.cuda.current_stream())
            got = _attend(T, c, dict(d, q=q), 50, 2, 0.3, stream=s, out=out[:, :c.hq * c.hd].unflatten(1, (c.hq, c.hd)))
            _hold(c, d, got, ref)
            assert (out[:, c.hq * c.hd:] == 3).all()


def test_scales_of_a_4bit_cache_far_apart(T):
    """Groups whose values differ by many orders of magnitude, groups of one value, and entries that dominate."""
    for new in ([1, 1], [5, 8], [70, 140]):
        for hd in (64, 128):
            c = W.Cache4([100, 500], new, 4, 2, hd, "bf16", seed=hd)
            mag = 10.0 ** c.rng.uniform(-12, 6, c.pool.shape[:-1] + (1,))
            c.pool = np.where(np.arange(2)[:, None, None, None] == 1, c.pool * mag, c.pool).astype(np.float32)  # values
            c.pool[..., 5::7, :] = c.pool[..., 5::7, :1]  # entries of one value
            c.pool4 = W.blocks(*W.quantise(c.round(c.pool)))
            d = c.device()
            for window, first in ((0, 0), (33, 5)):
                ref = W.attention(c, window, first)
                got = _attend(T, c, d, window, first)
                # what a large entry adds with a tiny probability is rounded to the row's largest term, not to its own
                top = ref[2].max(-1, keepdims=True)
                _hold(c, d, got, (ref[0], ref[1], np.maximum(ref[2], top), ref[3]))


# ---- the 4-bit cache ----

PACK = {
    # old, new, hq, hkv, hd, dtype, rot, layout
    "half-64": ([0, 1, 63, 200], [1, 70, 2, 0], 4, 2, 64, "bf16", 64, "half"),
    "half-128-part": ([5, 64], [64, 1], 4, 2, 128, "bf16", 64, "half"),
    "half-128": ([5, 64], [3, 130], 2, 1, 128, "bf16", 128, "half"),
    "inter-64": ([0, 7], [9, 1], 6, 2, 64, "bf16", 32, "interleaved"),
    "inter-128": ([0], [300], 8, 8, 128, "bf16", 128, "interleaved"),
    "half-many": ([0, 7], [2500, 1200], 4, 4, 64, "bf16", 64, "half"),
    "f32-many": ([3, 0], [1500, 900], 4, 2, 64, "f32", 64, "interleaved"),
    "odd-rot": ([3, 60], [5, 8], 3, 1, 64, "bf16", 10, "half"),
    "odd-rot-inter": ([3, 60], [5, 8], 3, 3, 32, "bf16", 6, "interleaved"),
    "32": ([0, 50], [20, 30], 4, 2, 32, "bf16", 32, "half"),
    "f32-16": ([0, 63], [5, 2], 4, 4, 16, "f32", 16, "half"),
    "f32-32": ([1], [65], 4, 2, 32, "f32", 16, "half"),
    "f32-64": ([0, 10], [1, 90], 2, 2, 64, "f32", 64, "interleaved"),
    "f32-128": ([100], [7], 2, 1, 128, "f32", 96, "half"),
}


def _pack_problem(T, name, seed=0, aligned=True):
    import torch
    old, new, hq, hkv, hd, dtype, rot, layout = PACK[name]
    c = W.Cache4(old, new, hq, hkv, hd, dtype, seed=seed + len(name))
    d = c.device()
    rng, dt = np.random.default_rng(seed), torch.bfloat16 if dtype == "bf16" else torch.float32
    width = (hq + 2 * hkv) * hd + (0 if aligned else 3)
    x = torch.tensor(c.round(rng.standard_normal((max(1, c.T), width)) * 2)).to(dt).cuda()
    max_pos = 5000
    table = torch.empty(max_pos, rot // 2, 2, device="cuda")
    T.tlf_rope_table(T.rope_config(rot), max_pos, table)
    pos = torch.tensor(rng.integers(0, max_pos, max(1, c.T)).astype(np.int32)).cuda()
    parts = x[:, :(hq + 2 * hkv) * hd].split([hq * hd, hkv * hd, hkv * hd], 1)
    return c, d, parts, pos, table, rot, layout, dt


def _turned32(x, cs, rot, layout):
    """float32 values turned with every product and sum rounded on its own."""
    y = x.copy()
    co, si = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    xa, xb = x[..., a], x[..., b]
    y[..., a], y[..., b] = xa * co - xb * si, xb * co + xa * si
    return y


@pytest.mark.parametrize("name", PACK)
@pytest.mark.parametrize("aligned", [True, False])
def test_append_to_a_4bit_cache_and_read_back(T, name, aligned):
    import torch
    c, d, (q, k, v), pos, table, rot, layout, dt = _pack_problem(T, name, aligned=aligned)
    q_out = torch.full((max(1, c.T), c.hq, c.hd), 7.0, dtype=dt, device="cuda")
    entry_pos = torch.full((c.pages, 64), -5, dtype=torch.int32, device="cuda")
    weight = torch.full((c.pages, 64), 3.0, device="cuda")
    b = _batch(T, c, d)
    a = T.rope_args(q, k, v, pos, table, q_out, layout=layout, entry_pos=entry_pos, entry_weight=weight)
    T.tlf_kv4_append(b, a)
    k_out, v_out = (torch.full((max(1, c.T), c.hkv, c.hd), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    T.tlf_kv4_read(b, T.kv4_read_args(k_out, v_out))
    torch.cuda.synchronize()
    cs = table.cpu().numpy()[pos.cpu().numpy()]
    f = lambda x, h: x.float().cpu().numpy().reshape(-1, h, c.hd)  # noqa: E731
    kk, vv = c.round(_turned32(f(k, c.hkv), cs, rot, layout)), f(v, c.hkv)
    want, wpos, ww = c.pool4.copy(), np.full((c.pages, 64), -5), np.full((c.pages, 64), 3.0)
    codes, pairs = (x.copy() for x in W.parts(want, c.hd))
    hold = [np.zeros((c.T, c.hkv, c.hd)) for _ in range(2)]
    for r in range(c.n):
        t = np.arange(c.cu[r], c.cu[r + 1])
        p, o = c.at(r, c.old[r] + t - c.cu[r])
        for i, x in enumerate((kk, vv)):
            n, pr = W.quantise(x[t])
            codes[p, c.layer, i, :, o], pairs[p, c.layer, i, :, o] = n, pr
            hold[i][t] = sum(W.terms(n, pr))
        wpos[p, o], ww[p, o] = pos.cpu().numpy()[t], 0
    assert np.array_equal(d["pool"].cpu().numpy(), W.blocks(codes, pairs))  # every byte, the others' too
    assert np.array_equal(entry_pos.cpu().numpy(), wpos) and np.array_equal(weight.cpu().numpy(), ww)
    for got, x in zip((k_out, v_out), hold):
        assert np.array_equal(got.float().cpu().numpy()[:c.T], c.round(x.astype(np.float32)))
    exact = R.turn(f(q, c.hq), cs, rot, layout)
    # two products and a sum in float32 (3 u of the terms' magnitudes), rounded once to the type
    mag = np.abs(f(q, c.hq)) + np.abs(R.turn(np.abs(f(q, c.hq)), np.abs(cs), rot, layout)) + np.abs(R.turn(np.abs(f(q, c.hq)), -np.abs(cs), rot, layout))
    r = RB if c.dtype == "bf16" else U
    assert (np.abs(q_out.float().cpu().numpy()[:c.T] - exact[:c.T]) <= (r * np.abs(exact) + 4 * U * mag + 1e-30)[:c.T]).all()
    assert int(d["err"][0].item()) == 0


def test_4bit_groups_of_one_value_and_what_they_cannot_hold(T):
    """Constant groups, zeros, the type's ends, infinities and NaN: the bytes of the definition, and err bit 8 for the last two."""
    import torch
    c, d, (q, k, v), pos, table, rot, layout, dt = _pack_problem(T, "half-64", seed=4)
    v = v.clone()
    v[0] = 3.0
    v[1] = 0.0
    v[2, 5], v[2, 6] = 1e38, -1e38  # past 2^126: held as that
    T.tlf_kv4_append(_batch(T, c, d), T.rope_args(q, k, v, pos, table, torch.empty(c.T, c.hq, c.hd, dtype=dt, device="cuda")))
    assert int(d["err"][0].item()) == 8
    d["err"].zero_()
    v[2, 5:7] = 1.0
    v[3, 0], v[4, 1], v[5, 2] = 2.0 ** 126, float("nan"), float("-inf")
    v[6, 3], v[6, 4] = -(2.0 ** 126), 1e-38
    T.tlf_kv4_append(_batch(T, c, d), T.rope_args(q, k, v, pos, table, torch.empty(c.T, c.hq, c.hd, dtype=dt, device="cuda")))
    assert int(d["err"][0].item()) == 8
    got = d["pool"].cpu().numpy()
    codes, pairs = W.parts(got, c.hd)
    vv = v.float().cpu().numpy().reshape(-1, c.hkv, c.hd)
    for r in range(c.n):
        t = np.arange(c.cu[r], c.cu[r + 1])
        p, o = c.at(r, c.old[r] + t - c.cu[r])
        n, pr = W.quantise(vv[t])
        assert np.array_equal(codes[p, c.layer, 1, :, o], n) and np.array_equal(pairs[p, c.layer, 1, :, o], pr)


def test_append_and_read_with_bad_positions_pages_and_lengths(T):
    """A position out of range: a zero query and no entry; no page, or no entry: the query alone; reading gives zeros there."""
    import torch
    c, d, (q, k, v), pos, table, rot, layout, dt = _pack_problem(T, "half-64", seed=9)
    c.lens[3] = 0
    d["pos_bad"] = pos.clone()
    d["pos_bad"][0], d["pos_bad"][5] = -1, 5000
    bad_page = c.table[1, 1]
    d["table"][1, 1] = c.pages + 3  # entries 64.. of row 1
    q_out = torch.full((c.T, c.hq, c.hd), 7.0, dtype=dt, device="cuda")
    before = d["pool"].clone()
    b = _batch(T, c, d)
    T.tlf_kv4_append(b, T.rope_args(q, k, v, d["pos_bad"], table, q_out))
    out = torch.full((c.T, c.hkv, c.hd), float("nan"), dtype=dt, device="cuda")
    T.tlf_kv4_read(b, T.kv4_read_args(None, out))
    torch.cuda.synchronize()
    assert int(d["err"][0].item()) == 2
    assert (q_out[0] == 0).all() and (q_out[5] == 0).all() and (q_out[1:5].float().abs().sum((1, 2)) > 0).all()
    after = d["pool"]
    assert torch.equal(after[int(bad_page)], before[int(bad_page)])
    e = c.at(1, np.array([c.old[1] + 4]))  # token 5 is row 1's fifth
    for x, y in zip(W.parts(after.cpu().numpy(), c.hd), W.parts(before.cpu().numpy(), c.hd)):
        assert np.array_equal(x[e[0], :, :, :, e[1]], y[e[0], :, :, :, e[1]])
    assert (out[1 + 63:1 + 70] == 0).all() and torch.isfinite(out.float()).all()


# ---- pages ----

def _pages_problem(seed, n_in, n_out, width, most, shared, kind, hd=64, layers=2, hkv=2, spare=20):
    """Rows over a pool, some of whose full pages several rows share (prefixes); random parents."""
    import torch
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, most + 1, n_in)
    lens[rng.integers(0, n_in)] = most // 64 * 64
    need = -(-lens // 64)
    held = -(-(lens + rng.integers(0, 100, n_in)) // 64)  # some rows have room for tokens to come
    held = np.minimum(held, width)
    pages = int(held.sum()) + spare
    ids = rng.permutation(pages)
    table, refs, at = np.full((n_in, width), -1, np.int32), np.zeros(pages, np.int32), 0
    for b in range(n_in):
        for s in range(held[b]):
            if shared and b and s < min(lens[b], lens[b - 1]) // 64 and table[b - 1, s] >= 0 and rng.random() < 0.7:
                table[b, s] = table[b - 1, s]
            elif shared and rng.random() < 0.1 and s < need[b] - 1:
                continue  # given up by a window before
            else:
                table[b, s] = ids[at]
                at += 1
            refs[table[b, s]] += 1
    refs[ids[at:at + 2]] = 1  # of others
    parents = rng.integers(-1, n_in, n_out).astype(np.int32)
    if kind == "4bit":
        pool = rng.integers(0, 256, (pages, layers, 2, hkv, W.PAGE * (hd // 2 + 4 * W.groups(hd)))).astype(np.uint8)
    else:
        pool = rng.standard_normal((pages, layers, 2, hkv, 64, hd)).astype(np.float32)
    pos = rng.integers(0, 1000, (pages, 64)).astype(np.int32)
    dev = lambda x: torch.tensor(x).cuda()  # noqa: E731
    return table, lens.astype(np.int32), parents, refs, pool, pos, dev


FORKS = [
    # n_in, n_out, width, most, reserve, window, first, shared, kind, spare
    (1, 1, 4, 100, 1, 0, 0, False, "plain", 9), (5, 9, 9, 400, 1, 0, 0, True, "plain", 60), (64, 64, 6, 300, 70, 0, 0, True, "4bit", 200),
    (3, 200, 5, 200, 0, 0, 0, False, "plain", 250), (40, 7, 8, 500, 200, 100, 3, True, "plain", 60), (9, 30, 7, 380, 5, 64, 70, True, "4bit", 60),
    (9, 30, 7, 380, 5, 1, 0, True, "plain", 60), (6, 50, 5, 300, 40, 0, 0, False, "plain", 12), (4, 6, 4, 256, 300, 0, 0, True, "plain", 40),
    (2000, 3000, 3, 150, 64, 0, 0, True, "plain", 9000), (12, 12, 5, 300, 10, 5000, 2, True, "4bit", 40)]


@pytest.mark.parametrize("case", FORKS, ids=lambda v: "-".join(map(str, v)))
def test_fork(T, case):
    import torch
    n_in, n_out, width, most, reserve, window, first, shared, kind, spare = case
    for seed in range(3):
        hd = (64, 128, 32)[seed]
        table, lens, parents, refs, pool, pos, dev = _pages_problem(seed, n_in, n_out, width, most, shared, kind, hd,
                                                                    layers=1 if n_in > 1000 else 2, spare=spare)
        if seed == 1 and n_out > 3:
            parents[:3] = -7, n_in, parents[3]
        side = hd if kind == "4bit" else None
        want = W.fork(pool, table, lens, parents, refs, reserve, window, first, side)
        wpos = W.fork(pos[:, None, None, None, :, None], table, lens, parents, refs, reserve, window, first)[0][:, 0, 0, 0, :, 0]
        for in_place in (False, True):
            d = [dev(x) for x in (pool, table, lens, parents, refs, pos)]
            weight = dev(pos.astype(np.float32))
            out = torch.full((n_out, width), 99, dtype=torch.int32, device="cuda")
            lens_out = d[2] if in_place and n_in == n_out else torch.full((n_out,), 99, dtype=torch.int32, device="cuda")
            refs_out = d[4] if in_place else torch.full_like(d[4], 99)
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            a = T.fork_args(d[0], d[1], d[2], d[3], d[4], out, lens_out, refs_out, reserve=reserve, window=window, n_first=first,
                            entry_pos=d[5], entry_weight=weight, head_dim=side, err=err)
            n = T.tlf_cache_fork_scratch_bytes(a)
            T.tlf_cache_fork(a, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n)
            torch.cuda.synchronize()
            assert int(err.item()) == want[4]
            assert np.array_equal(out.cpu().numpy(), want[1])
            assert np.array_equal(lens_out.cpu().numpy(), want[2])
            assert np.array_equal(refs_out.cpu().numpy(), want[3])
            assert np.array_equal(d[0].cpu().numpy(), want[0])
            assert np.array_equal(d[5].cpu().numpy(), wpos) and np.array_equal(weight.cpu().numpy(), wpos)
            assert np.array_equal(d[1].cpu().numpy(), table)


@pytest.mark.parametrize("kind,hd", [("plain", 64), ("4bit", 128), ("4bit", 16), ("plain", 16)])
@pytest.mark.parametrize("n,most,drop", [(1, 60, 0.0), (30, 400, 0.5), (200, 200, 0.9), (50, 300, 0.0), (4, 100, 1.0), (900, 100, 0.3)])
def test_compact(T, kind, hd, n, most, drop):
    import torch
    table, lens, _, refs, pool, pos, dev = _pages_problem(n, n, 1, most // 64 + 2, most, True, kind, hd, spare=n // 2)
    rng = np.random.default_rng(n)
    refs[:] = 0
    table[rng.random(n) < drop] = -1
    for p in table[table >= 0]:
        refs[p] += 1
    want, wpos = W.compact(pool, table, refs), W.compact(pos, table, refs)[0]
    for in_place in (False, True):
        d = [dev(x) for x in (pool, table, refs, pos)]
        weight = dev(pos.astype(np.float32))
        out = d[1] if in_place else torch.full_like(d[1], 99)
        refs_out = d[2] if in_place else torch.full_like(d[2], 99)
        live, err = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        a = T.compact_args(d[0], d[1], d[2], out, refs_out, live, entry_pos=d[3], entry_weight=weight,
                           head_dim=hd if kind == "4bit" else None, err=err)
        size = T.tlf_cache_compact_scratch_bytes(a)
        T.tlf_cache_compact(a, torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda"), size)
        torch.cuda.synchronize()
        assert int(err.item()) == 0 and int(live.item()) == want[3]
        assert np.array_equal(out.cpu().numpy(), want[1]) and np.array_equal(refs_out.cpu().numpy(), want[2])
        assert np.array_equal(d[0].cpu().numpy(), want[0])
        assert np.array_equal(d[3].cpu().numpy(), wpos) and np.array_equal(weight.cpu().numpy(), wpos)


def test_compact_of_tables_that_name_what_nobody_counts(T):
    import torch
    pool = torch.randn(8, 1, 2, 1, 64, 64, device="cuda")
    table = torch.tensor([[7, 3, -1, 99], [6, -9, 0, 2]], dtype=torch.int32, device="cuda")
    refs = torch.tensor([1, 0, 1, 1, 0, 0, 0, 1], dtype=torch.int32, device="cuda")  # page 6 is named and not counted
    out, refs_out = torch.zeros_like(table), torch.zeros_like(refs)
    live, err = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    a = T.compact_args(pool, table, refs, out, refs_out, live, err=err)
    n = T.tlf_cache_compact_scratch_bytes(a)
    T.tlf_cache_compact(a, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n)
    torch.cuda.synchronize()
    assert out.tolist() == [[1, 3, -1, -1], [-1, -1, 0, 2]] and int(err.item()) == 2
    assert int(live.item()) == 4 and refs_out.tolist() == [1, 1, 1, 1, 0, 0, 0, 0]


# ---- together ----

@pytest.mark.parametrize("window,first", [(0, 0), (100, 4)])
def test_append_attend_fork_and_compact_together(T, window, first):
    """A prompt of every row, answers forked off it, steps of single tokens and a compaction in between: every step's attention is
    that of the whole sequences, kept beside, under the window."""
    import torch
    rng = np.random.default_rng(7)
    hq, hkv, hd, pages, width = 4, 2, 64, 160, 12
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
    pool = torch.randint(0, 256, (pages, 1, 2, hkv, T.kv4_block_bytes(hd)), dtype=torch.uint8, device="cuda")
    table, lens, refs = torch.full((3, width), -1, dtype=torch.int32, device="cuda"), i32([0, 0, 0]), i32(np.zeros(pages))
    max_pos = 900
    rope = torch.empty(max_pos, hd // 2, 2, device="cuda")
    T.tlf_rope_table(T.rope_config(hd), max_pos, rope)
    seqs = [[], [], []]  # (k, v) of every entry of every row
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def fork(parents, reserve):
        nonlocal table, lens, refs, seqs
        out, lo, ro = torch.zeros(len(parents), width, dtype=torch.int32, device="cuda"), i32(parents), torch.zeros_like(refs)
        a = T.fork_args(pool, table, lens, i32(parents), refs, out, lo, ro, reserve=reserve, window=window, n_first=first, head_dim=hd, err=err)
        n = T.tlf_cache_fork_scratch_bytes(a)
        T.tlf_cache_fork(a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
        table, lens, refs, seqs = out, lo, ro, [list(seqs[p]) if p >= 0 else [] for p in parents]

    def step(new):
        nonlocal lens
        new = np.asarray(new)
        cu = np.concatenate([[0], np.cumsum(new)])
        n = int(cu[-1])
        lens = lens + i32(new)
        x = torch.tensor(R.bf16(rng.standard_normal((n, (hq + 2 * hkv) * hd)))).bfloat16().cuda()
        q, k, v = x.split([hq * hd, hkv * hd, hkv * hd], 1)
        pos = np.concatenate([len(s) + np.arange(m) for s, m in zip(seqs, new)]).astype(np.int32)
        q_out, out = (torch.empty(n, hq, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lse = torch.empty(n, hq, device="cuda")
        b = T.chunk4_args(pool, table, i32(cu), lens, hq, n, hd, max_chunk=int(new.max()), err=err)
        T.tlf_kv4_append(b, T.rope_args(q, k, v, i32(pos), rope, q_out))
        a = T.attn_window_args(q_out, out, lse=lse, window=window, n_first=first, kv4=True)
        size = T.tlf_attn_window_scratch_bytes(b, a)
        T.tlf_attn_window(b, a, torch.empty(size, dtype=torch.uint8, device="cuda"), size)
        torch.cuda.synchronize()
        assert int(err.item()) == 0
        kk = R.bf16(_turned32(k.float().cpu().numpy().reshape(n, hkv, hd), rope.cpu().numpy()[pos], hd, "half"))
        vv = v.float().cpu().numpy().reshape(n, hkv, hd)
        held = [W.terms(*W.quantise(y)) for y in (kk, vv)]
        for r, m in enumerate(new):
            seqs[r] += [(held[0][0][t], held[0][1][t], held[1][0][t], held[1][1][t]) for t in range(cu[r], cu[r + 1])]

        class Whole(W.Cache4):
            def __init__(self):
                self.T, self.hq, self.hkv, self.hd, self.n, self.dtype = n, hq, hkv, hd, len(new), "bf16"
                self.cu, self.new, self.lens = cu, new, np.array([len(s) for s in seqs])
                self.q = q_out.float().cpu().numpy()

            def two(self, r, kv):
                return tuple(np.array([e[2 * kv + i] for e in seqs[r]]).reshape(-1, hkv, hd) for i in range(2))
        c = Whole()
        _hold(c, {"err": err}, (out, lse), W.attention(c, window, first))

    fork([-1, -1, -1], 300)
    step([300, 65, 128])
    fork([0, 0, 1, 2, 2, 2, 0], 1)
    for i in range(3):
        step([1] * 7)
        fork([0, 1, 1, 2, 3, 4, 5], 1)
    out, ro, live = torch.zeros_like(table), torch.zeros_like(refs), i32([0])
    a = T.compact_args(pool, table, refs, out, ro, live, head_dim=hd, err=err)
    n = T.tlf_cache_compact_scratch_bytes(a)
    T.tlf_cache_compact(a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    assert int(out.max().item()) < int(live.item()) == int((refs > 0).sum().item())
    table, refs = out, ro
    pool[int(live.item()):] = 255  # given back
    step([1, 0, 1, 1, 1, 0, 1])
    fork([6, 5, 0, -1], 80)
    step([70, 1, 3, 80])
    table[:] = -1
    assert int((refs < 0).sum().item()) == 0


@pytest.mark.parametrize("new", [1, 6, 100])
def test_a_captured_step_replays_on_changed_buffers(T, new):
    """Append, attention and fork in a graph; replayed after the inputs have changed, with eager calls in between."""
    import torch
    c = W.Cache4([70, 129, 64], [new] * 3, 4, 2, 64, "bf16", seed=new)
    d = c.device()
    q, out, lse = d["q"], torch.zeros(c.T, c.hq, c.hd, dtype=torch.bfloat16, device="cuda"), torch.zeros(c.T, c.hq, device="cuda")
    b = _batch(T, c, d, max_chunk=new)
    a = T.attn_window_args(q, out, lse=lse, window=90, n_first=2, kv4=True)
    scratch = torch.zeros(T.tlf_attn_window_scratch_bytes(b, a), dtype=torch.uint8, device="cuda")
    kv = [torch.zeros(c.T, c.hkv, c.hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    read = T.kv4_read_args(*kv)

    def call(s):
        T.tlf_kv4_read(b, read, s)
        T.tlf_attn_window(b, a, scratch, scratch.numel(), s)

    call(torch.cuda.current_stream())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(torch.cuda.current_stream())
    other = W.Cache4([70, 129, 64], [new] * 3, 4, 2, 64, "bf16", seed=new + 50)
    other.table = c.table
    q.copy_(other.device()["q"])
    d["pool"].copy_(other.device()["pool"])
    for _ in range(2):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        _hold(other, d, (out, lse), W.attention(other, 90, 2))
        first = out.clone()
        call(torch.cuda.current_stream())
        assert torch.equal(out, first)


def test_a_pool_whose_bytes_pass_32_bits(T):
    """Pages past 2^32 bytes from the pool's start, in both formats, and in a fork."""
    import torch
    for kind in ("plain", "4bit"):
        c = _cache(kind, [100, 70], [1, 40], 4, 2, 128, "bf16", layers=1, layer=0, seed=3)
        d = c.device()
        size = d["pool"][0].numel() * d["pool"].element_size()
        far = (1 << 32) // size + 5
        big = torch.empty((far + c.pages,) + tuple(d["pool"].shape[1:]), dtype=d["pool"].dtype, device="cuda")
        big[far:] = d["pool"]
        d["pool"] = big
        d["table"] = torch.where(d["table"] >= 0, d["table"] + far, -1)
        _hold(c, d, _attend(T, c, d, 90, 3), W.attention(c, 90, 3))
        free = [int(p) for p in np.setdiff1d(np.arange(c.pages), c.table)]
        refs = torch.ones(len(big), dtype=torch.int32, device="cuda")
        refs[torch.tensor([far + p for p in free], device="cuda")] = 0
        out, lens, ro = torch.zeros(3, c.table.shape[1], dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros_like(refs)
        parents = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
        f = T.fork_args(big, d["table"], d["lens"], parents, refs, out, lens, ro, head_dim=128 if kind == "4bit" else None)
        n = T.tlf_cache_fork_scratch_bytes(f)
        T.tlf_cache_fork(f, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
        torch.cuda.synchronize()
        page, old = int(out[2, 1].item()), int(d["table"][0, 1].item())
        assert page == far + min(free)
        k = int(c.lens[0]) % 64
        if kind == "plain":
            assert torch.equal(big[page, :, :, :, :k], big[old, :, :, :, :k])
        else:
            assert torch.equal(big[page, ..., :k * 64], big[old, ..., :k * 64]) and torch.equal(big[page, ..., 4096:4096 + 8 * k], big[old, ..., 4096:4096 + 8 * k])
        del big, d
