"""Attention over 4-bit caches at the ends of what they hold: values, keys, queries and scales of any magnitude.

Bounds as in test_gpu_window_ops, with a little more for the statistics: they are kept relative to powers of two of up to 126 to
either side, so that sums and differences of numbers below 256 are rounded to half a step of 2^-16 up to four times, each a
relative error of 2^-17 ln 2 of a probability: 2^-15 in all, in lse and, beside the rounding to bfloat16, in out.
"""
import numpy as np
import pytest

import _serve_ref as R
import _window_ref as W
from test_gpu_window_ops import RB, T, U, _attend  # noqa: F401

pytestmark = pytest.mark.gpu
STAT = 2.0 ** -15


def _hold_far(c, d, got, ref, tokens=None):
    out, lse, spread, terms = (x if tokens is None else x[tokens] for x in ref)
    D = 2 * (c.hd + 8) * U * terms
    o, l = (x[:c.T].float().cpu().numpy().astype(np.float64) for x in got)
    if tokens is not None:
        o, l = o[tokens], l[tokens]
    bound = (2 * D + STAT + RB)[..., None] * spread + (RB + 4 * U) * np.abs(out) * (1 + RB)
    assert np.isfinite(o).all() and (np.abs(o - out) <= bound).all(), np.nanmax(np.abs(o - out) / np.maximum(bound, 1e-300))
    lb = D + STAT + 2 * U * np.abs(lse)
    assert (np.abs(l - lse) <= lb).all(), np.max(np.abs(l - lse) / lb)
    assert int(d["err"][0].item()) == 0


def _filled(c, what, size, seed=0):
    """Values of about `size`: each entry's all the same, the same behind 150 entries of zeros, or at random."""
    rng = np.random.default_rng(seed)
    v = c.pool[:, :, 1]
    if what == "random":
        v *= np.float32(size / 16)  # (heads off centre and entries four times the others: up to 2^4)
        np.clip(v, -size, size, out=v)
    else:
        v[:] = (size * rng.choice([-1.0, 1.0], v.shape[:-1] + (1,)) * rng.uniform(0.5, 1, v.shape[:-1] + (1,))).astype(np.float32)
    if what == "zeros":
        for b in range(c.n):
            p, o = c.at(b, np.arange(min(150, c.lens[b])))
            c.pool[p, c.layer, 1, :, o] = 0
    c.pool4 = W.blocks(*W.quantise(c.round(c.pool)))


@pytest.mark.parametrize("what", ["one value", "zeros", "random"])
@pytest.mark.parametrize("old,new,hq,hkv,hd", [
    ([0, 0, 40], [1, 1, 1], 4, 2, 64), ([5000, 300], [1, 1], 4, 2, 128), ([600, 150], [1, 1], 4, 4, 32), ([3000, 0], [3, 1], 8, 2, 128),
    ([5000, 300], [9, 16], 2, 2, 64)], ids=["one", "ones", "ones-32", "few", "few-64"])
@pytest.mark.parametrize("size", [2.0 ** -70, 2.0 ** -40, 2.0 ** 13, 2.0 ** 28, 2.0 ** 70, 2.0 ** 126])
def test_values_of_any_magnitude_few_tokens(T, what, old, new, hq, hkv, hd, size):
    """32768 entries of 8192, or one of 2^28, in all dims once passed float32's range in the sums."""
    c = W.Cache4(old, new, hq, hkv, hd, "bf16", seed=hd)
    _filled(c, what, min(size, 2.0 ** 100) if what == "random" else size)
    d = c.device()
    for window, first in ((0, 0), (70, 3)):
        _hold_far(c, d, _attend(T, c, d, window, first, max_chunk=max(new)), W.attention(c, window, first))


@pytest.mark.parametrize("new", [[1, 1], [4, 7]], ids=["one", "few"])
@pytest.mark.parametrize("hd", [64, 128])
def test_magnitudes_beside_each_other_few_tokens(T, new, hd):
    """Entries from 2^-70 to 2^90, some with all values alike, some with large scores. What a small term adds is rounded to the row's
    largest."""
    c = W.Cache4([700, 200], new, 4, 2, hd, "bf16", seed=hd + 1)
    rng = np.random.default_rng(5)
    c.pool[:, :, 1] *= (2.0 ** rng.uniform(-70, 90, c.pool[:, :, 1].shape[:-1] + (1,))).astype(np.float32)
    c.pool[:, :, 1, :, 5::7] = c.pool[:, :, 1, :, 5::7, :1]
    c.pool[:, :, 0, :, 3::50] *= 20
    c.pool4 = W.blocks(*W.quantise(c.round(c.pool)))
    d = c.device()
    for window, first in ((0, 0), (33, 5)):
        ref = W.attention(c, window, first)
        top = ref[2].max(-1, keepdims=True)
        _hold_far(c, d, _attend(T, c, d, window, first, max_chunk=max(new)), (ref[0], ref[1], np.maximum(ref[2], top), ref[3]))


def _scaled(c, q, every):
    """Queries times q, every third one zero, every other third (the one behind it) as `every` says."""
    c.q = R.bf16(c.q * np.float32(q))
    c.q[::3] = 0
    c.q[1::3] = R.bf16(c.q[1::3] * np.float32(every))


@pytest.mark.parametrize("scale,q", [(1e19, 2.0 ** -63), (1e31, 2.0 ** -103), (1e31, 1.0), (1e35, 2.0 ** -116), (1e35, 1.0), (2e38, 2.0 ** -122)])
@pytest.mark.parametrize("new,hq,hkv,hd", [([1, 1], 4, 2, 64), ([2, 3], 8, 2, 128), ([9, 12], 2, 2, 64), ([3, 1], 4, 4, 32)],
                         ids=["one", "few", "few-64", "few-32"])
def test_the_largest_scales_few_tokens(T, new, hq, hkv, hd, scale, q):
    """With queries as small as the scale is large, and with ordinary ones, of which the largest score takes all; queries of zeros see
    every entry alike."""
    c = W.Cache4([100, 300], new, hq, hkv, hd, "bf16", seed=hd)
    _scaled(c, q, 2.0 ** -4)
    d = c.device()
    for window, first in ((0, 0), (64, 5)):
        _hold_far(c, d, _attend(T, c, d, window, first, scale, max_chunk=max(new)), W.attention(c, window, first, scale))


@pytest.mark.parametrize("q", [2.0 ** -120, 2.0 ** -40, 2.0 ** 40, 2.0 ** 115])
@pytest.mark.parametrize("new,hq,hkv,hd", [([1, 1], 4, 2, 64), ([2, 3], 8, 2, 128)], ids=["one", "few"])
def test_queries_and_keys_of_any_magnitude_few_tokens(T, new, hq, hkv, hd, q):
    """Keys as small as the queries are large."""
    c = W.Cache4([100, 300], new, hq, hkv, hd, "bf16", seed=hd + 2)
    c.pool[:, :, 0] *= np.float32(1 / q)
    c.pool4 = W.blocks(*W.quantise(c.round(c.pool)))
    _scaled(c, q, 0.5)
    d = c.device()
    for window, first in ((0, 0), (64, 5)):
        _hold_far(c, d, _attend(T, c, d, window, first, max_chunk=max(new)), W.attention(c, window, first))


@pytest.mark.parametrize("scale,q", [(1e8, 1.0), (1e12, 2.0 ** -40), (1e31, 2.0 ** -103), (1e31, 1.0), (1e35, 2.0 ** -116), (1e35, 1.0), (2e38, 2.0 ** -118)])
@pytest.mark.parametrize("hd", [64, 128])
def test_the_largest_scales_many_tokens(T, hd, scale, q):
    c = W.Cache4([100, 300], [60, 90], 4, 2, hd, "bf16", seed=hd)
    _scaled(c, q, 2.0 ** -4)
    d = c.device()
    for window, first in ((0, 0), (64, 5)):
        _hold_far(c, d, _attend(T, c, d, window, first, scale), W.attention(c, window, first, scale))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("to", [2.0 ** 30, 2.0 ** 60])
def test_one_score_beyond_all_others_many_tokens(T, hd, to):
    """Scores of up to `to`: the entry with the largest takes all, whatever rounds beside it. Keys, queries and values are powers of two
    and zeros, so that the largest score is exact and some distance ahead."""
    c = W.Cache4([100, 300], [60, 90], 4, 2, hd, "bf16", seed=hd)
    c.pool[:, :, 0] = 0
    c.q[:] = 0
    c.q[:, :, 3] = 2.0 ** 20
    for b in range(c.n):
        for e, k in ((7, to / 2.0 ** 21), (33, to / 2.0 ** 20), (99, to / 2.0 ** 22)):
            p, o = c.at(b, np.array([e]))
            c.pool[p, c.layer, 0, :, o, 3] = k
    c.pool4 = W.blocks(*W.quantise(c.round(c.pool)))
    d = c.device()
    out, _ = _attend(T, c, d, 0, 0, 1.0)
    o = out.float().cpu().numpy()
    for b in range(c.n):
        vl, vn = c.two(b, 1)
        want = np.repeat((vl + vn)[33], 2, 0)
        assert (np.abs(o[c.cu[b]:c.cu[b + 1]] - want) <= (RB + 2.0 ** -11) * (np.abs(vl) + np.abs(vn))[33].repeat(2, 0)).all()


@pytest.mark.parametrize("values", ["alike", "apart", "zeros"])
@pytest.mark.parametrize("k,q,scale", [(2.0 ** -14, 2.0 ** 14, 0), (2.0 ** -20, 2.0 ** 20, 0), (2.0 ** -28, 1.0, 2.0 ** 25), (2.0 ** -100, 2.0 ** 100, 0),
                                       (2.0 ** -35, 2.0 ** 35, 0), (2.0 ** 20, 2.0 ** -20, 0), (2.0 ** 60, 1.0, 2.0 ** -63), (2.0 ** 115, 2.0 ** -115, 0),
                                       (1.0, 2.0 ** -60, 2.0 ** 57), (2.0 ** -118, 2.0 ** 115, 1.0)])
@pytest.mark.parametrize("new,hd", [([60, 90], 64), ([60, 90], 128), ([2, 3], 64), ([2, 3], 128)], ids=["many-64", "many-128", "few-64", "few-128"])
def test_keys_queries_and_scales_of_any_magnitude(T, new, hd, k, q, scale, values):
    """Small keys under large queries and the other way round, or under scales of any size: the same scores as ever; beside values that are
    alike, 2^-30 to 2^30 and 2^-12 zeros."""
    c = W.Cache4([100, 300], new, 4, 2, hd, "bf16", seed=hd + 3)
    rng = np.random.default_rng(7)
    c.pool[:, :, 0] *= np.float32(k)
    if values == "apart":
        c.pool[:, :, 1] *= (2.0 ** rng.uniform(-30, 30, c.pool[:, :, 1].shape[:-1] + (1,))).astype(np.float32)
    if values == "zeros":
        c.pool[:, :, 1] *= 2.0 ** -12 * rng.integers(0, 2, c.pool[:, :, 1].shape[:-1] + (1,)).astype(np.float32)
    c.pool4 = W.blocks(*W.quantise(c.round(c.pool)))
    _scaled(c, q, 0.5)
    d = c.device()
    for window, first in ((0, 0), (64, 5)):
        ref = W.attention(c, window, first, scale)
        top = ref[2].max(-1, keepdims=True)  # (a small term is rounded to the row's largest)
        _hold_far(c, d, _attend(T, c, d, window, first, scale, max_chunk=max(new)), (ref[0], ref[1], np.maximum(ref[2], top), ref[3]))


@pytest.mark.parametrize("what", ["one value", "zeros", "random"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("size", [2.0 ** -70, 2.0 ** -40, 2.0 ** 28, 2.0 ** 90])
def test_values_of_any_magnitude_many_tokens(T, what, hd, size):
    c = W.Cache4([1000, 150], [60, 90], 4, 2, hd, "bf16", seed=hd)
    _filled(c, what, size)
    d = c.device()
    for window, first in ((0, 0), (70, 3)):
        _hold_far(c, d, _attend(T, c, d, window, first), W.attention(c, window, first))


@pytest.mark.parametrize("what", ["one value", "random"])
@pytest.mark.parametrize("new", [[60, 90], [300, 40]], ids=["parts", "whole"])
@pytest.mark.parametrize("hd", [64, 128])
def test_the_largest_values_many_tokens(T, what, new, hd):
    """1 / l is 2^126 with values of 2^126."""
    c = W.Cache4([1000, 150] if new[0] < 100 else [0, 20], new, 8, 4, hd, "bf16", seed=hd)
    _filled(c, what, 2.0 ** 126)
    d = c.device()
    for window, first in ((0, 0), (70, 3)):
        _hold_far(c, d, _attend(T, c, d, window, first), W.attention(c, window, first))


@pytest.mark.parametrize("scale,q", [(1e8, 1.0), (1e31, 2.0 ** -103), (1e31, 1.0), (1e35, 1.0), (2e38, 2.0 ** -118)])
@pytest.mark.parametrize("new", [[1, 1], [5, 8], [60, 90]], ids=["one", "few", "many"])
@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_the_largest_scales_over_plain_caches(T, dtype, hd, new, scale, q):
    c = R.Cache([100, 300], new, 4, 2, hd, dtype, seed=3)
    _scaled(c, q, 2.0 ** -4)
    d = c.device()
    for window, first in ((0, 0), (64, 5)):
        _hold_far(c, d, _attend(T, c, d, window, first, scale, max_chunk=max(new)), W.attention(c, window, first, scale))
