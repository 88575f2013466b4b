"""Where the operators on paged caches and logits could go wrong for one row because of another, at the ends of their types, and
in the paths that only large calls take. Bounds as in test_gpu_serve_ops."""
import numpy as np
import pytest

import _serve_ref as R
from test_gpu_serve_ops import RB, T, U, _attend, _draw, _hold, _hold_weights  # noqa: F401

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
