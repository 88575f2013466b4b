"""Forks and compactions at the sizes where their plans change, of counts that do not fit the tables, beside other calls and captured."""
import numpy as np
import pytest

import _window_ref as W
from test_gpu_window_ops import T  # noqa: F401

pytestmark = pytest.mark.gpu


def _i32(x):
    import torch
    return torch.tensor(np.asarray(x, np.int32)).cuda()


def _compact(T, pool, table, refs, in_place=False, stream=None):
    """(table, refs, live, err) on the device; the pool is changed."""
    import torch
    out, refs_out = (table, refs) if in_place else (torch.full_like(table, 77), torch.full_like(refs, 77))
    live, err = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    a = T.compact_args(pool, table, refs, out, refs_out, live, err=err)
    n = T.tlf_cache_compact_scratch_bytes(a)
    T.tlf_cache_compact(a, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n, stream)
    return out, refs_out, live, err


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pages", [8, 300, 8192, 30000])
def test_compact_leaves_out_what_nobody_counts_before_and_behind_the_live_pages(T, pages, in_place):
    """Tables that name pages with a count of 0: those below the number of live pages once stayed, and named what moved there."""
    import torch
    rng = np.random.default_rng(pages)
    refs = rng.integers(0, 2, pages)
    refs[:2] = (1, 0)
    table = rng.permutation(pages).astype(np.int32).reshape(4, -1)
    pool = torch.arange(pages, device="cuda", dtype=torch.float32).view(pages, 1, 1, 1, 1, 1).repeat(1, 1, 2, 1, 64, 16)
    wp, wt, wr, wl = W.compact(pool.cpu().numpy(), table, refs)
    wt = np.where(refs[table] > 0, wt, -1)
    out, refs_out, live, err = _compact(T, pool, _i32(table), _i32(refs), in_place)
    assert int(err.item()) == 2 and int(live.item()) == wl
    assert np.array_equal(out.cpu().numpy(), wt) and np.array_equal(refs_out.cpu().numpy(), wr)
    assert np.array_equal(pool.cpu().numpy(), wp)
    # every page that is still named holds what it held
    named = wt[wt >= 0]
    assert np.array_equal(pool[torch.as_tensor(named, device="cuda").long(), 0, 0, 0, 0, 0].cpu().numpy(), table[wt >= 0])
