"""CPU tests of what the operators on paged caches and logits refuse at the ends of their arguments' ranges."""
import ctypes as C

import pytest

from paper_2609_15160_gb300 import build, tlf

P = 1 << 20  # a made-up device address, aligned; nothing is launched by a refused call


@pytest.fixture(scope="module")
def lib():
    build.build()
    return tlf.load_library()


def test_a_batch_that_changes_is_looked_at_again():
    """Fields of a batch that a program keeps may change between calls: tensors that no longer fit are refused."""
    torch = pytest.importorskip("torch")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    pool = torch.zeros(9, 2, 2, 2, 64, 64, dtype=torch.bfloat16)
    q = torch.zeros(7, 4, 64, dtype=torch.bfloat16)
    for field, value in (("n_tokens", 8), ("n_heads", 2), ("head_dim", 32), ("dtype", 0), ("n_pages", 10)):
        c = tlf.chunk_args(pool, i32(3, 4), i32(4), i32(3), 4, 7)
        a = tlf.attn_chunk_args(q, q, weight_out=torch.zeros(9, 64))
        tlf._pair(c, a)
        tlf._pair(c, a)
        setattr(c, field, value)
        with pytest.raises(ValueError):
            tlf.tlf_attn_chunk(c, a, None, 0)
    c = tlf.chunk_args(pool, i32(3, 4), i32(4), i32(3), 4, 7)
    r = tlf.rope_args(q, q[:, :2], q[:, 2:], i32(7), torch.zeros(9, 32, 2), torch.zeros_like(q))
    tlf._pair(c, r)
    c.n_kv_heads = 1
    with pytest.raises(ValueError):
        tlf.tlf_rope_append(c, r)


def test_evictions_scratch_goes_by_what_a_row_can_hold(lib):
    a = dict(n=2, n_kv_heads=2, head_dim=64, n_layers=1, page_size=64, dtype=1, max_pages=4, n_first=4, n_recent=10, n_pages=9, pool=P,
             page_table=P, lens=P, next_pos=P, pos_in=P, pos_out=P, weight_in=P, weight_out=P, lens_out=P)
    size = lambda b: lib.tlf_cache_evict_scratch_bytes(C.byref(tlf.TlfEvictArgs(budget=b, **a)))  # noqa: E731
    assert size(100) < size(256) == size(257) == size(2 ** 31 - 1) < 1 << 13


@pytest.mark.parametrize("max_pages", [(1 << 25) - 1, (1 << 25) - 64])
def test_page_tables_that_leave_no_room_below_32_bits_are_refused(lib, max_pages):
    """Entries are counted in 32 bits, in strides and rounded up: the last 4096 numbers are room for that."""
    size = lambda m: lib.tlf_cache_evict_scratch_bytes(C.byref(tlf.TlfEvictArgs(  # noqa: E731
        n=2, n_kv_heads=2, head_dim=64, n_layers=1, page_size=64, dtype=1, max_pages=m, budget=9, n_pages=9, pool=P, page_table=P, lens=P,
        next_pos=P, pos_in=P, pos_out=P, weight_in=P, weight_out=P, lens_out=P)))
    assert size(max_pages) == 0 and size((1 << 25) - 65) > 0
    c = tlf.TlfChunk(n=2, n_tokens=5, n_heads=4, n_kv_heads=2, head_dim=64, n_layers=2, page_size=64, dtype=1, max_pages=max_pages,
                     n_pages=20, pool=P, page_table=P, cu_tokens=P, lens=P)
    a = tlf.TlfAttnChunkArgs(q=P, out=P)
    assert lib.tlf_attn_chunk(C.byref(c), C.byref(a), P, 1 << 40, None) == tlf.CODES["INVALID_ARG"]
    assert "max_pages" in lib.tlf_last_error(None).decode()


@pytest.mark.parametrize("scale", [2.5e38, 3.4028234663852886e38, float("inf"), float("-inf"), -1e-45, float("nan")])
def test_a_scale_that_is_not_finite_in_base_2_is_refused(lib, scale):
    c = tlf.TlfChunk(n=2, n_tokens=5, n_heads=4, n_kv_heads=2, head_dim=64, n_layers=2, page_size=64, dtype=1, max_pages=9, n_pages=20,
                     pool=P, page_table=P, cu_tokens=P, lens=P)
    a = tlf.TlfAttnChunkArgs(q=P, out=P, scale=scale)
    assert lib.tlf_attn_chunk(C.byref(c), C.byref(a), None, 0, None) == tlf.CODES["INVALID_ARG"]
    assert "scale" in lib.tlf_last_error(None).decode()
