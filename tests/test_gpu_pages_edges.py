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


def _pool(pages, seed, hd=16):
    """A pool whose every entry says which page it is of and where it stands, on the device and on the host."""
    import torch
    p = torch.arange(pages, device="cuda", dtype=torch.float32).view(-1, 1, 1, 1, 1, 1) * 256 + seed
    pool = (p + torch.arange(64, device="cuda", dtype=torch.float32).view(1, 1, 1, 1, 64, 1)).repeat(1, 1, 2, 1, 1, hd)
    return pool, pool.cpu().numpy()


def _live_case(pages, live, seed=0):
    """refs with `live` pages of one owner, in a table of one page a row."""
    rng = np.random.default_rng(seed)
    used = rng.permutation(pages)[:live].astype(np.int32)
    refs = np.zeros(pages, np.int32)
    refs[used] = rng.integers(1, 3, live)
    return (used if live else np.full(1, -1, np.int32)).reshape(-1, 1), refs


@pytest.mark.parametrize("pages", [8191, 8192, 8193, 12000])
@pytest.mark.parametrize("live", [0, 1, 64, 256, 2048, 4096, 8190, -1])
def test_compact_where_plans_change_and_at_the_ends_of_their_runs(T, pages, live):
    """Up to 8192 pages a plan by one CTA, then by a cluster; live pages that end with a warp's run of pages, a CTA's, or the pool."""
    live = pages if live < 0 else live
    pool, host = _pool(pages, 0)
    table, refs = _live_case(pages, live, live)
    want = W.compact(host, table, refs)
    out, refs_out, n, err = _compact(T, pool, _i32(table), _i32(refs))
    assert int(err.item()) == 0 and int(n.item()) == want[3]
    assert np.array_equal(out.cpu().numpy(), want[1]) and np.array_equal(refs_out.cpu().numpy(), want[2])
    assert np.array_equal(pool.cpu().numpy(), want[0])


def _fork_case(n_in, n_out, pages, width, seed=0):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, width * 64 - 70, n_in).astype(np.int32)
    table, ids, at, refs = np.full((n_in, width), -1, np.int32), rng.permutation(pages).astype(np.int32), 0, np.zeros(pages, np.int32)
    for b in range(n_in):
        k = -(-int(lens[b]) // 64)
        table[b, :k] = ids[at:at + k]
        at += k
    refs[ids[:at]] = 1
    refs[ids[at:at + pages // 8]] = 1  # of others
    return table, lens, rng.integers(-1, n_in, n_out).astype(np.int32), refs


class _Fork:
    def __init__(self, T, case, pool, reserve=70, stream=None):
        import torch
        table, lens, parents, refs = (_i32(x) for x in case)
        self.T, self.stream = T, stream
        self.out = torch.full((len(parents), table.shape[1]), 77, dtype=torch.int32, device="cuda")
        self.lens, self.refs, self.err = torch.zeros_like(parents), torch.zeros_like(refs), torch.zeros(1, dtype=torch.int32, device="cuda")
        self.a = T.fork_args(pool, table, lens, parents, refs, self.out, self.lens, self.refs, reserve=reserve, err=self.err)
        self.scratch = torch.full((T.tlf_cache_fork_scratch_bytes(self.a),), 0xFF, dtype=torch.uint8, device="cuda")

    def __call__(self):
        self.T.tlf_cache_fork(self.a, self.scratch, self.scratch.numel(), self.stream)

    def hold(self, want):
        assert int(self.err.item()) == want[4]
        assert np.array_equal(self.out.cpu().numpy(), want[1]) and np.array_equal(self.lens.cpu().numpy(), want[2])
        assert np.array_equal(self.refs.cpu().numpy(), want[3])


@pytest.mark.parametrize("n_in,n_out,pages", [(60, 90, 32768), (60, 90, 32769), (4096, 4096, 16000), (4097, 4096, 16000), (4096, 4097, 16000)])
def test_fork_where_plans_change(T, n_in, n_out, pages):
    """One CTA plans up to 32768 pages and 4096 rows."""
    pool, host = _pool(pages, 1)
    case = _fork_case(n_in, n_out, pages, 5, n_in)
    want = W.fork(host, *case, 70)
    f = _Fork(T, case, pool)
    f()
    f.hold(want)
    assert np.array_equal(pool.cpu().numpy(), want[0])


def test_forks_compactions_and_an_append_on_streams_of_their_own(T):
    """All in flight at once, again and again: plans by one CTA and by clusters, each call with its pool, scratch and outputs."""
    import torch
    streams = [torch.cuda.Stream() for _ in range(5)]
    jobs = []
    for i, (n_in, n_out, pages) in enumerate(((20, 30, 600), (300, 400, 33000))):
        pool, host = _pool(pages, 2 + i)
        case = _fork_case(n_in, n_out, pages, 6, i)
        jobs.append((_Fork(T, case, pool, stream=streams[i]), W.fork(host, *case, 70), pool))
    moves = []
    for i, pages in enumerate((500, 9000)):
        pool, host = _pool(pages, 9 + i)
        table, refs = _live_case(pages, pages // 2, i)
        dev = [_i32(table), _i32(refs)]
        out, refs_out, live, err = torch.zeros_like(dev[0]), torch.zeros_like(dev[1]), _i32([0]), _i32([0])
        a = T.compact_args(pool, *dev, out, refs_out, live, err=err)
        scratch = torch.full((T.tlf_cache_compact_scratch_bytes(a),), 0xFF, dtype=torch.uint8, device="cuda")
        moves.append((lambda a=a, x=scratch, s=streams[2 + i]: T.tlf_cache_compact(a, x, x.numel(), s), W.compact(host, table, refs),
                      pool, out, refs_out, live, err))
    import _serve_ref as R
    rng = np.random.default_rng(0)
    t, hq, hkv, hd = 700, 4, 2, 64
    q, k, v = (torch.tensor(R.bf16(rng.standard_normal((t, h, hd)))).bfloat16().cuda() for h in (hq, hkv, hkv))
    rope = torch.empty(t, hd // 2, 2, device="cuda")
    T.tlf_rope_table(T.rope_config(hd), t, rope)
    cache = [torch.zeros(11, 1, 2, hkv, T.kv4_block_bytes(hd), dtype=torch.uint8, device="cuda") for _ in range(2)]
    table, aerr, q_out = _i32([np.arange(11)[::-1]]), _i32([0]), torch.zeros_like(q)
    app = T.rope_args(q, k, v, _i32(np.arange(t)), rope, q_out)
    batches = [T.chunk4_args(c, table, _i32([0, t]), _i32([t]), hq, t, hd, err=aerr) for c in cache]
    T.tlf_kv4_append(batches[1], app)  # alone
    alone = q_out.clone()
    torch.cuda.synchronize()
    for _ in range(20):
        for f, _, _ in jobs:
            f()
        for m in moves:
            m[0]()
        T.tlf_kv4_append(batches[0], app, streams[4])
    torch.cuda.synchronize()
    for f, want, pool in jobs:
        f.hold(want)
        assert np.array_equal(pool.cpu().numpy(), want[0])
    for _, want, pool, out, refs_out, live, err in moves:
        assert int(err.item()) == 0 and int(live.item()) == want[3] and np.array_equal(out.cpu().numpy(), want[1])
        assert np.array_equal(refs_out.cpu().numpy(), want[2]) and np.array_equal(pool.cpu().numpy(), want[0])
    assert int(aerr.item()) == 0 and torch.equal(cache[0], cache[1]) and torch.equal(q_out, alone)


@pytest.mark.parametrize("pages", [700, 9000])
def test_a_captured_fork_and_compaction_replay_on_changed_tables(T, pages):
    import torch
    n, width = 24, 6
    pool, host = _pool(pages, 3)
    case = _fork_case(n, n, pages, width, 0)
    f = _Fork(T, case, pool)
    table, lens, parents, refs = f.a.kept[1:5]
    out, refs_out, live, err = torch.zeros_like(f.out), torch.zeros_like(f.refs), _i32([0]), _i32([0])
    a = T.compact_args(pool, f.out, f.refs, out, refs_out, live, err=err)
    scratch = torch.empty(T.tlf_cache_compact_scratch_bytes(a), dtype=torch.uint8, device="cuda")

    def step():
        s = torch.cuda.current_stream()
        f.stream = s
        f()
        T.tlf_cache_compact(a, scratch, scratch.numel(), s)

    step()  # (loads the kernels)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in range(1, 6):
        case = _fork_case(n, n, pages, width, seed)
        case[3][:] = 0  # the tables of the call are all there are
        for p in case[0][case[0] >= 0]:
            case[3][p] += 1
        fresh, host = _pool(pages, seed)
        pool.copy_(fresh)
        for t, x in zip((table, lens, parents, refs), case):
            t.copy_(_i32(x))
        f.err.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = W.fork(host, *case, 70)
        f.hold(want)
        moved = W.compact(want[0], want[1], want[3])
        assert int(err.item()) == 0 and int(live.item()) == moved[3] and np.array_equal(out.cpu().numpy(), moved[1])
        assert np.array_equal(refs_out.cpu().numpy(), moved[2]) and np.array_equal(pool.cpu().numpy(), moved[0])
