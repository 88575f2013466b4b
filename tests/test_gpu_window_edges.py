"""Where the 4-bit cache, windowed attention and the page operators could go wrong for one row because of another, at the ends of
their types, and in calls that overlap. Bounds as in test_gpu_window_ops."""
import numpy as np
import pytest

import _serve_ref as R
import _window_ref as W
from test_gpu_window_ops import T, _attend, _batch, _cache, _hold  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["plain", "4bit"])
@pytest.mark.parametrize("new,hd", [(3, 64), (3, 128), (20, 128), (70, 64), (70, 128)])
def test_rows_without_a_number_leave_the_others_alone(T, kind, new, hd):
    """Queries of some tokens are NaN, of others infinite: every other token is right."""
    rng = np.random.default_rng(new)
    c = _cache(kind, rng.integers(0, 200, 12), [new] * 12, 4, 2, hd, "bf16", seed=new)
    ref = W.attention(c, 90, 3)
    bad = np.concatenate([np.arange(c.cu[b], c.cu[b] + max(1, new // 2)) for b in (1, 4, 11)])
    c.q[bad] = np.where(np.arange(len(bad))[:, None, None] % 2, np.inf, np.nan)
    d = c.device()
    got = _attend(T, c, d, 90, 3)
    rest = np.setdiff1d(np.arange(c.T), bad)
    _hold(c, d, got, ref, tokens=rest)
    o = got[0].float().cpu().numpy()[bad]
    assert not np.isfinite(o[::2]).any()


@pytest.mark.parametrize("kind", ["plain", "4bit"])
@pytest.mark.parametrize("new,max_chunk", [(1, 1), (5, 5), (9, 40)])
@pytest.mark.parametrize("hd", [64, 128])
def test_1024_rows(T, kind, new, max_chunk, hd):
    rng = np.random.default_rng(5)
    n = rng.integers(0, new + 1, 1024)
    c = _cache(kind, rng.integers(0, 80, 1024), n, 2, 1, hd, "bf16", layers=1, layer=0, seed=7)
    d = c.device()
    _hold(c, d, _attend(T, c, d, 50, 2, max_chunk=max_chunk), W.attention(c, 50, 2))


@pytest.mark.parametrize("new", [[2, 3], [60, 90]], ids=["few", "many"])
@pytest.mark.parametrize("scale", [1e-38, 1e-4, 3.0, 1e4])
@pytest.mark.parametrize("hd", [64, 128])
def test_scales_and_zero_queries_of_a_4bit_cache(T, new, scale, hd):
    """From scores that are all alike to one that takes everything; some queries are zero, so that all entries weigh the same."""
    c = W.Cache4([100, 300], new, 4, 2, hd, "bf16", seed=hd)
    c.q[::3] = 0
    c.q[1::3] *= 2.0 ** -30
    d = c.device()
    for window, first in ((0, 0), (64, 5)):
        ref = W.attention(c, window, first, scale)
        _hold(c, d, _attend(T, c, d, window, first, scale), ref)


@pytest.mark.parametrize("new", [[2, 3], [60, 90]], ids=["few", "many"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("size", [0.0, 2.0 ** -12, 2.0 ** 9])
def test_a_first_entry_that_takes_nearly_everything(T, new, hd, size):
    """A sink: its key takes all but 2^-9 .. 2^-14 of the probability, its value is nothing, tiny or large beside the others'."""
    c = W.Cache4([150, 400], new, 4, 2, hd, "bf16", seed=3)
    for b in range(c.n):
        p, o = c.at(b, np.array([0]))
        c.pool[p, c.layer, 0, :, o] = 1.5
        c.pool[p, c.layer, 1, :, o] *= size
    c.pool4 = W.blocks(*W.quantise(c.round(c.pool)))
    c.q = R.bf16(np.abs(c.q) * (64 / hd))
    d = c.device()
    for window, first in ((0, 0), (100, 1)):
        _hold(c, d, _attend(T, c, d, window, first), W.attention(c, window, first))


@pytest.mark.parametrize("kind", ["plain", "4bit"])
@pytest.mark.parametrize("new", [1, 4, 70])
def test_rows_behind_the_last_token_and_past_max_chunk_stay_as_they_were(T, kind, new):
    import torch
    c = _cache(kind, [90, 40, 10], [new] * 3, 4, 2, 64, "bf16", seed=new)
    d = c.device()
    out = torch.full((c.T + 5, c.hq, c.hd), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.T + 5, c.hq), 7.0, device="cuda")
    q = torch.zeros(c.T + 5, c.hq, c.hd, dtype=torch.bfloat16, device="cuda")
    q[:c.T] = d["q"][:c.T]
    b = _batch(T, c, d)
    a = T.attn_window_args(q, out, lse=lse, window=30, n_first=1, kv4=kind == "4bit")
    n = T.tlf_attn_window_scratch_bytes(b, a)
    T.tlf_attn_window(b, a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    torch.cuda.synchronize()
    _hold(c, d, (out, lse), W.attention(c, 30, 1))
    assert (out[c.T:] == 7).all() and (lse[c.T:] == 7).all()
    if new > 1:  # rows of more tokens than max_chunk says are cut, and it is reported
        out[:], lse[:] = 7, 7
        b = _batch(T, c, d, max_chunk=new - 1)
        n = T.tlf_attn_window_scratch_bytes(b, a)
        T.tlf_attn_window(b, a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
        torch.cuda.synchronize()
        assert int(d["err"][0].item()) == 2
        last = torch.as_tensor(c.cu[1:] - 1, device="cuda").long()
        assert (out[last] == 7).all() and (lse[last] == 7).all()
        assert (lse[:c.T] == 7).sum() == 3 * c.hq


@pytest.mark.parametrize("kind", ["plain", "4bit"])
@pytest.mark.parametrize("hq,hd,dtype", [(4, 64, "bf16"), (64, 64, "bf16"), (64, 128, "bf16"), (4, 64, "f32")])
def test_a_batch_without_tokens_writes_nothing(T, kind, hq, hd, dtype):
    import torch
    c = _cache(kind, [70, 0, 300], [0, 0, 0], hq, 2, hd, dtype, seed=1)
    d = c.device()
    q = torch.ones(3, hq, hd, dtype=getattr(torch, {"bf16": "bfloat16", "f32": "float32"}[dtype]), device="cuda")
    out, lse = torch.full_like(q, 7), torch.full((3, hq), 7.0, device="cuda")
    b, a = _batch(T, c, d), T.attn_window_args(q, out, lse=lse, window=30, n_first=1, kv4=kind == "4bit")
    n = T.tlf_attn_window_scratch_bytes(b, a)
    T.tlf_attn_window(b, a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    torch.cuda.synchronize()
    assert (out == 7).all() and (lse == 7).all() and int(d["err"][0].item()) == 0


def test_calls_on_two_streams_at_once(T):
    """Attention of two batches, a fork and a compaction of two pools, each with its own scratch, at the same time."""
    import torch
    batches = [W.Cache4([3000, 10, 500], [1, 1, 1], 8, 4, 128, "bf16", seed=1), W.Cache4([200, 900], [120, 33], 4, 2, 64, "bf16", seed=2)]
    devs, calls = [c.device() for c in batches], []
    outs = [(torch.empty(c.T, c.hq, c.hd, dtype=torch.bfloat16, device="cuda"), torch.empty(c.T, c.hq, device="cuda")) for c in batches]
    streams = [torch.cuda.Stream() for _ in batches]
    for c, d, (o, l), s in zip(batches, devs, outs, streams):
        b, a = _batch(T, c, d), T.attn_window_args(d["q"], o, lse=l, window=800, n_first=4, kv4=True)
        scratch = torch.empty(T.tlf_attn_window_scratch_bytes(b, a), dtype=torch.uint8, device="cuda")
        calls.append(lambda b=b, a=a, x=scratch, s=s: T.tlf_attn_window(b, a, x, x.numel(), s))
    torch.cuda.synchronize()
    for _ in range(20):
        for call in calls:
            call()
    torch.cuda.synchronize()
    for c, d, o in zip(batches, devs, outs):
        _hold(c, d, o, W.attention(c, 800, 4))


def test_a_partly_filled_page_that_somebody_else_holds_is_copied_for_every_child(T):
    import torch
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pool = torch.arange(6 * 2 * 64 * 32, device="cuda", dtype=torch.float32).view(6, 1, 2, 1, 64, 32)
    before = pool.clone()
    table, lens, refs = i32([[4, 1, -1]]), i32([70]), i32([0, 2, 0, 0, 1, 0])  # page 1 has an owner outside of the call
    out, lens_out, refs_out, err = i32([[9] * 3] * 2), i32([0, 0]), i32([0] * 6), i32([0])
    a = T.fork_args(pool, table, lens, i32([0, 0]), refs, out, lens_out, refs_out, reserve=64, err=err)
    n = T.tlf_cache_fork_scratch_bytes(a)
    T.tlf_cache_fork(a, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    assert out.tolist() == [[4, 0, 2], [4, 3, 5]] and lens_out.tolist() == [70, 70]
    assert refs_out.tolist() == [1, 1, 1, 1, 2, 1] and int(err.item()) == 0
    for page in (0, 3):
        assert torch.equal(pool[page, ..., :6, :], before[1, ..., :6, :]) and torch.equal(pool[page, ..., 6:, :], before[page, ..., 6:, :])


def test_a_fork_of_large_pools_and_many_rows(T):
    """Plans by a cluster: more than 65536 pages, more than 4096 rows."""
    import torch
    rng = np.random.default_rng(0)
    for n_in, n_out, pages in ((50, 70, 150000), (5000, 6000, 40000)):
        width = 4
        lens = rng.integers(0, 200, n_in)
        table, ids, at, refs = np.full((n_in, width), -1, np.int32), rng.permutation(pages), 0, np.zeros(pages, np.int32)
        for b in range(n_in):
            k = -(-int(lens[b]) // 64)
            table[b, :k] = ids[at:at + k]
            at += k
        refs[ids[:at]] = 1
        refs[ids[at:at + pages // 3]] = 1  # of others
        parents = rng.integers(-1, n_in, n_out).astype(np.int32)
        pool = rng.integers(0, 1000, (pages, 1, 2, 1, 64, 16)).astype(np.float32) if pages < 100000 else np.zeros((pages, 1, 2, 1, 64, 16), np.float32)
        if pages >= 100000:
            pool[ids[:at]] = rng.standard_normal((at, 1, 2, 1, 64, 16))
        want = W.fork(pool, table, lens, parents, refs, 70)
        dev = [torch.tensor(x).cuda() for x in (pool, table, lens.astype(np.int32), parents, refs)]
        out = torch.zeros(n_out, width, dtype=torch.int32, device="cuda")
        lens_out, refs_out, err = torch.zeros(n_out, dtype=torch.int32, device="cuda"), torch.zeros_like(dev[4]), torch.zeros(1, dtype=torch.int32, device="cuda")
        a = T.fork_args(*dev, out, lens_out, refs_out, reserve=70, err=err)
        n = T.tlf_cache_fork_scratch_bytes(a)
        T.tlf_cache_fork(a, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n)
        assert int(err.item()) == want[4]
        assert np.array_equal(out.cpu().numpy(), want[1]) and np.array_equal(lens_out.cpu().numpy(), want[2])
        assert np.array_equal(refs_out.cpu().numpy(), want[3]) and np.array_equal(dev[0].cpu().numpy(), want[0])
        # and the compaction of what it leaves; pages of others have no table here: they get one each
        others = np.nonzero(want[3] > 0)[0].astype(np.int32)
        tab = others.reshape(-1, 1)[:65535]
        refs2 = np.zeros(pages, np.int32)
        refs2[tab[:, 0]] = 1
        cw = W.compact(want[0], tab, refs2)
        t2, r2 = torch.tensor(tab).cuda(), torch.tensor(refs2).cuda()
        t3, r3, live = torch.zeros_like(t2), torch.zeros_like(r2), torch.zeros(1, dtype=torch.int32, device="cuda")
        a = T.compact_args(dev[0], t2, r2, t3, r3, live)
        n = T.tlf_cache_compact_scratch_bytes(a)
        T.tlf_cache_compact(a, torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda"), n)
        assert int(live.item()) == cw[3] and np.array_equal(t3.cpu().numpy(), cw[1]) and np.array_equal(r3.cpu().numpy(), cw[2])
        assert np.array_equal(dev[0].cpu().numpy(), cw[0])


def test_a_captured_step_of_append_attention_and_fork(T):
    """Replayed on other inputs, tables and lengths in the same buffers."""
    import torch
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32)).cuda()  # noqa: E731
    hq, hkv, hd, rows, pages, width = 4, 2, 64, 3, 40, 5
    rng = np.random.default_rng(0)
    rope = torch.empty(600, hd // 2, 2, device="cuda")
    T.tlf_rope_table(T.rope_config(hd), 600, rope)
    pool = torch.zeros(pages, 1, 2, hkv, T.kv4_block_bytes(hd), dtype=torch.uint8, device="cuda")
    tables, refs, lens = [i32(np.full((rows, width), -1)) for _ in range(2)], [i32(np.zeros(pages)) for _ in range(2)], [i32([0] * rows) for _ in range(2)]
    x = torch.zeros(rows, (hq + 2 * hkv) * hd, dtype=torch.bfloat16, device="cuda")
    pos, parents, err = i32([0] * rows), i32([-1] * rows), i32([0])
    q_out, out = (torch.zeros(rows, hq, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros(rows, hq, device="cuda")
    fork = T.fork_args(pool, tables[0], lens[0], parents, refs[0], tables[1], lens[1], refs[1], reserve=1, head_dim=hd, err=err)
    f_scratch = torch.empty(T.tlf_cache_fork_scratch_bytes(fork), dtype=torch.uint8, device="cuda")
    now = i32([0] * rows)  # entries with the new tokens
    batch = T.chunk4_args(pool, tables[1], i32(np.arange(rows + 1)), now, hq, rows, hd, max_chunk=1, err=err)
    q, k, v = x.split([hq * hd, hkv * hd, hkv * hd], 1)
    app = T.rope_args(q, k, v, pos, rope, q_out)
    att = T.attn_window_args(q_out, out, lse=lse, window=70, n_first=2, kv4=True)
    a_scratch = torch.empty(T.tlf_attn_window_scratch_bytes(batch, att), dtype=torch.uint8, device="cuda")

    def step():
        s = torch.cuda.current_stream()
        T.tlf_cache_fork(fork, f_scratch, f_scratch.numel(), s)
        torch.add(lens[1], 1, out=now)
        pos.copy_(lens[1])
        T.tlf_kv4_append(batch, app, s)
        T.tlf_attn_window(batch, att, a_scratch, a_scratch.numel(), s)
        tables[0].copy_(tables[1])
        refs[0].copy_(refs[1])
        lens[0].copy_(now)

    step()  # (loads the kernels)
    for t in tables + refs + lens + [now]:
        t.fill_(-1 if t.dim() == 2 else 0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    seqs = [[] for _ in range(rows)]
    for i in range(150):
        par = [-1] * rows if i == 0 else [0, 1, 2] if i % 10 else list(rng.integers(0, rows, rows))
        x.copy_(torch.tensor(R.bf16(rng.standard_normal(x.shape))).bfloat16())
        parents.copy_(i32(par))
        g.replay()
        torch.cuda.synchronize()
        seqs = [list(seqs[p]) if p >= 0 else [] for p in par]
        from test_gpu_window_ops import _turned32
        at = np.array([len(s) for s in seqs])
        kk = R.bf16(_turned32(k.float().cpu().numpy().reshape(rows, hkv, hd), rope.cpu().numpy()[at], hd, "half"))
        held = [W.terms(*W.quantise(y)) for y in (kk, v.float().cpu().numpy().reshape(rows, hkv, hd))]
        for r in range(rows):
            seqs[r].append((held[0][0][r], held[0][1][r], held[1][0][r], held[1][1][r]))
        if i % 7 and i < 140:
            continue

        class Whole(W.Cache4):
            def __init__(self):
                self.T, self.hq, self.hkv, self.hd, self.n, self.dtype = rows, hq, hkv, hd, rows, "bf16"
                self.cu, self.new, self.lens = np.arange(rows + 1), np.ones(rows, int), np.array([len(s) for s in seqs])
                self.q = q_out.float().cpu().numpy()

            def two(self, r, kv):
                return tuple(np.array([e[2 * kv + j] for e in seqs[r]]).reshape(-1, hkv, hd) for j in range(2))
        _hold(Whole(), {"err": err}, (out, lse), W.attention(Whole(), 70, 2))
