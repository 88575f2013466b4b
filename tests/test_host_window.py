"""CPU tests of the 4-bit cache, the windowed attention and the page operators: refused arguments, struct layouts, the split."""
import ctypes as C
import shutil
import subprocess

import pytest

from paper_2609_15160_gb300 import build, tlf

SPLIT = r"""
#define __host__
#define __device__
#include "k_chunk.cuh"
#include <stdio.h>
#include <stdlib.h>
int main() {
  for (int it = 0; it < 12000; ++it) {
    tlf::WindowSplit s;
    s.qt_log = rand() % 9, s.bk_log = 6, s.pad = it % 3 ? rand() % 12 : 0;
    s.window = it % 7 == 0 ? 0x7fffffff : 1 + rand() % (it % 2 ? 40 : 3000), s.first = it % 2 ? 0 : rand() % 300;
    const int ql = rand() % 700, any = it % 5 ? rand() % 1500 - 700 : rand() % 100000, s0 = any < -ql ? -ql : any, nt = s.tiles(ql);
    long long sum = 0;
    for (int t = 0; t <= nt; ++t) {
      if (s.before(s0, ql, t) != sum) return 1;
      if (t == nt) break;
      // blocks that the tile's first query's window, its last query and the first entries leave, counted one by one
      const int q0 = t << s.qt_log, q1 = (q0 + (1 << s.qt_log) < ql ? q0 + (1 << s.qt_log) : ql) - 1;
      int n = 0, skipped = 0;
      for (long long k = 0; k == 0 || k * 64 <= s0 + q1; ++k) {
        const bool sink = k * 64 < s.first, win = k * 64 + 63 > (long long)s0 + q0 - s.window;
        n += sink || win;
        skipped += !(sink || win);
      }
      if (s0 + q1 < 0) n = 1, skipped = 0;
      if (s.blocks(s0, ql, t) != n || s.skip(s0, t) != skipped) return 2;
      if (s.tile_of(s0, ql, sum) != t || s.tile_of(s0, ql, sum + s.pad + n - 1) != t) return 3;
      sum += s.pad + n;
    }
  }
  // far entries: nothing passes 32 bits on the way
  tlf::WindowSplit s;
  s.qt_log = 7, s.bk_log = 6, s.pad = 4, s.window = 1000, s.first = 0x7fffffff;
  if (s.blocks(2000000000, 100, 0) != (2000000000 + 100 + 63) / 64 || s.skip(2000000000, 0) != 0) return 4;
  s.first = 0;
  if (s.blocks(2000000000, 100, 0) > 19) return 5;
  printf("ok\n");
  return 0;
}
"""


def _run(tmp_path, name, text):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    src, exe = tmp_path / name, tmp_path / "a.out"
    src.write_text(text)
    subprocess.run(["g++", "-x", "c++", "-std=c++17", "-O1", "-I", build.INCLUDE, "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.returncode
    return r.stdout


def test_the_windowed_work_split_counts_every_block_once(tmp_path):
    """The closed forms under a window against counting blocks one by one."""
    assert _run(tmp_path, "split.cpp", SPLIT) == "ok\n"


P = 1 << 20  # a made-up device address, aligned; nothing is launched by a refused call


@pytest.fixture(scope="module")
def lib():
    build.build()
    return tlf.load_library()


def _chunk(**kw):
    c = dict(n=2, n_tokens=5, max_chunk=4, n_heads=4, n_kv_heads=2, head_dim=64, n_layers=2, layer=1, page_size=64, dtype=1,
             max_pages=10, n_pages=20, pool=P, page_table=P, cu_tokens=P, lens=P)
    c.update(kw)
    return tlf.TlfChunk(**c)


def _refused(rc, what):
    assert rc == tlf.CODES["INVALID_ARG"]
    assert what in tlf.load_library().tlf_last_error(None).decode()


ROPE = dict(q=P, k=P, v=P, q_stride=512, k_stride=512, v_stride=512, positions=P, table=P, max_pos=9, rot_dim=64, q_out=P)


@pytest.mark.parametrize("kw,what", [(dict(n=0), "n must"), (dict(n_heads=3), "divide"), (dict(head_dim=16), "head_dim"), (dict(head_dim=48), "head_dim"),
                                     (dict(layer=2), "layer"), (dict(page_size=32), "page_size"), (dict(dtype=2), "dtype"), (dict(pool=P + 8), "aligned"),
                                     (dict(pool=None), "NULL"), (dict(cu_tokens=None), "NULL"), (dict(reserved0=1), "reserved0")], ids=str)
def test_a_bad_batch_is_refused(lib, kw, what):
    c = _chunk(**kw)
    a = tlf.TlfAttnWindowArgs(q=P, out=P, window=9)
    _refused(lib.tlf_kv4_append(C.byref(c), C.byref(tlf.TlfRopeArgs(**ROPE)), None), what)
    _refused(lib.tlf_kv4_read(C.byref(c), C.byref(tlf.TlfKv4ReadArgs(k=P)), None), what)
    assert lib.tlf_attn_window_scratch_bytes(C.byref(c), C.byref(a)) == 0
    _refused(lib.tlf_attn_window(C.byref(c), C.byref(a), P, 1 << 40, None), what)


@pytest.mark.parametrize("kw,what", [(dict(q=None), "NULL"), (dict(rot_dim=66), "rot_dim"), (dict(layout=2), "layout"), (dict(v_stride=127), "stride"),
                                     (dict(table=P + 4), "aligned"), (dict(q_f32=2), "q_f32")], ids=str)
def test_bad_arguments_of_an_append_are_refused(lib, kw, what):
    c = _chunk()
    _refused(lib.tlf_kv4_append(C.byref(c), C.byref(tlf.TlfRopeArgs(**dict(ROPE, **kw))), None), what)
    _refused(lib.tlf_kv4_append(C.byref(c), None, None), "NULL")
    _refused(lib.tlf_kv4_read(C.byref(c), C.byref(tlf.TlfKv4ReadArgs(k=P, k_stride=127)), None), "stride")
    _refused(lib.tlf_kv4_read(C.byref(c), None, None), "NULL")


@pytest.mark.parametrize("kw,what", [(dict(q=None), "NULL"), (dict(out=None), "NULL"), (dict(q_stride=255), "stride"), (dict(scale=float("nan")), "scale"),
                                     (dict(window=-1), "window"), (dict(n_first=-2), "n_first"), (dict(kv_format=2), "kv_format")], ids=str)
def test_bad_arguments_of_the_attention_are_refused(lib, kw, what):
    a = tlf.TlfAttnWindowArgs(**dict(dict(q=P, out=P, window=7, n_first=2), **kw))
    c = _chunk()
    assert lib.tlf_attn_window_scratch_bytes(C.byref(c), C.byref(a)) == 0
    _refused(lib.tlf_attn_window(C.byref(c), C.byref(a), P, 1 << 40, None), what)
    _refused(lib.tlf_attn_window(C.byref(c), None, P, 1 << 40, None), "NULL")


def _fork(**kw):
    a = dict(n_in=2, n_out=3, n_kv_heads=2, head_dim=64, n_layers=1, page_size=64, dtype=1, max_pages=4, reserve=1, n_pages=9, pool=P,
             page_table=P, lens=P, parents=P, refs=P, table_out=2 * P, lens_out=P, refs_out=P)
    a.update(kw)
    return tlf.TlfForkArgs(**a)


@pytest.mark.parametrize("kw,what", [
    (dict(n_in=0), "n_in"), (dict(n_out=65536), "n_out"), (dict(head_dim=20), "head_dim"), (dict(head_dim=16), "head_dim"), (dict(page_size=16), "page_size"),
    (dict(kv_format=3), "kv_format"), (dict(max_pages=0), "max_pages"), (dict(reserve=-1), "reserve"), (dict(window=-1), "window"), (dict(n_first=-1), "n_first"),
    (dict(n_pages=0), "n_pages"), (dict(pool=P + 4), "aligned"), (dict(lens=None), "NULL"), (dict(parents=None), "NULL"), (dict(refs=None), "NULL"),
    (dict(table_out=None), "NULL"), (dict(refs_out=None), "NULL"), (dict(lens_out=None), "NULL"), (dict(table_out=P), "overlap"),
    (dict(table_out=P + 28), "overlap"), (dict(table_out=P - 44), "overlap"), (dict(n_out=65535, max_pages=1 << 24, reserve=1 << 30, table_out=P << 40), "reserve")], ids=str)
def test_bad_arguments_of_a_fork_are_refused(lib, kw, what):
    a = _fork(**kw)
    assert lib.tlf_cache_fork_scratch_bytes(C.byref(a)) == 0
    _refused(lib.tlf_cache_fork(C.byref(a), P, 1 << 40, None), what)


@pytest.mark.parametrize("kw,what", [
    (dict(n=0), "n must"), (dict(head_dim=20), "head_dim"), (dict(kv_format=-1), "kv_format"), (dict(n_live=None), "NULL"), (dict(refs_out=None), "NULL"),
    (dict(table_out=None), "NULL"), (dict(n_pages=1 << 31), "n_pages")], ids=str)
def test_bad_arguments_of_a_compaction_are_refused(lib, kw, what):
    a = dict(n=2, n_kv_heads=2, head_dim=64, n_layers=1, page_size=64, dtype=1, max_pages=4, n_pages=9, pool=P, page_table=P, refs=P, table_out=P,
             refs_out=P, n_live=P)
    a.update(kw)
    a = tlf.TlfCompactArgs(**a)
    assert lib.tlf_cache_compact_scratch_bytes(C.byref(a)) == 0
    _refused(lib.tlf_cache_compact(C.byref(a), P, 1 << 40, None), what)


def test_short_scratch_is_refused(lib):
    a = _fork()
    n = lib.tlf_cache_fork_scratch_bytes(C.byref(a))
    b = tlf.TlfCompactArgs(n=2, n_kv_heads=2, head_dim=64, n_layers=1, page_size=64, dtype=1, max_pages=4, n_pages=9, pool=P, page_table=P, refs=P,
                           table_out=P, refs_out=P, n_live=P)
    m = lib.tlf_cache_compact_scratch_bytes(C.byref(b))
    assert n > 0 and m > 0
    for at, size in ((P, n - 1), (None, n), (P + 4, n)):
        _refused(lib.tlf_cache_fork(C.byref(a), at, size, None), "scratch")
    for at, size in ((P, m - 1), (None, m), (P + 4, m)):
        _refused(lib.tlf_cache_compact(C.byref(b), at, size, None), "scratch")


def test_block_bytes(lib):
    for hd, size in ((16, 768), (32, 1280), (64, 2304), (128, 4608)):
        assert lib.tlf_kv4_block_bytes(hd) == tlf.kv4_block_bytes(hd) == size
    assert lib.tlf_kv4_block_bytes(48) == 0 and lib.tlf_kv4_block_bytes(-1) == 0
    with pytest.raises(ValueError):
        tlf.kv4_block_bytes(48)


def test_builders_refuse_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    pool4 = torch.zeros(9, 2, 2, 2, 2304, dtype=torch.uint8)
    pool = torch.zeros(9, 2, 2, 2, 64, 64, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    c4 = tlf.chunk4_args(pool4, i32(3, 4), i32(4), i32(3), 4, 7, 64)
    assert (c4.n, c4.n_kv_heads, c4.head_dim, c4.n_layers, c4.page_size, c4.dtype, c4.n_pages) == (3, 2, 64, 2, 64, 1, 9)
    c = tlf.chunk_args(pool, i32(3, 4), i32(4), i32(3), 4, 7)
    for bad in (pool4[..., :2303], pool4.float(), pool4[:, :, :1], pool):
        with pytest.raises(ValueError):
            tlf.chunk4_args(bad, i32(3, 4), i32(4), i32(3), 4, 7, 64)
    q = torch.zeros(7, 4, 64, dtype=torch.bfloat16)
    for batch, kv4 in ((c, True), (c4, False)):  # a call for one format on a cache in the other
        with pytest.raises(ValueError):
            tlf.tlf_attn_window(batch, tlf.attn_window_args(q, q, kv4=kv4), None, 0)
    with pytest.raises(ValueError):
        tlf.tlf_attn_chunk(c4, tlf.attn_chunk_args(q, q), None, 0)
    with pytest.raises(ValueError):
        tlf.tlf_attn_window(c4, tlf.attn_window_args(q[:6], q[:6], kv4=True), None, 0)
    with pytest.raises(ValueError):
        tlf.tlf_kv4_read(c, tlf.kv4_read_args(q[:, :2].contiguous()), None)
    with pytest.raises(ValueError):
        tlf.tlf_kv4_read(c4, tlf.kv4_read_args(q), None)  # four kv heads
    with pytest.raises(ValueError):
        tlf.kv4_read_args()
    with pytest.raises(ValueError):
        tlf.fork_args(pool, i32(3, 4), i32(3), i32(5), i32(8), i32(5, 4), i32(5), i32(9))  # refs of eight pages
    with pytest.raises(ValueError):
        tlf.fork_args(pool, i32(3, 4), i32(3), i32(5), i32(9), i32(5, 3), i32(5), i32(9))
    with pytest.raises(ValueError):
        tlf.fork_args(pool4, i32(3, 4), i32(3), i32(5), i32(9), i32(5, 4), i32(5), i32(9))  # 4 bits want head_dim
    with pytest.raises(ValueError):
        tlf.compact_args(pool, i32(3, 4), i32(9), i32(3, 4), i32(9), i32(2))


SIZES = r"""
#include <stddef.h>
#include <stdio.h>
#include "tlf.h"
int main(void) {
  printf("%zu %zu %zu %zu\n", sizeof(tlf_kv4_read_args), sizeof(tlf_attn_window_args), sizeof(tlf_fork_args), sizeof(tlf_compact_args));
  printf("%zu %zu %zu %zu\n", offsetof(tlf_kv4_read_args, v_stride), offsetof(tlf_attn_window_args, kv_format), offsetof(tlf_fork_args, err),
         offsetof(tlf_compact_args, err));
  return 0;
}
"""


def test_struct_layouts_match_the_header(tmp_path):
    a, b = (list(map(int, line.split())) for line in _run(tmp_path, "sizes.cpp", SIZES).splitlines())
    types = (tlf.TlfKv4ReadArgs, tlf.TlfAttnWindowArgs, tlf.TlfForkArgs, tlf.TlfCompactArgs)
    assert a == [C.sizeof(t) for t in types]
    assert b == [getattr(t, f).offset for t, f in zip(types, ("v_stride", "kv_format", "err", "err"))]


def test_every_entry_of_the_header_is_bound(lib):
    import os
    import re
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(build.INCLUDE, "tlf.h")).read(), flags=re.S)
    for name in set(re.findall(r"\b(tlf_[a-z0-9_]+)\s*\(", text)):
        assert hasattr(lib, name) and name in tlf._SIGS, name
