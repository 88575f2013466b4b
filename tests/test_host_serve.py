"""CPU tests of the operators on a caller's paged caches and logits: refused arguments, struct layouts, the work split."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2609_15160_gb300 import build, tlf

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


BAD_CHUNK = [(dict(n=0), "n must"), (dict(n=1025), "n must"), (dict(n_tokens=-1), "n_tokens"), (dict(max_chunk=-1), "max_chunk"),
             (dict(n_heads=3), "divide"), (dict(n_heads=0), "divide"), (dict(n_heads=130), "64 query heads"),
             (dict(n_kv_heads=0), "n_kv_heads"), (dict(head_dim=16), "head_dim"), (dict(head_dim=48), "head_dim"),
             (dict(n_layers=0), "n_layers"), (dict(layer=2), "layer"), (dict(layer=-1), "layer"), (dict(page_size=32), "page_size"),
             (dict(dtype=2), "dtype"), (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 26), "max_pages"),
             (dict(n_pages=0), "n_pages"), (dict(n_pages=1 << 31), "n_pages"), (dict(pool=P + 8), "aligned"), (dict(pool=None), "NULL"),
             (dict(page_table=None), "NULL"), (dict(cu_tokens=None), "NULL"), (dict(lens=None), "NULL"), (dict(reserved0=1), "reserved0"),
             (dict(n_layers=1 << 25), "too large")]


@pytest.mark.parametrize("kw,what", BAD_CHUNK, ids=lambda v: str(v))
def test_a_bad_batch_is_refused(lib, kw, what):
    c = _chunk(**kw)
    r = tlf.TlfRopeArgs(q=P, k=P, v=P, q_stride=512, k_stride=512, v_stride=512, positions=P, table=P, max_pos=9, rot_dim=64, q_out=P)
    a = tlf.TlfAttnChunkArgs(q=P, out=P)
    _refused(lib.tlf_rope_append(C.byref(c), C.byref(r), None), what)
    assert lib.tlf_attn_chunk_scratch_bytes(C.byref(c), C.byref(a)) == 0
    _refused(lib.tlf_attn_chunk(C.byref(c), C.byref(a), P, 1 << 40, None), what)


@pytest.mark.parametrize("kw,what", [
    (dict(q=None), "NULL"), (dict(v=None), "NULL"), (dict(table=None), "NULL"), (dict(table=P + 4), "aligned"), (dict(q_out=None), "NULL"),
    (dict(positions=None), "NULL"), (dict(rot_dim=66), "rot_dim"), (dict(rot_dim=7), "rot_dim"), (dict(rot_dim=0), "rot_dim"),
    (dict(max_pos=0), "max_pos"), (dict(layout=2), "layout"), (dict(q_f32=2), "q_f32"), (dict(q_stride=255), "stride"),
    (dict(v_stride=127), "stride")], ids=str)
def test_bad_rotary_arguments_are_refused(lib, kw, what):
    r = dict(q=P, k=P, v=P, q_stride=256, k_stride=128, v_stride=128, positions=P, table=P, max_pos=9, rot_dim=64, q_out=P)
    r.update(kw)
    c = _chunk()
    _refused(lib.tlf_rope_append(C.byref(c), C.byref(tlf.TlfRopeArgs(**r)), None), what)
    _refused(lib.tlf_rope_append(C.byref(c), None, None), "NULL")
    _refused(lib.tlf_rope_append(None, C.byref(tlf.TlfRopeArgs(**r)), None), "NULL")


@pytest.mark.parametrize("kw,what", [
    (dict(rot_dim=3), "rot_dim"), (dict(rot_dim=258), "rot_dim"), (dict(base=1.0), "base"), (dict(base=float("nan")), "base"),
    (dict(scaling="linear", factor=0.5), "factor"), (dict(scaling="ntk", rot_dim=2, factor=2.0), "NTK"),
    (dict(scaling="ramp", factor=2.0), "RAMP"), (dict(scaling="ramp", factor=2.0, original_len=100, high_turns=1.0), "RAMP"),
    (dict(magnitude=float("inf")), "magnitude")], ids=str)
def test_bad_rotary_tables_are_refused(lib, kw, what):
    cfg = tlf.rope_config(**dict(dict(rot_dim=64), **kw))
    _refused(lib.tlf_rope_table(C.byref(cfg), 10, P, None), what)
    good = tlf.rope_config(64)
    _refused(lib.tlf_rope_table(C.byref(good), 0, P, None), "max_pos")
    _refused(lib.tlf_rope_table(C.byref(good), 10, None, None), "table")
    _refused(lib.tlf_rope_table(None, 10, P, None), "NULL")


@pytest.mark.parametrize("kw,what", [
    (dict(q=None), "NULL"), (dict(out=None), "NULL"), (dict(q_stride=255), "stride"), (dict(out_stride=-1), "stride"),
    (dict(weight_in=P), "weight_in"), (dict(scale=float("nan")), "scale"), (dict(reserved0=3), "reserved0")], ids=str)
def test_bad_attention_arguments_are_refused(lib, kw, what):
    a = tlf.TlfAttnChunkArgs(**dict(dict(q=P, out=P), **kw))
    c = _chunk()
    assert lib.tlf_attn_chunk_scratch_bytes(C.byref(c), C.byref(a)) == 0
    _refused(lib.tlf_attn_chunk(C.byref(c), C.byref(a), P, 1 << 40, None), what)


def _evict(**kw):
    a = dict(n=2, n_kv_heads=2, head_dim=64, n_layers=1, page_size=64, dtype=1, max_pages=4, budget=100, n_first=4, n_recent=10,
             n_pages=9, pool=P, page_table=P, lens=P, next_pos=P, pos_in=P, pos_out=P, weight_in=P, weight_out=P, lens_out=P)
    a.update(kw)
    return tlf.TlfEvictArgs(**a)


@pytest.mark.parametrize("kw,what", [
    (dict(n=0), "n must"), (dict(budget=0), "budget"), (dict(n_first=95), "budget"), (dict(n_recent=-1), "budget"),
    (dict(head_dim=20), "head_dim"), (dict(page_size=128), "page_size"), (dict(lens_out=None), "NULL"), (dict(pos_in=None), "NULL"),
    (dict(weight_out=None), "NULL"), (dict(next_pos=None), "NULL"), (dict(pool=P + 2), "aligned")], ids=str)
def test_bad_eviction_arguments_are_refused(lib, kw, what):
    a = _evict(**kw)
    assert lib.tlf_cache_evict_scratch_bytes(C.byref(a)) == 0
    _refused(lib.tlf_cache_evict(C.byref(a), P, 1 << 40, None), what)


def test_short_scratch_is_refused(lib):
    a = _evict()
    n = lib.tlf_cache_evict_scratch_bytes(C.byref(a))
    assert n > 0
    _refused(lib.tlf_cache_evict(C.byref(a), P, n - 1, None), "scratch")
    _refused(lib.tlf_cache_evict(C.byref(a), None, n, None), "scratch")
    _refused(lib.tlf_cache_evict(C.byref(a), P + 4, n, None), "scratch")


@pytest.mark.parametrize("kw,what", [
    (dict(n=0), "n must"), (dict(n=65536), "n must"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 22) + 1), "vocab"),
    (dict(logits=None), "NULL"), (dict(noise=None), "NULL"), (dict(tokens=None), "NULL"), (dict(logits_stride=99), "stride"),
    (dict(noise_stride=0), "stride")], ids=str)
def test_bad_sampling_arguments_are_refused(lib, kw, what):
    a = dict(n=3, vocab=100, logits=P, logits_stride=100, noise=P, noise_stride=100, tokens=P)
    a.update(kw)
    _refused(lib.tlf_sample(C.byref(tlf.TlfSampleArgs(**a)), None), what)
    _refused(lib.tlf_sample(None, None), "NULL")


def test_builders_refuse_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    pool = torch.zeros(9, 2, 2, 2, 64, 64, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    c = tlf.chunk_args(pool, i32(3, 4), i32(4), i32(3), 4, 7)
    assert (c.n, c.n_kv_heads, c.head_dim, c.n_layers, c.page_size, c.dtype, c.n_pages) == (3, 2, 64, 2, 64, 1, 9)
    for bad in (dict(pool=pool[:, :, :1]), dict(pool=pool.transpose(3, 4)), dict(cu=i32(3)), dict(lens=i32(3).long()), dict(table=i32(4, 3).T)):
        with pytest.raises(ValueError):
            tlf.chunk_args(bad.get("pool", pool), bad.get("table", i32(3, 4)), bad.get("cu", i32(4)), bad.get("lens", i32(3)), 4, 7)
    q = torch.zeros(7, 4, 64, dtype=torch.bfloat16)
    for bad in (dict(out=q.float()), dict(q=q.transpose(1, 2)), dict(lse=torch.zeros(7, 3)), dict(weight_out=torch.zeros(9, 32))):
        with pytest.raises(ValueError):
            tlf.attn_chunk_args(**dict(dict(q=q, out=q), **bad))
    for q_bad in (q[:6], torch.zeros(7, 8, 64, dtype=torch.bfloat16), q.float()):
        with pytest.raises(ValueError):  # fewer tokens, other heads or another type than the batch's
            tlf.tlf_attn_chunk(c, tlf.attn_chunk_args(q_bad, q_bad), None, 0)
    with pytest.raises(ValueError):
        tlf.tlf_attn_chunk(c, tlf.attn_chunk_args(q, q, weight_out=torch.zeros(8, 64)), None, 0)
    with pytest.raises(ValueError):
        tlf.sample_args(torch.zeros(2, 9).T, torch.zeros(9, 2), i32(9))
    with pytest.raises(ValueError):
        tlf.sample_args(torch.zeros(9, 2), torch.zeros(9, 2), i32(9), top_k=torch.zeros(9))


SIZES = r"""
#include <stddef.h>
#include <stdio.h>
#include "tlf.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu\n", sizeof(tlf_chunk), sizeof(tlf_rope_config), sizeof(tlf_rope_args), sizeof(tlf_attn_chunk_args),
         sizeof(tlf_evict_args), sizeof(tlf_sample_args));
  printf("%zu %zu %zu %zu %zu %zu\n", offsetof(tlf_chunk, err), offsetof(tlf_rope_config, magnitude), offsetof(tlf_rope_args, entry_weight),
         offsetof(tlf_attn_chunk_args, scale), offsetof(tlf_evict_args, lens_out), offsetof(tlf_sample_args, logprobs));
  return 0;
}
"""

SPLIT = r"""
#define __host__
#define __device__
#include "k_chunk.cuh"
#include <stdio.h>
#include <stdlib.h>
int main() {
  for (int bl = 6; bl <= 7; ++bl)
    for (int it = 0; it < 6000; ++it) {
      const tlf::ChunkSplit s{rand() % 9, bl, it % 3 ? rand() % 12 : 0};
      const int ql = rand() % 700, any = it % 5 ? rand() % 1500 - 700 : rand() % 100000, s0 = any < -ql ? -ql : any, nt = s.tiles(ql);
      long long sum = 0;
      if (nt != (ql + (1 << s.qt_log) - 1) / (1 << s.qt_log)) return 1;
      for (int t = 0; t <= nt; ++t) {
        if (s.before(s0, ql, t) != sum) return 2;
        if (t == nt) break;
        const int end = (t + 1) << s.qt_log, keys = s0 + (end < ql ? end : ql), want = keys <= 0 ? 1 : (keys + (1 << bl) - 1) / (1 << bl);
        if (s.blocks(s0, ql, t) != want) return 3;
        if (s.tile_of(s0, ql, sum) != t || s.tile_of(s0, ql, sum + s.pad + want - 1) != t) return 4;
        sum += s.pad + want;
      }
    }
  for (int it = 0; it < 6000; ++it) {
    const tlf::WeighSplit s{1 + rand() % 7, 8};
    const int ql = rand() % 700, any = it % 5 ? rand() % 1500 - 700 : rand() % 100000, s0 = any < -ql ? -ql : any, nb = s.blocks(s0, ql);
    const int nt = (ql + (1 << s.qt_log) - 1) >> s.qt_log, heads = 1 + rand() % 8;
    if (nb != (ql > 0 ? (s0 + ql + 255) / 256 : 0)) return 5;
    long long sum = 0;
    for (int kb = 0; kb <= nb; ++kb) {
      if (s.before(s0, ql, kb) != sum) return 6;
      if (kb == nb) break;
      int first = 0;  // the first tile whose last query (whole tiles) sees entry 256 kb
      while (s0 + ((first + 1) << s.qt_log) - 1 < 256 * kb) ++first;
      if (s.first(s0, kb) != first || first >= nt) return 7;
      if (s.block_of(s0, ql, heads, sum * heads) != kb || s.block_of(s0, ql, heads, (sum + nt - first) * heads - 1) != kb) return 8;
      sum += nt - first;
    }
  }
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


def test_struct_layouts_match_the_header(tmp_path):
    a, b = (list(map(int, line.split())) for line in _run(tmp_path, "sizes.cpp", SIZES).splitlines())
    types = (tlf.TlfChunk, tlf.TlfRopeConfig, tlf.TlfRopeArgs, tlf.TlfAttnChunkArgs, tlf.TlfEvictArgs, tlf.TlfSampleArgs)
    assert a == [C.sizeof(t) for t in types]
    assert b == [getattr(t, f).offset for t, f in zip(types, ("err", "magnitude", "entry_weight", "scale", "lens_out", "logprobs"))]


def test_the_work_split_counts_every_block_once(tmp_path):
    """The closed forms of the split against counting, with fewer entries than new tokens among the rows."""
    assert _run(tmp_path, "split.cpp", SPLIT) == "ok\n"
    assert os.path.exists(os.path.join(build.CSRC, "k_chunk.cuh"))
