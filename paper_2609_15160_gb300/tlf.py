"""ctypes binding of libtlf (include/tlf.h): argument marshalling only.

Module-level functions carry the C names (``tlf_create``, ``tlf_prefill``,
``tlf_decode_step``, ``tlf_release``, ...). ``Context`` wraps them for
numpy / torch callers. Every computation of the decode step runs in the CUDA
kernels of libtlf; when the library has not been built this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import numpy as np

from . import build as _build
from . import synth as _synth

TLF_OK = 0
ERRORS = {-1: "INVALID_ARG", -2: "UNKNOWN_SEQ", -3: "DUPLICATE_SEQ", -4: "OUT_OF_PAGES", -5: "SEQ_TOO_LONG",
          -6: "CUDA", -7: "BAD_WEIGHTS", -8: "DEVICE", -9: "NO_DEVICE", -10: "CAPACITY"}
CODES = {v: k for k, v in ERRORS.items()}
KERNEL_CLASSES = ("router", "plan", "attn_norm", "qkv_gemm", "rope_append", "attention", "o_gemm", "mlp_norm",
                  "gate_up_gemm", "swiglu", "down_gemm", "final_norm", "lm_head")
DTYPE = {"f32": 0, "bf16": 1}
EXIT = {"argmax": 0, "survival": 1}
GEMM = {"auto": 0, "simt": 1}
ABLATION = {"none": 0, "no_gather": 1, "dense_cache": 2}
ROPE_SCALING = {"none": 0, "linear": 1, "ntk": 2, "ramp": 3}
ROPE_LAYOUT = {"half": 0, "interleaved": 1}
KV_FORMAT = {"plain": 0, "4bit": 1}


class TlfConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("vocab", "d_model", "n_heads", "n_kv_heads", "head_dim", "n_layers",
                                         "ffn_hidden", "max_loops")] + [
        ("rope_base", C.c_float), ("norm_eps", C.c_float), ("dtype", C.c_int32), ("exit_rule", C.c_int32),
        ("threshold", C.c_float), ("max_seqs", C.c_int32), ("max_batch", C.c_int32), ("max_seq_len", C.c_int32),
        ("page_size", C.c_int32), ("gemm_impl", C.c_int32), ("host_only", C.c_int32), ("prefill_chunk", C.c_int32),
        ("kv_pool_pages", C.c_int64), ("ablation", C.c_int32), ("conditioning", C.c_int32),
        ("router_hidden", C.c_int32), ("reserved", C.c_int32)]


COND_WEIGHTS = ("cond_t_w1", "cond_t_b1", "cond_t_w2", "cond_t_b2", "cond_dt_w1", "cond_dt_b1", "cond_dt_w2",
                "cond_dt_b2", "mod_w", "mod_b")


class TlfWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("embedding", "router_w", "router_b", "wq", "wk", "wv", "wo", "w_gate",
                                          "w_up", "w_down", "attn_norm", "mlp_norm", "final_norm") + COND_WEIGHTS
                + ("router_w1", "router_b1")]


class TlfAttnArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n", "n_heads", "n_kv_heads", "head_dim", "n_layers", "layer",
                                         "page_size", "dtype", "max_pages", "reserved0")] + [
        ("n_pages", C.c_int64)] + [(n, C.c_void_p) for n in ("q", "pool", "page_table", "lens", "out", "err")]


class TlfChunk(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n", "n_tokens", "max_chunk", "n_heads", "n_kv_heads", "head_dim", "n_layers",
                                         "layer", "page_size", "dtype", "max_pages", "reserved0")] + [
        ("n_pages", C.c_int64)] + [(n, C.c_void_p) for n in ("pool", "page_table", "cu_tokens", "lens", "err")]


class TlfRopeConfig(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("scaling", C.c_int32)] + [
        (n, C.c_double) for n in ("base", "factor", "original_len", "low_turns", "high_turns", "magnitude")]


class TlfRopeArgs(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "k", "v")] + [
        (n, C.c_int64) for n in ("q_stride", "k_stride", "v_stride")] + [("positions", C.c_void_p), ("table", C.c_void_p)] + [
        (n, C.c_int32) for n in ("max_pos", "rot_dim", "layout", "q_f32")] + [
        (n, C.c_void_p) for n in ("q_out", "entry_pos", "entry_weight")]


class TlfAttnChunkArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_stride", C.c_int64), ("out", C.c_void_p), ("out_stride", C.c_int64)] + [
        (n, C.c_void_p) for n in ("lse", "weight_in", "weight_out")] + [("scale", C.c_float), ("reserved0", C.c_int32)]


class TlfEvictArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n", "n_kv_heads", "head_dim", "n_layers", "page_size", "dtype", "max_pages",
                                         "budget", "n_first", "n_recent")] + [("n_pages", C.c_int64)] + [
        (n, C.c_void_p) for n in ("pool", "page_table", "lens", "next_pos", "pos_in", "pos_out", "weight_in", "weight_out",
                                  "lens_out", "err")]


class TlfSampleArgs(C.Structure):
    _fields_ = [("n", C.c_int32), ("vocab", C.c_int32), ("logits", C.c_void_p), ("logits_stride", C.c_int64),
                ("noise", C.c_void_p), ("noise_stride", C.c_int64)] + [
        (n, C.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p", "tokens", "logprobs")]


class TlfKv4ReadArgs(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_stride", C.c_int64), ("v_stride", C.c_int64)]


class TlfAttnWindowArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("q_stride", C.c_int64), ("out", C.c_void_p), ("out_stride", C.c_int64), ("lse", C.c_void_p),
                ("scale", C.c_float)] + [(n, C.c_int32) for n in ("window", "n_first", "kv_format")]


class TlfForkArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_in", "n_out", "n_kv_heads", "head_dim", "n_layers", "page_size", "dtype", "kv_format",
                                         "max_pages", "reserve", "window", "n_first")] + [("n_pages", C.c_int64)] + [
        (n, C.c_void_p) for n in ("pool", "page_table", "lens", "parents", "refs", "table_out", "lens_out", "refs_out",
                                  "entry_pos", "entry_weight", "err")]


class TlfCompactArgs(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n", "n_kv_heads", "head_dim", "n_layers", "page_size", "dtype", "kv_format",
                                         "max_pages")] + [("n_pages", C.c_int64)] + [
        (n, C.c_void_p) for n in ("pool", "page_table", "refs", "table_out", "refs_out", "n_live", "entry_pos", "entry_weight",
                                  "err")]


class TlfError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code
        self.name = ERRORS.get(code, str(code))


_LIB = None
_P = C.c_void_p
_I32P = C.POINTER(C.c_int32)
_U64P = C.POINTER(C.c_uint64)
_F32P = C.POINTER(C.c_float)

_SIGS = {
    "tlf_validate_config": (C.c_int, [C.POINTER(TlfConfig), C.c_char_p, C.c_size_t]),
    "tlf_page_bytes": (C.c_int64, [C.POINTER(TlfConfig)]),
    "tlf_create": (C.c_int, [C.POINTER(TlfConfig), C.POINTER(TlfWeights), C.POINTER(_P)]),
    "tlf_destroy": (None, [_P]),
    "tlf_last_error": (C.c_char_p, [_P]),
    "tlf_prefill": (C.c_int, [_P, C.c_int32, _U64P, _I32P, _I32P, _I32P, _P, _I32P, _P]),
    "tlf_decode_step": (C.c_int, [_P, C.c_int32, _U64P, _I32P, _I32P, _P, _I32P, _F32P, _P]),
    "tlf_release": (C.c_int, [_P, C.c_uint64]),
    "tlf_load_cache": (C.c_int, [_P, C.c_uint64, _I32P, _I32P, _P, _P]),
    "tlf_stats": (C.c_int, [_P, _I32P, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
    "tlf_cache_len": (C.c_int, [_P, C.c_uint64, C.c_int32, _I32P]),
    "tlf_read_cache": (C.c_int, [_P, C.c_uint64, C.c_int32, C.c_int32, _I32P, _F32P, _F32P]),
    "tlf_last_active_sets": (C.c_int, [_P, _I32P, _I32P]),
    "tlf_set_profiling": (C.c_int, [_P, C.c_int32]),
    "tlf_last_step_profile": (C.c_int, [_P, _F32P, C.POINTER(C.c_double), _I32P]),
    "tlf_last_step_kernel_times": (C.c_int, [_P, _F32P, C.c_int32]),
    "tlf_attn_decode_scratch_bytes": (C.c_size_t, [C.POINTER(TlfAttnArgs)]),
    "tlf_attn_decode": (C.c_int, [C.POINTER(TlfAttnArgs), _P, C.c_size_t, _P]),
    "tlf_attn_decode_static": (C.c_int, [C.POINTER(TlfAttnArgs), _P]),
    "tlf_rope_table": (C.c_int, [C.POINTER(TlfRopeConfig), C.c_int32, _P, _P]),
    "tlf_rope_append": (C.c_int, [C.POINTER(TlfChunk), C.POINTER(TlfRopeArgs), _P]),
    "tlf_attn_chunk_scratch_bytes": (C.c_size_t, [C.POINTER(TlfChunk), C.POINTER(TlfAttnChunkArgs)]),
    "tlf_attn_chunk": (C.c_int, [C.POINTER(TlfChunk), C.POINTER(TlfAttnChunkArgs), _P, C.c_size_t, _P]),
    "tlf_cache_evict_scratch_bytes": (C.c_size_t, [C.POINTER(TlfEvictArgs)]),
    "tlf_cache_evict": (C.c_int, [C.POINTER(TlfEvictArgs), _P, C.c_size_t, _P]),
    "tlf_sample": (C.c_int, [C.POINTER(TlfSampleArgs), _P]),
    "tlf_kv4_block_bytes": (C.c_int64, [C.c_int32]),
    "tlf_kv4_append": (C.c_int, [C.POINTER(TlfChunk), C.POINTER(TlfRopeArgs), _P]),
    "tlf_kv4_read": (C.c_int, [C.POINTER(TlfChunk), C.POINTER(TlfKv4ReadArgs), _P]),
    "tlf_attn_window_scratch_bytes": (C.c_size_t, [C.POINTER(TlfChunk), C.POINTER(TlfAttnWindowArgs)]),
    "tlf_attn_window": (C.c_int, [C.POINTER(TlfChunk), C.POINTER(TlfAttnWindowArgs), _P, C.c_size_t, _P]),
    "tlf_cache_fork_scratch_bytes": (C.c_size_t, [C.POINTER(TlfForkArgs)]),
    "tlf_cache_fork": (C.c_int, [C.POINTER(TlfForkArgs), _P, C.c_size_t, _P]),
    "tlf_cache_compact_scratch_bytes": (C.c_size_t, [C.POINTER(TlfCompactArgs)]),
    "tlf_cache_compact": (C.c_int, [C.POINTER(TlfCompactArgs), _P, C.c_size_t, _P]),
}


def library_path() -> str:
    return _build.LIB


def load_library(path: Optional[str] = None):
    """Load libtlf.so (built in-tree by __graft_entry__.build()); raises if missing."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    p = path or library_path()
    if not os.path.exists(p):
        raise RuntimeError(f"libtlf.so not found at {p}: build it with __graft_entry__.build() "
                           "(the decode step has no fallback path)")
    lib = C.CDLL(p)
    for name, (res, args) in _SIGS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path is None:
        _LIB = lib
    return lib


def _ptr(a, ctype):
    return None if a is None else a.ctypes.data_as(C.POINTER(ctype))


def _check(rc: int, ctx=None):
    if rc != TLF_OK:
        msg = load_library().tlf_last_error(ctx).decode()
        raise TlfError(rc, msg)


def _addr(buf) -> Optional[int]:
    """Address of a numpy array or a torch tensor (host or device)."""
    if buf is None:
        return None
    if hasattr(buf, "data_ptr"):
        return buf.data_ptr()
    return buf.ctypes.data


def _stream(stream) -> Optional[int]:
    if stream is None:
        return None
    try:
        return stream.cuda_stream
    except AttributeError:
        return int(stream)


# ----------------------------------------------------------------------------
# C names
# ----------------------------------------------------------------------------

def make_config(m, max_seqs: int, max_batch: int, max_seq_len: int, page_size: int = 64,
                kv_pool_pages: int = 0, gemm_impl: str = "auto", host_only: bool = False,
                prefill_chunk: int = 0, ablation: str = "none") -> TlfConfig:
    return TlfConfig(vocab=m.vocab, d_model=m.d_model, n_heads=m.n_heads, n_kv_heads=m.n_kv_heads,
                     head_dim=m.head_dim, n_layers=m.n_layers, ffn_hidden=m.ffn_hidden, max_loops=m.max_loops,
                     rope_base=m.rope_base, norm_eps=m.norm_eps, dtype=DTYPE[m.dtype], exit_rule=EXIT[m.exit_rule],
                     threshold=m.threshold, max_seqs=max_seqs, max_batch=max_batch, max_seq_len=max_seq_len,
                     page_size=page_size, gemm_impl=GEMM[gemm_impl], host_only=int(host_only), prefill_chunk=prefill_chunk,
                     kv_pool_pages=kv_pool_pages, ablation=ABLATION[ablation],
                     conditioning=int(getattr(m, "conditioning", False)),
                     router_hidden=int(getattr(m, "router_hidden", 0)))


def tlf_validate_config(cfg: TlfConfig):
    buf = C.create_string_buffer(256)
    rc = load_library().tlf_validate_config(C.byref(cfg), buf, 256)
    return rc, buf.value.decode()


def tlf_page_bytes(cfg: TlfConfig) -> int:
    return load_library().tlf_page_bytes(C.byref(cfg))


def _matrix(a: np.ndarray, dtype: str) -> np.ndarray:
    if dtype == "bf16":
        return np.ascontiguousarray(_synth.bf16_bits(a))
    return np.ascontiguousarray(a, dtype=np.float32)


def tlf_create(cfg: TlfConfig, weights: Optional[Dict[str, np.ndarray]], dtype: str):
    """Returns (ctx handle, kept arrays). weights: the dict of synth.make_weights."""
    keep = {}
    w = TlfWeights()
    if weights is not None:
        for name in ("embedding", "router_w", "wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down"):
            keep[name] = _matrix(weights[name], dtype)
        for name in ("router_b", "attn_norm", "mlp_norm", "final_norm"):
            keep[name] = np.ascontiguousarray(weights[name], dtype=np.float32)
        if cfg.conditioning:
            for name in COND_WEIGHTS:
                keep[name] = np.ascontiguousarray(weights[name], dtype=np.float32)
        if cfg.router_hidden:
            keep["router_w1"] = _matrix(weights["router_w1"], dtype)
            keep["router_b1"] = np.ascontiguousarray(weights["router_b1"], dtype=np.float32)
        for name, arr in keep.items():
            setattr(w, name, arr.ctypes.data)
    h = _P()
    rc = load_library().tlf_create(C.byref(cfg), C.byref(w) if weights is not None else None, C.byref(h))
    _check(rc, None)
    return h, keep


def tlf_destroy(ctx):
    load_library().tlf_destroy(ctx)


def tlf_prefill(ctx, seq_ids: np.ndarray, offsets: np.ndarray, tokens: np.ndarray, forced, last_logits, loops,
                stream=None):
    rc = load_library().tlf_prefill(ctx, len(seq_ids), _ptr(seq_ids, C.c_uint64), _ptr(offsets, C.c_int32),
                                    _ptr(tokens, C.c_int32), _ptr(forced, C.c_int32), _addr(last_logits),
                                    _ptr(loops, C.c_int32), _stream(stream))
    _check(rc, ctx)


def tlf_decode_step(ctx, seq_ids: np.ndarray, tokens: np.ndarray, forced, logits, loops: np.ndarray, margin,
                    stream=None):
    rc = load_library().tlf_decode_step(ctx, len(seq_ids), _ptr(seq_ids, C.c_uint64), _ptr(tokens, C.c_int32),
                                        _ptr(forced, C.c_int32), _addr(logits), _ptr(loops, C.c_int32),
                                        _ptr(margin, C.c_float), _stream(stream))
    _check(rc, ctx)


def tlf_release(ctx, seq_id: int):
    _check(load_library().tlf_release(ctx, C.c_uint64(seq_id)), ctx)


def tlf_load_cache(ctx, seq_id: int, lens: np.ndarray, positions: np.ndarray, k: Optional[np.ndarray],
                   v: Optional[np.ndarray]):
    """k = v = None: entries are filled on the device (see include/tlf.h)."""
    _check(load_library().tlf_load_cache(ctx, C.c_uint64(seq_id), _ptr(lens, C.c_int32), _ptr(positions, C.c_int32),
                                         None if k is None else k.ctypes.data,
                                         None if v is None else v.ctypes.data), ctx)


def attn_args(n, n_heads, n_kv_heads, head_dim, n_layers, layer, dtype, max_pages, n_pages, q, pool, page_table,
              lens, out, err=None) -> TlfAttnArgs:
    """Arguments of tlf_attn_decode; buffers are torch CUDA tensors (or raw device addresses)."""
    return TlfAttnArgs(n=n, n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, n_layers=n_layers,
                       layer=layer, page_size=64, dtype=DTYPE[dtype] if isinstance(dtype, str) else dtype,
                       max_pages=max_pages, reserved0=0, n_pages=n_pages, q=_addr(q), pool=_addr(pool),
                       page_table=_addr(page_table), lens=_addr(lens), out=_addr(out), err=_addr(err))


def tlf_attn_decode_scratch_bytes(a: TlfAttnArgs) -> int:
    return load_library().tlf_attn_decode_scratch_bytes(C.byref(a))


def tlf_attn_decode(a: TlfAttnArgs, scratch, scratch_bytes: int, stream=None):
    _check(load_library().tlf_attn_decode(C.byref(a), _addr(scratch), scratch_bytes, _stream(stream)), None)


def tlf_attn_decode_static(a: TlfAttnArgs, stream=None):
    """tlf_attn_decode without caller scratch: uses the library's built-in 4 MiB device array."""
    _check(load_library().tlf_attn_decode_static(C.byref(a), _stream(stream)), None)


# Operators on a caller's paged caches and logits. The builders take torch CUDA tensors, read shapes, types and strides off
# them, and keep them alive with the arguments; a program makes the arguments once for its buffers and calls with them.

def _torch_dtype(t) -> int:
    name = str(t.dtype)
    if name == "torch.float32":
        return DTYPE["f32"]
    if name in ("torch.bfloat16", "torch.int16", "torch.uint16"):  # bfloat16, or its bits
        return DTYPE["bf16"]
    raise ValueError(f"{name}: float32 or bfloat16 is wanted")


def _dense(what: str, t, dtype: Optional[str], *shape):
    """A contiguous tensor of the given type and shape (None: any extent), or None."""
    if t is None:
        return None
    if not t.is_contiguous() or (dtype and str(t.dtype) != "torch." + dtype) or len(t.shape) != len(shape) or any(
            w is not None and w != h for w, h in zip(shape, t.shape)):
        raise ValueError(f"{what}: a contiguous {dtype or ''} tensor of shape {shape} is wanted, got {str(t.dtype)} "
                         f"{tuple(t.shape)}")
    return t


def _heads(what: str, t, dtype: int, rows: int, heads: int, hd: int) -> int:
    """Elements between the rows of a tensor of shape [rows or more, heads, hd] or [rows or more, heads * hd]."""
    if _torch_dtype(t) != dtype or tuple(t.shape[1:]) not in ((heads, hd), (heads * hd,)) or t.shape[0] < rows or \
            t.stride(-1) != 1 or (t.dim() == 3 and t.stride(1) != hd):
        raise ValueError(f"{what}: {rows} rows of {heads} heads of {hd} in the pool's type are wanted, each row contiguous, got "
                         f"{str(t.dtype)} {tuple(t.shape)} with strides {t.stride()}")
    return t.stride(0)


def chunk_args(pool, page_table, cu_tokens, lens, n_heads: int, n_tokens: int, layer: int = 0, max_chunk: int = 0,
               err=None) -> TlfChunk:
    """A batch of chunks over a paged cache: pool [pages, layers, 2, kv heads, 64, head_dim], page_table [n, most pages]
    int32, cu_tokens [n + 1] int32, lens [n] int32 (with the new tokens)."""
    if len(pool.shape) != 6 or pool.shape[2] != 2:
        raise ValueError(f"pool: [pages, layers, 2, kv heads, 64, head_dim] is wanted, got {tuple(pool.shape)}")
    _dense("pool", pool, None, *pool.shape)
    n = page_table.shape[0]
    _dense("page_table", page_table, "int32", n, None)
    _dense("cu_tokens", cu_tokens, "int32", n + 1)
    _dense("lens", lens, "int32", n)
    c = TlfChunk(n=n, n_tokens=n_tokens, max_chunk=max_chunk, n_heads=n_heads, n_kv_heads=pool.shape[3],
                 head_dim=pool.shape[5], n_layers=pool.shape[1], layer=layer, page_size=pool.shape[4],
                 dtype=_torch_dtype(pool), max_pages=page_table.shape[1], n_pages=pool.shape[0], pool=_addr(pool),
                 page_table=_addr(page_table), cu_tokens=_addr(cu_tokens), lens=_addr(lens), err=_addr(err))
    c.kept = (pool, page_table, cu_tokens, lens, err)
    return c


def rope_config(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original_len: float = 0.0,
                low_turns: float = 1.0, high_turns: float = 32.0, magnitude: float = 1.0) -> TlfRopeConfig:
    return TlfRopeConfig(rot_dim=rot_dim, scaling=ROPE_SCALING[scaling], base=base, factor=factor,
                         original_len=original_len, low_turns=low_turns, high_turns=high_turns, magnitude=magnitude)


def tlf_rope_table(cfg: TlfRopeConfig, max_pos: int, table, stream=None):
    """Fills table, a float32 tensor [max_pos, rot_dim / 2, 2]."""
    _dense("table", table, "float32", max_pos, cfg.rot_dim // 2, 2)
    _check(load_library().tlf_rope_table(C.byref(cfg), max_pos, _addr(table), _stream(stream)), None)


def rope_args(q, k, v, positions, table, q_out, layout: str = "half", entry_pos=None, entry_weight=None) -> TlfRopeArgs:
    """q, k, v: [tokens, heads, head_dim] or [tokens, heads * head_dim], for example three parts of one projection's output;
    table [max_pos, rot_dim / 2, 2]; q_out [tokens, heads, head_dim] in the pool's type or in float32."""
    T, hq, hd = q_out.shape
    _dense("table", table, "float32", None, None, 2)
    _dense("positions", positions, "int32", None)
    _dense("q_out", q_out, None, T, hq, hd)
    _dense("entry_pos", entry_pos, "int32", None, 64)
    _dense("entry_weight", entry_weight, "float32", None, 64)
    dt = _torch_dtype(q)
    kh = k.shape[1] if k.dim() == 3 else k.shape[1] // hd
    a = TlfRopeArgs(q=_addr(q), k=_addr(k), v=_addr(v), q_stride=_heads("q", q, dt, 0, hq, hd),
                    k_stride=_heads("k", k, dt, 0, kh, hd), v_stride=_heads("v", v, dt, 0, kh, hd),
                    positions=_addr(positions), table=_addr(table), max_pos=table.shape[0], rot_dim=2 * table.shape[1],
                    layout=ROPE_LAYOUT[layout], q_f32=int(_torch_dtype(q_out) == DTYPE["f32"] != dt), q_out=_addr(q_out),
                    entry_pos=_addr(entry_pos), entry_weight=_addr(entry_weight))
    a.kept = (q, k, v, positions, table, q_out, entry_pos, entry_weight)
    a.fits = (min(x.shape[0] for x in (q, k, v, positions, q_out)), hq, kh, hd, dt, [
        t.shape[0] for t in (entry_pos, entry_weight) if t is not None])
    return a


def _format(c: TlfChunk, four_bits: bool):
    if getattr(c, "four_bits", False) != four_bits:
        raise ValueError("the batch's cache is in 4 bits (chunk4_args) and the call is for one in the dtype, or the other way round")


def _pair(c: TlfChunk, a):
    """The arguments' tensors are large enough for the batch (looked at once for the same batch: a program may change it)."""
    batch = bytes(c)  # (one copy instead of six fields, each call)
    if getattr(a, "batch", None) == batch:
        return
    rows, hq, kh, hd, dt, pages = a.fits
    if rows < c.n_tokens or (hq and hq != c.n_heads) or (kh and kh != c.n_kv_heads) or hd != c.head_dim or dt != c.dtype or any(
            p != c.n_pages for p in pages):
        raise ValueError(f"the arguments are for {rows} tokens of {hq} heads of {hd} and caches of {pages} pages, the batch has "
                         f"{c.n_tokens} tokens of {c.n_heads} heads of {c.head_dim} and {c.n_pages} pages")
    a.batch = batch


def tlf_rope_append(c: TlfChunk, a: TlfRopeArgs, stream=None):
    _format(c, False)
    _pair(c, a)
    _check(load_library().tlf_rope_append(C.byref(c), C.byref(a), _stream(stream)), None)


def attn_chunk_args(q, out, lse=None, weight_in=None, weight_out=None, scale: float = 0.0) -> TlfAttnChunkArgs:
    """q, out: [tokens, heads, head_dim], rows any stride apart; lse [tokens, heads] float32; weights [pages, 64] float32."""
    _, hq, hd = q.shape
    _dense("lse", lse, "float32", None, hq)
    _dense("weight_in", weight_in, "float32", None, 64)
    _dense("weight_out", weight_out, "float32", None, 64)
    dt = _torch_dtype(q)
    a = TlfAttnChunkArgs(q=_addr(q), q_stride=_heads("q", q, dt, 0, hq, hd), out=_addr(out),
                         out_stride=_heads("out", out, dt, q.shape[0], hq, hd), lse=_addr(lse), weight_in=_addr(weight_in),
                         weight_out=_addr(weight_out), scale=scale)
    a.kept = (q, out, lse, weight_in, weight_out)
    a.fits = (min(x.shape[0] for x in (q, out, lse) if x is not None), hq, 0, hd, dt,
              [t.shape[0] for t in (weight_in, weight_out) if t is not None])
    return a


def tlf_attn_chunk_scratch_bytes(c: TlfChunk, a: TlfAttnChunkArgs) -> int:
    return load_library().tlf_attn_chunk_scratch_bytes(C.byref(c), C.byref(a))


def tlf_attn_chunk(c: TlfChunk, a: TlfAttnChunkArgs, scratch, scratch_bytes: int, stream=None):
    _format(c, False)
    _pair(c, a)
    _check(load_library().tlf_attn_chunk(C.byref(c), C.byref(a), _addr(scratch), scratch_bytes, _stream(stream)), None)


def evict_args(pool, page_table, lens, next_pos, pos_in, pos_out, weight_in, weight_out, lens_out, budget: int,
               n_first: int = 0, n_recent: int = 0, err=None) -> TlfEvictArgs:
    """Shapes as in chunk_args; pos [pages, 64] int32, weight [pages, 64] float32."""
    if len(pool.shape) != 6 or pool.shape[2] != 2:
        raise ValueError(f"pool: [pages, layers, 2, kv heads, 64, head_dim] is wanted, got {tuple(pool.shape)}")
    _dense("pool", pool, None, *pool.shape)
    n, pages = page_table.shape[0], pool.shape[0]
    _dense("page_table", page_table, "int32", n, None)
    for what, t in (("lens", lens), ("next_pos", next_pos), ("lens_out", lens_out)):
        _dense(what, t, "int32", n)
    for what, t, dt in (("pos_in", pos_in, "int32"), ("pos_out", pos_out, "int32"), ("weight_in", weight_in, "float32"),
                        ("weight_out", weight_out, "float32")):
        _dense(what, t, dt, pages, 64)
    a = TlfEvictArgs(n=n, n_kv_heads=pool.shape[3], head_dim=pool.shape[5], n_layers=pool.shape[1], page_size=pool.shape[4],
                     dtype=_torch_dtype(pool), max_pages=page_table.shape[1], budget=budget, n_first=n_first,
                     n_recent=n_recent, n_pages=pages, pool=_addr(pool), page_table=_addr(page_table), lens=_addr(lens),
                     next_pos=_addr(next_pos), pos_in=_addr(pos_in), pos_out=_addr(pos_out), weight_in=_addr(weight_in),
                     weight_out=_addr(weight_out), lens_out=_addr(lens_out), err=_addr(err))
    a.kept = (pool, page_table, lens, next_pos, pos_in, pos_out, weight_in, weight_out, lens_out, err)
    return a


def tlf_cache_evict_scratch_bytes(a: TlfEvictArgs) -> int:
    return load_library().tlf_cache_evict_scratch_bytes(C.byref(a))


def tlf_cache_evict(a: TlfEvictArgs, scratch, scratch_bytes: int, stream=None):
    _check(load_library().tlf_cache_evict(C.byref(a), _addr(scratch), scratch_bytes, _stream(stream)), None)


def sample_args(logits, noise, tokens, logprobs=None, temperature=None, top_k=None, top_p=None, min_p=None) -> TlfSampleArgs:
    """logits, noise: float32 [rows, vocab], rows any stride apart; tokens int32 [rows]; logprobs and the parameters [rows]."""
    n, V = logits.shape
    for what, t in (("logits", logits), ("noise", noise)):
        if str(t.dtype) != "torch.float32" or tuple(t.shape) != (n, V) or t.stride(1) != 1:
            raise ValueError(f"{what}: float32 [{n}, {V}] with contiguous rows is wanted, got {str(t.dtype)} {tuple(t.shape)}")
    _dense("tokens", tokens, "int32", n)
    for what, t, dt in (("logprobs", logprobs, "float32"), ("temperature", temperature, "float32"), ("top_k", top_k, "int32"),
                        ("top_p", top_p, "float32"), ("min_p", min_p, "float32")):
        _dense(what, t, dt, n)
    a = TlfSampleArgs(n=n, vocab=V, logits=_addr(logits), logits_stride=logits.stride(0), noise=_addr(noise),
                      noise_stride=noise.stride(0), temperature=_addr(temperature), top_k=_addr(top_k), top_p=_addr(top_p),
                      min_p=_addr(min_p), tokens=_addr(tokens), logprobs=_addr(logprobs))
    a.kept = (logits, noise, tokens, logprobs, temperature, top_k, top_p, min_p)
    return a


def tlf_sample(a: TlfSampleArgs, stream=None):
    _check(load_library().tlf_sample(C.byref(a), _stream(stream)), None)


# ---- caches in 4 bits, windows, and who owns a page ----

def kv4_block_bytes(head_dim: int) -> int:
    """Bytes of a block (one layer, K or V, one head) of a page in 4 bits."""
    if head_dim not in (16, 32, 64, 128):
        raise ValueError(f"head_dim {head_dim}: 16, 32, 64 or 128 is wanted")
    return 64 * (head_dim // 2 + 4 * max(1, head_dim // 64))


def _pool4(pool, head_dim: int):
    size = kv4_block_bytes(head_dim)
    if len(pool.shape) != 5 or pool.shape[2] != 2 or pool.shape[4] != size:
        raise ValueError(f"pool: [pages, layers, 2, kv heads, {size}] bytes are wanted for a cache in 4 bits with head_dim "
                         f"{head_dim}, got {tuple(pool.shape)}")
    _dense("pool", pool, "uint8", *pool.shape)


def chunk4_args(pool, page_table, cu_tokens, lens, n_heads: int, n_tokens: int, head_dim: int, dtype: str = "bf16", layer: int = 0,
                max_chunk: int = 0, err=None) -> TlfChunk:
    """chunk_args for a cache in 4 bits: pool [pages, layers, 2, kv heads, kv4_block_bytes(head_dim)] uint8; dtype: of the queries,
    keys, values and outputs."""
    _pool4(pool, head_dim)
    n = page_table.shape[0]
    _dense("page_table", page_table, "int32", n, None)
    _dense("cu_tokens", cu_tokens, "int32", n + 1)
    _dense("lens", lens, "int32", n)
    c = TlfChunk(n=n, n_tokens=n_tokens, max_chunk=max_chunk, n_heads=n_heads, n_kv_heads=pool.shape[3], head_dim=head_dim,
                 n_layers=pool.shape[1], layer=layer, page_size=64, dtype=DTYPE[dtype], max_pages=page_table.shape[1],
                 n_pages=pool.shape[0], pool=_addr(pool), page_table=_addr(page_table), cu_tokens=_addr(cu_tokens),
                 lens=_addr(lens), err=_addr(err))
    c.kept = (pool, page_table, cu_tokens, lens, err)
    c.four_bits = True
    return c


def tlf_kv4_append(c: TlfChunk, a: TlfRopeArgs, stream=None):
    """tlf_rope_append (its rope_args) into a cache in 4 bits."""
    _format(c, True)
    _pair(c, a)
    _check(load_library().tlf_kv4_append(C.byref(c), C.byref(a), _stream(stream)), None)


def kv4_read_args(k=None, v=None) -> TlfKv4ReadArgs:
    """k, v: [tokens, kv heads, head_dim], rows any stride apart; None: not wanted."""
    t = k if k is not None else v
    if t is None:
        raise ValueError("k or v is wanted")
    _, kh, hd = t.shape
    dt = _torch_dtype(t)
    a = TlfKv4ReadArgs(k=_addr(k), v=_addr(v), k_stride=0 if k is None else _heads("k", k, dt, 0, kh, hd),
                       v_stride=0 if v is None else _heads("v", v, dt, 0, kh, hd))
    a.kept = (k, v)
    a.fits = (min(x.shape[0] for x in (k, v) if x is not None), 0, kh, hd, dt, [])
    return a


def tlf_kv4_read(c: TlfChunk, a: TlfKv4ReadArgs, stream=None):
    _format(c, True)
    _pair(c, a)
    _check(load_library().tlf_kv4_read(C.byref(c), C.byref(a), _stream(stream)), None)


def attn_window_args(q, out, lse=None, window: int = 0, n_first: int = 0, kv4: bool = False, scale: float = 0.0) -> TlfAttnWindowArgs:
    """As attn_chunk_args, without weights; window 0: no window; kv4: the batch's cache is in 4 bits (chunk4_args)."""
    _, hq, hd = q.shape
    _dense("lse", lse, "float32", None, hq)
    dt = _torch_dtype(q)
    a = TlfAttnWindowArgs(q=_addr(q), q_stride=_heads("q", q, dt, 0, hq, hd), out=_addr(out),
                          out_stride=_heads("out", out, dt, q.shape[0], hq, hd), lse=_addr(lse), scale=scale, window=window,
                          n_first=n_first, kv_format=int(kv4))
    a.kept = (q, out, lse)
    a.fits = (min(x.shape[0] for x in (q, out, lse) if x is not None), hq, 0, hd, dt, [])
    return a


def tlf_attn_window_scratch_bytes(c: TlfChunk, a: TlfAttnWindowArgs) -> int:
    return load_library().tlf_attn_window_scratch_bytes(C.byref(c), C.byref(a))


def tlf_attn_window(c: TlfChunk, a: TlfAttnWindowArgs, scratch, scratch_bytes: int, stream=None):
    _format(c, a.kv_format == KV_FORMAT["4bit"])
    _pair(c, a)
    _check(load_library().tlf_attn_window(C.byref(c), C.byref(a), _addr(scratch), scratch_bytes, _stream(stream)), None)


def _page_pool(pool, head_dim: Optional[int]) -> dict:
    """The shape fields of a pool: [pages, layers, 2, kv heads, 64, head_dim], or in 4 bits (head_dim given) [.., block bytes] uint8."""
    if head_dim is not None:
        _pool4(pool, head_dim)
        return dict(n_kv_heads=pool.shape[3], head_dim=head_dim, n_layers=pool.shape[1], page_size=64,
                    dtype=DTYPE["f32" if head_dim == 16 else "bf16"], kv_format=KV_FORMAT["4bit"], n_pages=pool.shape[0], pool=_addr(pool))
    if len(pool.shape) != 6 or pool.shape[2] != 2:
        raise ValueError(f"pool: [pages, layers, 2, kv heads, 64, head_dim] is wanted, got {tuple(pool.shape)}")
    _dense("pool", pool, None, *pool.shape)
    return dict(n_kv_heads=pool.shape[3], head_dim=pool.shape[5], n_layers=pool.shape[1], page_size=pool.shape[4],
                dtype=_torch_dtype(pool), kv_format=KV_FORMAT["plain"], n_pages=pool.shape[0], pool=_addr(pool))


def fork_args(pool, page_table, lens, parents, refs, table_out, lens_out, refs_out, reserve: int = 0, window: int = 0,
              n_first: int = 0, entry_pos=None, entry_weight=None, head_dim: Optional[int] = None, err=None) -> TlfForkArgs:
    """page_table [old rows, most pages], lens [old rows]; parents, lens_out [new rows], table_out [new rows, most pages]; refs,
    refs_out [pages]; entry_pos, entry_weight [pages, 64]. head_dim: of a pool in 4 bits (None: the pool has its dtype)."""
    n_in, width = page_table.shape
    n_out, pages = parents.shape[0], pool.shape[0]
    for what, t, shape in (("page_table", page_table, (n_in, width)), ("lens", lens, (n_in,)), ("parents", parents, (n_out,)),
                           ("table_out", table_out, (n_out, width)), ("lens_out", lens_out, (n_out,)), ("refs", refs, (pages,)),
                           ("refs_out", refs_out, (pages,)), ("entry_pos", entry_pos, (pages, 64))):
        _dense(what, t, "int32", *shape)
    _dense("entry_weight", entry_weight, "float32", pages, 64)
    a = TlfForkArgs(n_in=n_in, n_out=n_out, max_pages=width, reserve=reserve, window=window, n_first=n_first,
                    page_table=_addr(page_table), lens=_addr(lens), parents=_addr(parents), refs=_addr(refs),
                    table_out=_addr(table_out), lens_out=_addr(lens_out), refs_out=_addr(refs_out), entry_pos=_addr(entry_pos),
                    entry_weight=_addr(entry_weight), err=_addr(err), **_page_pool(pool, head_dim))
    a.kept = (pool, page_table, lens, parents, refs, table_out, lens_out, refs_out, entry_pos, entry_weight, err)
    return a


def tlf_cache_fork_scratch_bytes(a: TlfForkArgs) -> int:
    return load_library().tlf_cache_fork_scratch_bytes(C.byref(a))


def tlf_cache_fork(a: TlfForkArgs, scratch, scratch_bytes: int, stream=None):
    _check(load_library().tlf_cache_fork(C.byref(a), _addr(scratch), scratch_bytes, _stream(stream)), None)


def compact_args(pool, page_table, refs, table_out, refs_out, n_live, entry_pos=None, entry_weight=None,
                 head_dim: Optional[int] = None, err=None) -> TlfCompactArgs:
    """Shapes as in fork_args; table_out as page_table, n_live [1] int32."""
    n, width = page_table.shape
    pages = pool.shape[0]
    for what, t, shape in (("page_table", page_table, (n, width)), ("table_out", table_out, (n, width)), ("refs", refs, (pages,)),
                           ("refs_out", refs_out, (pages,)), ("n_live", n_live, (1,)), ("entry_pos", entry_pos, (pages, 64))):
        _dense(what, t, "int32", *shape)
    _dense("entry_weight", entry_weight, "float32", pages, 64)
    a = TlfCompactArgs(n=n, max_pages=width, page_table=_addr(page_table), refs=_addr(refs), table_out=_addr(table_out),
                       refs_out=_addr(refs_out), n_live=_addr(n_live), entry_pos=_addr(entry_pos), entry_weight=_addr(entry_weight),
                       err=_addr(err), **_page_pool(pool, head_dim))
    a.kept = (pool, page_table, refs, table_out, refs_out, n_live, entry_pos, entry_weight, err)
    return a


def tlf_cache_compact_scratch_bytes(a: TlfCompactArgs) -> int:
    return load_library().tlf_cache_compact_scratch_bytes(C.byref(a))


def tlf_cache_compact(a: TlfCompactArgs, scratch, scratch_bytes: int, stream=None):
    _check(load_library().tlf_cache_compact(C.byref(a), _addr(scratch), scratch_bytes, _stream(stream)), None)


# ----------------------------------------------------------------------------
# convenience wrapper
# ----------------------------------------------------------------------------

class Context:
    """One library context for a model configuration (synth.ModelConfig)."""

    def __init__(self, model, weights: Optional[Dict[str, np.ndarray]], max_seqs: int, max_batch: int,
                 max_seq_len: int, kv_pool_pages: int = 0, gemm_impl: str = "auto", host_only: bool = False,
                 prefill_chunk: int = 0, ablation: str = "none"):
        self.model = model
        self.cfg = make_config(model, max_seqs, max_batch, max_seq_len, kv_pool_pages=kv_pool_pages,
                               gemm_impl=gemm_impl, host_only=host_only, prefill_chunk=prefill_chunk,
                               ablation=ablation)
        self.handle, _ = tlf_create(self.cfg, weights, model.dtype)
        self.max_batch = max_batch

    def close(self):
        if self.handle:
            tlf_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill(self, seq_ids: Sequence[int], prompts: Sequence[np.ndarray], forced=None, logits: bool = True,
                logits_out=None, stream=None):
        """Returns (last logits [n, V] numpy or logits_out, loops list of int32 arrays)."""
        ids = np.asarray(seq_ids, dtype=np.uint64)
        lens = np.array([len(p) for p in prompts], dtype=np.int64)
        offsets = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        toks = np.ascontiguousarray(np.concatenate([np.asarray(p, dtype=np.int32) for p in prompts]))
        frc = None if forced is None else np.ascontiguousarray(np.concatenate(
            [np.asarray(f, dtype=np.int32) for f in forced]))
        out = logits_out
        if logits and out is None:
            out = np.zeros((len(prompts), self.model.vocab), dtype=np.float32)
        loops = np.zeros(int(offsets[-1]), dtype=np.int32)
        tlf_prefill(self.handle, ids, offsets, toks, frc, out if logits else None, loops, stream)
        return out, [loops[offsets[i]:offsets[i + 1]] for i in range(len(prompts))]

    def decode_step(self, seq_ids: Sequence[int], tokens: Sequence[int], forced=None, logits=True, stream=None):
        """Returns (logits [B, V] (numpy, or the given buffer), loops [B], margins [B])."""
        ids = np.asarray(seq_ids, dtype=np.uint64)
        toks = np.ascontiguousarray(tokens, dtype=np.int32)
        frc = None if forced is None else np.ascontiguousarray(forced, dtype=np.int32)
        if logits is True:
            out = np.zeros((len(ids), self.model.vocab), dtype=np.float32)
        elif logits is False or logits is None:
            out = None
        else:
            out = logits
        loops = np.zeros(len(ids), dtype=np.int32)
        margin = np.zeros(len(ids), dtype=np.float32)
        tlf_decode_step(self.handle, ids, toks, frc, out, loops, margin, stream)
        return out, loops, margin

    def release(self, seq_id: int):
        tlf_release(self.handle, seq_id)

    def load_cache(self, seq_id: int, snapshot: dict):
        """snapshot: synth.make_cache_snapshot output (values exact in the model dtype); without
        "k"/"v" entries (synth.make_cache_positions) the values are filled on the device."""
        lens = np.array([len(p) for p in snapshot["positions"]], dtype=np.int32)
        pos = np.ascontiguousarray(np.concatenate(snapshot["positions"]).astype(np.int32))
        if "k" not in snapshot:
            tlf_load_cache(self.handle, seq_id, lens, pos, None, None)
            return
        k = np.concatenate(snapshot["k"]).astype(np.float32)
        v = np.concatenate(snapshot["v"]).astype(np.float32)
        tlf_load_cache(self.handle, seq_id, lens, pos, _matrix(k, self.model.dtype), _matrix(v, self.model.dtype))

    def stats(self):
        live, free, total = C.c_int32(), C.c_int64(), C.c_int64()
        _check(load_library().tlf_stats(self.handle, C.byref(live), C.byref(free), C.byref(total)), self.handle)
        return live.value, free.value, total.value

    def cache_len(self, seq_id: int, loop: int) -> int:
        n = C.c_int32()
        _check(load_library().tlf_cache_len(self.handle, C.c_uint64(seq_id), loop, C.byref(n)), self.handle)
        return n.value

    def read_cache(self, seq_id: int, loop: int, layer: int):
        n = self.cache_len(seq_id, loop)
        m = self.model
        pos = np.zeros(n, dtype=np.int32)
        k = np.zeros((n, m.n_kv_heads, m.head_dim), dtype=np.float32)
        v = np.zeros_like(k)
        _check(load_library().tlf_read_cache(self.handle, C.c_uint64(seq_id), loop, layer, _ptr(pos, C.c_int32),
                                             _ptr(k, C.c_float), _ptr(v, C.c_float)), self.handle)
        return pos, k, v

    def last_active_sets(self, batch: int):
        M = self.model.max_loops
        counts = np.zeros(M, dtype=np.int32)
        idx = np.zeros(M * batch, dtype=np.int32)
        _check(load_library().tlf_last_active_sets(self.handle, _ptr(counts, C.c_int32), _ptr(idx, C.c_int32)),
               self.handle)
        return counts, [idx[r * batch: r * batch + counts[r]] for r in range(M)]

    def set_profiling(self, on: bool):
        _check(load_library().tlf_set_profiling(self.handle, int(on)), self.handle)

    def last_step_profile(self):
        ms, by, nl = C.c_float(), C.c_double(), C.c_int32()
        _check(load_library().tlf_last_step_profile(self.handle, C.byref(ms), C.byref(by), C.byref(nl)), self.handle)
        return ms.value, by.value, nl.value

    def last_step_kernel_times(self) -> Dict[str, float]:
        """Milliseconds per kernel class of the last profiled step."""
        ms = np.zeros(len(KERNEL_CLASSES), dtype=np.float32)
        _check(load_library().tlf_last_step_kernel_times(self.handle, _ptr(ms, C.c_float), len(ms)), self.handle)
        return dict(zip(KERNEL_CLASSES, ms.tolist()))
