"""Python binding of the operators of a prompt's pass (include/argus_prompt.h), beside those of a
decode step and over the same paged cache.

The functions named ``argus_prompt_*`` are one-to-one wrappers (argument marshalling only).
The others take torch CUDA tensors, as those of ``decode`` do: the same checks, streams, errors and
markers, no fallback, and no derivatives (a tensor that requires gradients is refused unless
gradients are off, and one with a forward-mode tangent).
"""
from __future__ import annotations

import ctypes
import math
import struct

from . import decode
from .attr import ABI_VERSION
from .decode import (BF16, FP8, FP16, FP32, NUM_REGIONS, REGION_NAMES, _bad, _buffer, _differentiable, _done, _elsewhere,
                     _ints, _marks, _no_tangents, _on, _pack, _scales, _table, _type, _view, _workspace, argus_markers, argus_page_view)

PROMPT_REGION_NAMES = ["chunk.plan", "chunk", "chunk.join", "rotate", "score.rows", "score.join"]
ALL_REGION_NAMES = REGION_NAMES + PROMPT_REGION_NAMES
NUM_ALL_REGIONS = len(ALL_REGION_NAMES)
MAX_TOP = 64

_u32, _i64, _p = ctypes.c_uint32, ctypes.c_int64, ctypes.c_void_p


class argus_chunk_config(ctypes.Structure):
    _fields_ = [(k, _u32) for k in ("abi_version", "q_type", "cache_type", "seqs", "rows", "kv_heads", "group",
                                    "head_dim", "page_size", "num_pages", "columns", "window", "sinks")]
    _fields_ += [("scale", ctypes.c_float)]


class argus_chunk_io(ctypes.Structure):
    _fields_ = [("d_q", _p), ("q_row_stride", _i64), ("q_head_stride", _i64), ("k", argus_page_view),
                ("v", argus_page_view), ("d_table", _p), ("table_stride", _i64), ("d_lens", _p), ("d_offsets", _p),
                ("d_k_scale", _p), ("d_v_scale", _p), ("d_out", _p), ("d_lse", _p)]


class argus_rotate_config(ctypes.Structure):
    _fields_ = [(k, _u32) for k in ("abi_version", "source_type", "cache_type", "seqs", "rows", "heads", "kv_heads",
                                    "head_dim", "pairs", "interleaved", "page_size", "num_pages", "columns")]
    _fields_ += [("amplitude", ctypes.c_float)]


class argus_rotate_io(ctypes.Structure):
    _fields_ = [("d_q", _p), ("q_row_stride", _i64), ("q_head_stride", _i64), ("d_out", _p), ("out_row_stride", _i64),
                ("out_head_stride", _i64), ("d_new_k", _p), ("d_new_v", _p), ("k_row_stride", _i64),
                ("k_head_stride", _i64), ("v_row_stride", _i64), ("v_head_stride", _i64), ("k", argus_page_view),
                ("v", argus_page_view), ("d_table", _p), ("table_stride", _i64), ("d_starts", _p), ("d_offsets", _p),
                ("d_frequencies", _p), ("d_k_scale", _p), ("d_v_scale", _p)]


class argus_score_config(ctypes.Structure):
    _fields_ = [(k, _u32) for k in ("abi_version", "type", "rows", "vocab", "top", "pad")]


class argus_score_io(ctypes.Structure):
    _fields_ = [("d_logits", _p), ("row_stride", _i64), ("d_tokens", _p), ("d_logprobs", _p), ("d_entropy", _p),
                ("d_ranks", _p), ("d_top_logprobs", _p), ("d_top_tokens", _p)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = decode._library()
        sz, mk = ctypes.c_size_t, ctypes.POINTER(argus_markers)
        for name, args in (("attend", [argus_chunk_config, argus_chunk_io, True]),
                           ("rotate", [argus_rotate_config, argus_rotate_io, False]),
                           ("score", [argus_score_config, argus_score_io, True])):
            f = getattr(lib, "argus_prompt_" + name)
            f.argtypes = [ctypes.POINTER(args[0]), ctypes.POINTER(args[1])]
            f.argtypes += ([_p, sz] if args[2] else []) + [mk, _p]
            f.restype = ctypes.c_int
            if args[2]:
                f = getattr(lib, f"argus_prompt_{name}_workspace_bytes")
                f.argtypes, f.restype = [ctypes.POINTER(args[0])], sz
        _lib = lib
    return _lib


def argus_prompt_attend_workspace_bytes(cfg) -> int:
    return _library().argus_prompt_attend_workspace_bytes(cfg)


def argus_prompt_attend(cfg, io, d_workspace, workspace_bytes, markers, stream) -> int:
    return _library().argus_prompt_attend(cfg, io, d_workspace, workspace_bytes, markers, stream)


def argus_prompt_rotate(cfg, io, markers, stream) -> int:
    return _library().argus_prompt_rotate(cfg, io, markers, stream)


def argus_prompt_score_workspace_bytes(cfg) -> int:
    return _library().argus_prompt_score_workspace_bytes(cfg)


def argus_prompt_score(cfg, io, d_workspace, workspace_bytes, markers, stream) -> int:
    return _library().argus_prompt_score(cfg, io, d_workspace, workspace_bytes, markers, stream)


# ------------------------------------------------------------ torch wrappers

_ready = False
_lib_attend = _lib_attend_bytes = _lib_rotate = _lib_score = _lib_score_bytes = None

# The structures of the header, field by field (native alignment).
_CHUNK_CONFIG, _CHUNK_IO = struct.Struct("13If"), struct.Struct("Q2q Q3q Q3q Qq 6Q")
_ROTATE_CONFIG, _ROTATE_IO = struct.Struct("13If"), struct.Struct("Q2q Q2q 2Q4q Q3q Q3q Qq 5Q")
_SCORE_CONFIG, _SCORE_IO = struct.Struct("6I"), struct.Struct("Qq 6Q")


def _t():
    global _ready, _lib_attend, _lib_attend_bytes, _lib_rotate, _lib_score, _lib_score_bytes
    torch = decode._t()
    if not _ready:
        lib, sz = _library(), ctypes.c_size_t

        def of(name, restype, *types):
            f = lib["argus_prompt_" + name]  # another object than the one with the structures' types
            f.argtypes, f.restype = [ctypes.c_char_p, *types], restype
            return f

        _lib_attend = of("attend", ctypes.c_int, ctypes.c_char_p, _p, sz, _p, _p)
        _lib_attend_bytes = of("attend_workspace_bytes", sz)
        _lib_rotate = of("rotate", ctypes.c_int, ctypes.c_char_p, _p, _p)
        _lib_score = of("score", ctypes.c_int, ctypes.c_char_p, _p, sz, _p, _p)
        _lib_score_bytes = of("score_workspace_bytes", sz)
        _ready = True
    return torch


def _rows(x, name: str, dev) -> tuple:
    """Strides of [rows, heads, head_dim] with contiguous rows."""
    st = x.stride()
    if not (len(st) == 3 and (st[2] == 1 or x.shape[2] == 1) and x.device == dev):
        _bad(f"{name}: [rows, heads, head_dim] with contiguous rows on {dev}")
    return st


def attend_chunks(q, k_cache, v_cache, table, lens, offsets, scale: float | None = None, window: int = 0,
                  sinks: int = 0, k_scale=None, v_scale=None, lse: bool = False, out=None, markers=None,
                  stream=None) -> dict:
    """Attention of chunks of new tokens over a paged cache that holds them already.

    q: [rows, heads, head_dim] bf16 or fp16, contiguous rows (a view of a fused projection's
    result does); sequence s has the rows offsets[s] to offsets[s + 1] (int32 [seqs + 1], never
    falling; one outside the rows is taken as the nearer end), the queries of its last positions; lens: int32 [seqs], its tokens, the new ones
    included.  A row sees the tokens up to its own; with a window the last `window` of these and
    the first `sinks`.  Caches, table and scales as in attend_pages.  Returns out (like q,
    dense) and, if asked, lse (float32 [rows, heads]); a row that sees nothing answers zeros and
    -inf.  Rows of no sequence are not written (a new `out` holds anything there)."""
    t = _t()
    dev = q.device
    if _elsewhere(stream, dev):
        with _on(stream, dev, q, k_cache, v_cache, table, lens, offsets, k_scale, v_scale, out, _buffer(markers)):
            return attend_chunks(q, k_cache, v_cache, table, lens, offsets, scale, window, sinks, k_scale, v_scale, lse,
                                 out, markers)
    qs = _rows(q, "q", dev)
    T, heads, D = q.shape
    qt = _type(q, (BF16, FP16), "q")
    ct = _type(k_cache, (qt, FP8), "k_cache")
    if q.requires_grad or k_cache.requires_grad or v_cache.requires_grad:
        _differentiable("q, k_cache or v_cache")
    if decode._forward._current_level >= 0:
        _no_tangents(q=q, k_cache=k_cache, v_cache=v_cache, out=out)
    k, v = _view(k_cache, "k_cache", dev), _view(v_cache, "v_cache", dev)
    N, H, ps, kd = k_cache.shape
    if not (v_cache.shape == k_cache.shape and v_cache.dtype == k_cache.dtype and kd == D):
        _bad(f"k_cache {tuple(k_cache.shape)} {k_cache.dtype}, v_cache {tuple(v_cache.shape)} {v_cache.dtype}, head_dim {D}")
    if H == 0 or heads % H:
        _bad(f"{heads} heads over {H} of the cache")
    tab, tab_stride = _table(table, "table", dev)
    S, P = table.shape
    if not (0 <= window < 2 ** 30 and 0 <= sinks < 2 ** 30):
        _bad(f"window {window}, sinks {sinks}")
    # (no heads: nothing to read or write)
    cfg = _pack(_CHUNK_CONFIG, ABI_VERSION, qt, ct, S, T if heads else 0, H, heads // H or 1, D, ps, N, P, window, sinks,
                D ** -0.5 if scale is None else scale)
    given = out is not None
    if not given:
        out = q.new_empty(T, heads, D)
    elif not (out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.is_contiguous()):
        _bad("out: like q, dense")
    elif out.requires_grad:
        _differentiable("out")
    res = dict(out=out)
    l_ptr = 0
    if lse:
        res["lse"] = q.new_empty(T, heads, dtype=t.float32)
        l_ptr = res["lse"].data_ptr()
    io = _pack(_CHUNK_IO, q.data_ptr(), qs[0], qs[1], *k, *v, tab, tab_stride, _ints(lens, (S,), "lens", dev),
               _ints(offsets, (S + 1,), "offsets", dev), _scales(k_scale, H, "k_scale", dev),
               _scales(v_scale, H, "v_scale", dev), out.data_ptr(), l_ptr)
    need = _lib_attend_bytes(cfg)
    ws, ws_ptr = _workspace(need, table)
    _done(_lib_attend(cfg, io, ws_ptr, need, _marks(markers, dev), decode._raw_stream(dev.index)), "argus_prompt_attend")
    if given:
        decode._written((out,))
    return res


def rotary_frequencies(rotated: int, base: float = 10000.0, factor: float = 1.0, original: int | None = None,
                       slow: float = 1.0, fast: float = 32.0, device="cuda"):
    """Radians per token of the pairs of `rotated` elements (float64 [rotated / 2], as rotate_tokens
    takes them): base ** (-2 i / rotated).  For a context stretched by `factor` all of them are
    divided by it; with `original`, the length that a model was made for, those that turn `fast` times or
    more over it stay, those that turn `slow` times or less are divided, and the ones between are mixed
    in proportion."""
    t = _t()
    if not (rotated >= 2 and rotated % 2 == 0 and base > 0 and factor > 0 and 0 <= slow < fast):
        _bad(f"rotated {rotated} (even), base {base}, factor {factor}, slow {slow} below fast {fast}")
    i = t.arange(rotated // 2, dtype=t.float64)
    f = base ** (-2.0 * i / rotated)
    keep = 0.0 if original is None else ((original * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
    return (f * keep + f / factor * (1 - keep)).to(device)


def rotate_tokens(q, new_k, new_v, k_cache, v_cache, table, starts, frequencies, offsets=None, interleaved: bool = False,
                  amplitude: float = 1.0, k_scale=None, v_scale=None, out=None, markers=None, stream=None) -> dict:
    """Rotary positions of new tokens: queries turned, keys turned and written with the values into
    their pages.

    q: [rows, heads, head_dim], new_k, new_v: [rows, kv_heads, head_dim], bf16 or fp16,
    contiguous rows; caches, table, starts, offsets and scales as in append_tokens: row r of sequence s has
    position starts[s] + r - offsets[s], an offset outside the rows taken as the nearer end.  frequencies: float64 [pairs], radians per token; the first 2 * pairs
    elements of a head turn, pair i of elements i and i + pairs, or (interleaved) 2 i and 2 i + 1; `amplitude`
    multiplies them.  q may be None (keys and values alone), or new_k, new_v, k_cache, v_cache and
    table (queries alone).  Returns out (like q; q itself may be given), without q nothing.  Rows of no sequence
    are not written; a row whose place is not held has its query turned alone."""
    t = _t()
    some = q if q is not None else new_k
    if some is None:
        _bad("neither queries nor keys")
    dev = some.device
    if _elsewhere(stream, dev):
        with _on(stream, dev, q, new_k, new_v, k_cache, v_cache, table, starts, frequencies, offsets, k_scale, v_scale, out,
                 _buffer(markers)):
            return rotate_tokens(q, new_k, new_v, k_cache, v_cache, table, starts, frequencies, offsets, interleaved,
                                 amplitude, k_scale, v_scale, out, markers)
    st = _type(some, (BF16, FP16), "q" if q is not None else "new_k")
    T, _, D = some.shape if some.dim() == 3 else _bad("q, new_k, new_v: [rows, heads, head_dim]")
    if starts.dim() != 1:
        _bad("starts: int32 [seqs]")
    S, heads, H, ps, N, P, ct = starts.shape[0], 0, 0, 0, 0, 0, st
    if not (frequencies.dtype == t.float64 and frequencies.dim() == 1 and frequencies.device == dev and frequencies.is_contiguous()):
        _bad(f"frequencies: float64 [pairs], dense, on {dev}")
    if frequencies.requires_grad:
        _differentiable("frequencies")
    if decode._forward._current_level >= 0:
        _no_tangents(q=q, new_k=new_k, new_v=new_v, k_cache=k_cache, v_cache=v_cache, frequencies=frequencies, out=out)
    q_part = o_part = (0, 0, 0)
    given = out is not None
    if q is not None:
        qs = _rows(q, "q", dev)
        if q.requires_grad:
            _differentiable("q")
        heads = q.shape[1]
        if not given:
            out, os_ = q.new_empty(T, heads, D), (heads * D, D)
        else:
            os_ = _rows(out, "out", dev)
            if not (out.shape == q.shape and out.dtype == q.dtype):
                _bad("out: like q")
            if out.requires_grad:
                _differentiable("out")
        q_part, o_part = (q.data_ptr(), qs[0], qs[1]), (out.data_ptr(), os_[0], os_[1])
    elif given:
        _bad("out without q")
    n_part, k, v, tab, scales = (0,) * 6, (0,) * 4, (0,) * 4, (0, 0), (0, 0)
    if new_k is not None:
        if new_v is None or k_cache is None or v_cache is None or table is None:
            _bad("new_k, new_v, k_cache, v_cache and table go together")
        ks, vs = _rows(new_k, "new_k", dev), _rows(new_v, "new_v", dev)
        k, v = _view(k_cache, "k_cache", dev), _view(v_cache, "v_cache", dev)
        N, H, ps, kd = k_cache.shape
        if new_k.requires_grad or new_v.requires_grad or k_cache.requires_grad or v_cache.requires_grad:
            _differentiable("new_k, new_v, k_cache or v_cache")
        ct = _type(k_cache, (st, FP8), "k_cache")
        if not (v_cache.shape == k_cache.shape and v_cache.dtype == k_cache.dtype and kd == D):
            _bad("k_cache and v_cache differ, or their head_dim from the rows'")
        if not (new_k.shape == (T, H, D) and new_v.shape == (T, H, D) and new_k.dtype == some.dtype and new_v.dtype == some.dtype):
            _bad(f"new_k {tuple(new_k.shape)} {new_k.dtype}, new_v {tuple(new_v.shape)} {new_v.dtype} for {T} rows and a cache of {H} heads of {D}")
        tab = _table(table, "table", dev)
        if table.shape[0] != S:
            _bad(f"table of {table.shape[0]} sequences, starts of {S}")
        P = table.shape[1]
        n_part = (new_k.data_ptr(), new_v.data_ptr(), ks[0], ks[1], vs[0], vs[1])
        scales = (_scales(k_scale, H, "k_scale", dev), _scales(v_scale, H, "v_scale", dev))
    elif not (new_v is None and k_cache is None and v_cache is None and table is None):
        _bad("new_k, new_v, k_cache, v_cache and table go together")
    cfg = _pack(_ROTATE_CONFIG, ABI_VERSION, st, ct, S, T, heads, H, D, frequencies.shape[0], 1 if interleaved else 0, ps, N, P,
                amplitude)
    io = _pack(_ROTATE_IO, *q_part, *o_part, *n_part, *k, *v, *tab, _ints(starts, (S,), "starts", dev),
               0 if offsets is None else _ints(offsets, (S + 1,), "offsets", dev), frequencies.data_ptr(), *scales)
    _done(_lib_rotate(cfg, io, _marks(markers, dev), decode._raw_stream(dev.index)), "argus_prompt_rotate")
    if new_k is not None:
        decode._written((k_cache, v_cache))
    if given:
        decode._written((out,))
    return dict(out=out) if q is not None else {}


def score_tokens(logits, tokens, top: int = 0, markers=None, stream=None) -> dict:
    """What a model's logits say of given tokens.

    logits: [rows, vocab] bf16, fp16 or fp32, contiguous rows; tokens: int32 [rows].  Returns
    logprobs (ln of the token's probability) and entropy (of the row's distribution, in nats), float32
    [rows]; ranks, int32 [rows]: how many tokens come before it (larger logits, or equal ones of lower
    tokens); with top (up to 64) the tokens that come first: top_logprobs float32 and top_tokens
    int32 [rows, top].  Logits of -inf are no alternatives: places left over have -1 and -inf.  A row with a NaN or
    +inf, or of -inf alone, has NaN, and -1 for ranks and tokens; a token outside the vocabulary has -inf and
    -1."""
    t = _t()
    dev = logits.device
    if _elsewhere(stream, dev):
        with _on(stream, dev, logits, tokens, _buffer(markers)):
            return score_tokens(logits, tokens, top, markers)
    lt = _type(logits, (BF16, FP16, FP32), "logits")
    ls = logits.stride()
    if not (len(ls) == 2 and (ls[1] == 1 or logits.shape[1] == 1)):
        _bad("logits: [rows, vocab], contiguous rows")
    R, V = logits.shape
    if logits.requires_grad:
        _differentiable("logits")
    if decode._forward._current_level >= 0:
        _no_tangents(logits=logits)
    if not 0 <= top <= MAX_TOP:
        _bad(f"top {top} (0..{MAX_TOP})")
    cfg = _pack(_SCORE_CONFIG, ABI_VERSION, lt, R, V, top, 0)
    chosen = _ints(tokens, (R,), "tokens", dev)
    logprobs = logits.new_empty(R, dtype=t.float32)
    out = dict(logprobs=logprobs, entropy=logprobs.new_empty(R), ranks=tokens.new_empty(R))
    best = (0, 0)
    if top:
        out["top_logprobs"], out["top_tokens"] = logprobs.new_empty(R, top), tokens.new_empty(R, top)
        best = (out["top_logprobs"].data_ptr(), out["top_tokens"].data_ptr())
    io = _pack(_SCORE_IO, logits.data_ptr(), ls[0], chosen, logprobs.data_ptr(), out["entropy"].data_ptr(),
               out["ranks"].data_ptr(), *best)
    need = _lib_score_bytes(cfg)
    ws, ws_ptr = _workspace(need, tokens)
    _done(_lib_score(cfg, io, ws_ptr, need, _marks(markers, dev), decode._raw_stream(dev.index)), "argus_prompt_score")
    return out
