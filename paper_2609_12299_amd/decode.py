"""Python binding of the decode-step operators (include/argus_decode.h).

The functions named ``argus_decode_*`` are one-to-one wrappers (argument
marshalling only).  The others take torch CUDA tensors: they check what the C
side cannot see (types, shapes, devices), allocate outputs and the workspace,
and enqueue on the current torch stream or the one given.  A stream that is given is
not made to wait for the current one, nor the current one for it: the order of their
work is the caller's, and what a call returns is valid once its stream has come that
far.  Every step of the computation runs in the HIP kernels of libargus_attr.so; there
is no fallback.  The operators have no backward pass: a tensor that requires gradients
is refused unless gradients are off (torch.no_grad), and one with a forward-mode tangent.
"""
from __future__ import annotations

import ctypes
import struct

from .attr import ABI_VERSION, ArgusError, load_library

BF16, FP16, FP32, FP8 = 0, 1, 2, 3
MAX_CACHES = 4
STEP_COUNTER_NAMES = ["needed", "short", "copied", "live", "bad_parents", "cut"]
COMPACT_COUNTER_NAMES = ["live", "moved"]
REGION_NAMES = ["attend", "attend.place", "attend.tokens", "attend.join", "append", "step.clear",
                "step.claim", "step.plan", "step.place", "compact.count", "compact.plan",
                "compact.move", "select.rows", "select.beams"]
NUM_REGIONS = len(REGION_NAMES)

_u32, _i32, _i64, _u64, _p = (ctypes.c_uint32, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64,
                              ctypes.c_void_p)


class argus_markers(ctypes.Structure):
    _fields_ = [("d_records", _p), ("capacity", _u64), ("used", _u64), ("ctx_base", _u32),
                ("region_base", _u32)]


class argus_page_view(ctypes.Structure):
    _fields_ = [("base", _p), ("page_stride", _i64), ("head_stride", _i64), ("token_stride", _i64)]


class argus_attend_config(ctypes.Structure):
    _fields_ = [(k, _u32) for k in ("abi_version", "q_type", "cache_type", "seqs", "kv_heads", "group",
                                    "head_dim", "page_size", "num_pages", "columns", "window", "sinks")]
    _fields_ += [("scale", ctypes.c_float), ("pad", _u32)]


class argus_attend_io(ctypes.Structure):
    _fields_ = [("d_q", _p), ("q_seq_stride", _i64), ("q_head_stride", _i64), ("k", argus_page_view),
                ("v", argus_page_view), ("d_table", _p), ("table_stride", _i64), ("d_lens", _p),
                ("d_k_scale", _p), ("d_v_scale", _p), ("d_out", _p), ("d_lse", _p)]


class argus_append_config(ctypes.Structure):
    _fields_ = [(k, _u32) for k in ("abi_version", "source_type", "cache_type", "seqs", "kv_heads",
                                    "head_dim", "page_size", "num_pages", "columns", "rows")]


class argus_append_io(ctypes.Structure):
    _fields_ = [("d_new_k", _p), ("d_new_v", _p), ("k_row_stride", _i64), ("k_head_stride", _i64),
                ("v_row_stride", _i64), ("v_head_stride", _i64), ("k", argus_page_view),
                ("v", argus_page_view), ("d_table", _p), ("table_stride", _i64), ("d_starts", _p),
                ("d_offsets", _p), ("d_k_scale", _p), ("d_v_scale", _p)]


class argus_page_planes(ctypes.Structure):
    _fields_ = [("base", _p), ("plane_stride", _i64), ("page_stride", _i64), ("planes", _u32),
                ("page_bytes", _u32)]


class argus_step_config(ctypes.Structure):
    _fields_ = [(k, _u32) for k in ("abi_version", "old_seqs", "new_seqs", "columns", "num_pages",
                                    "page_size", "window", "sinks", "num_caches", "pad")]


class argus_step_io(ctypes.Structure):
    _fields_ = [("d_table", _p), ("table_stride", _i64), ("d_lens", _p), ("d_parents", _p),
                ("d_grow", _p), ("d_held", _p), ("d_new_table", _p), ("d_new_lens", _p),
                ("d_refs", _p), ("d_counters", _p), ("caches", argus_page_planes * MAX_CACHES)]


class argus_compact_config(ctypes.Structure):
    _fields_ = [(k, _u32) for k in ("abi_version", "seqs", "columns", "num_pages", "num_caches", "pad")]


class argus_compact_io(ctypes.Structure):
    _fields_ = [("d_table", _p), ("table_stride", _i64), ("d_refs", _p), ("d_new_table", _p),
                ("d_new_refs", _p), ("d_map", _p), ("d_counters", _p),
                ("caches", argus_page_planes * MAX_CACHES)]


class argus_select_config(ctypes.Structure):
    _fields_ = [(k, _u32) for k in ("abi_version", "type", "groups", "beams", "vocab", "k")]
    _fields_ += [("eos", _i32), ("pad", _u32)]


class argus_select_io(ctypes.Structure):
    _fields_ = [("d_logits", _p), ("group_stride", _i64), ("beam_stride", _i64), ("d_scores", _p),
                ("d_finished", _p), ("d_new_scores", _p), ("d_parents", _p), ("d_tokens", _p),
                ("d_new_finished", _p)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        sz, mk = ctypes.c_size_t, ctypes.POINTER(argus_markers)
        for name, args in (("attend", [argus_attend_config, argus_attend_io, True]),
                           ("append", [argus_append_config, argus_append_io, False]),
                           ("step", [argus_step_config, argus_step_io, True]),
                           ("compact", [argus_compact_config, argus_compact_io, True]),
                           ("select", [argus_select_config, argus_select_io, True])):
            f = getattr(lib, "argus_decode_" + name)
            f.argtypes = [ctypes.POINTER(args[0]), ctypes.POINTER(args[1])]
            f.argtypes += ([_p, sz] if args[2] else []) + [mk, _p]
            f.restype = ctypes.c_int
        for name, args in (("attend", [ctypes.POINTER(argus_attend_config)]), ("step", [_u32, _u32]),
                           ("compact", [_u32]), ("select", [ctypes.POINTER(argus_select_config)])):
            f = getattr(lib, f"argus_decode_{name}_workspace_bytes")
            f.argtypes, f.restype = args, sz
        lib.argus_decode_last_error.argtypes = []
        lib.argus_decode_last_error.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def argus_decode_last_error() -> str:
    return _library().argus_decode_last_error().decode()


def argus_decode_attend_workspace_bytes(cfg) -> int:
    return _library().argus_decode_attend_workspace_bytes(cfg)


def argus_decode_attend(cfg, io, d_workspace, workspace_bytes, markers, stream) -> int:
    return _library().argus_decode_attend(cfg, io, d_workspace, workspace_bytes, markers, stream)


def argus_decode_append(cfg, io, markers, stream) -> int:
    return _library().argus_decode_append(cfg, io, markers, stream)


def argus_decode_step_workspace_bytes(new_seqs: int, num_pages: int) -> int:
    return _library().argus_decode_step_workspace_bytes(new_seqs, num_pages)


def argus_decode_step(cfg, io, d_workspace, workspace_bytes, markers, stream) -> int:
    return _library().argus_decode_step(cfg, io, d_workspace, workspace_bytes, markers, stream)


def argus_decode_compact_workspace_bytes(num_pages: int) -> int:
    return _library().argus_decode_compact_workspace_bytes(num_pages)


def argus_decode_compact(cfg, io, d_workspace, workspace_bytes, markers, stream) -> int:
    return _library().argus_decode_compact(cfg, io, d_workspace, workspace_bytes, markers, stream)


def argus_decode_select_workspace_bytes(cfg) -> int:
    return _library().argus_decode_select_workspace_bytes(cfg)


def argus_decode_select(cfg, io, d_workspace, workspace_bytes, markers, stream) -> int:
    return _library().argus_decode_select(cfg, io, d_workspace, workspace_bytes, markers, stream)


# ------------------------------------------------------------ torch wrappers
#
# A decode step's calls are short, and what the host does for one shows: the checks
# below cost one comparison each, messages are put together only where one fails,
# new tensors come from one at hand (new_empty: 1.4 us against 1.9), and the structures are
# packed as bytes (a configuration 0.2 us against 0.6, the rest of attend's 0.5 against 2.4).

_torch = None
_types = {}
_raw_stream = _device = _written = _forward = None
_lib_attend = _lib_attend_bytes = _lib_append = _lib_step = _lib_compact = _lib_select = _lib_select_bytes = None

# The structures of the header, field by field (native alignment).
_ATTEND_CONFIG, _ATTEND_IO = struct.Struct("12IfI"), struct.Struct("Q2q Q3q Q3q Qq 5Q")
_APPEND_CONFIG, _APPEND_IO = struct.Struct("10I"), struct.Struct("2Q4q Q3q Q3q Qq 4Q")
_CACHES = argus_page_planes * MAX_CACHES
_STEP_CONFIG, _STEP_IO = struct.Struct("10I"), struct.Struct("Qq 8Q %ds" % ctypes.sizeof(_CACHES))
_COMPACT_CONFIG, _COMPACT_IO = struct.Struct("6I"), struct.Struct("Qq 5Q %ds" % ctypes.sizeof(_CACHES))
_SELECT_CONFIG, _SELECT_IO = struct.Struct("6IiI"), struct.Struct("Q2q 6Q")


def _t():
    global _torch, _raw_stream, _device, _written, _forward, _lib_attend, _lib_attend_bytes, _lib_append, _lib_step, _lib_compact
    global _lib_select, _lib_select_bytes
    if _torch is None:
        import torch
        _types.update({torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32,
                       torch.float8_e4m3fn: FP8})
        # (the handle alone: a tenth of the time of a stream object)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda index: torch.cuda.current_stream(index).cuda_stream)
        _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        # (of tensors that a call writes in place, so that autograd sees it where it has kept them)
        _written = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)
        _forward = torch.autograd.forward_ad  # (its level is below 0 outside of forward-mode derivatives)
        lib = _library()

        def of(name, *types):
            f = lib["argus_decode_" + name]  # another object than the one with the structures' types
            f.argtypes, f.restype = [ctypes.c_char_p, *types], ctypes.c_int
            return f

        def bytes_of(name):
            f = of(name + "_workspace_bytes")
            f.restype = ctypes.c_size_t
            return f

        sz = ctypes.c_size_t
        _lib_attend, _lib_attend_bytes = of("attend", ctypes.c_char_p, _p, sz, _p, _p), bytes_of("attend")
        _lib_append = of("append", ctypes.c_char_p, _p, _p)
        _lib_step = of("step", ctypes.c_char_p, _p, sz, _p, _p)
        _lib_compact = of("compact", ctypes.c_char_p, _p, sz, _p, _p)
        _lib_select, _lib_select_bytes = of("select", ctypes.c_char_p, _p, sz, _p, _p), bytes_of("select")
        _torch = torch
    return _torch


def _bad(why: str):
    raise ArgusError(-1, why)


def _pack(layout, *fields) -> bytes:
    try:
        return layout.pack(*fields)
    except (struct.error, OverflowError):
        _bad(f"sizes or strides out of range: {fields}")


def _differentiable(name: str) -> None:
    if _torch.is_grad_enabled():
        _bad(f"{name} requires gradients, and there is no backward pass: detach it, or call under torch.no_grad()")


def _no_tangents(**tensors) -> None:
    """Within forward-mode derivatives: tensors with a tangent are refused, whose part in the results would be lost."""
    for name, x in tensors.items():
        if x is not None and _forward.unpack_dual(x).tangent is not None:
            _bad(f"{name} has a forward-mode tangent, and there is no derivative: unpack it first")


def _type(x, allowed, name: str) -> int:
    got = _types.get(x.dtype)
    if got not in allowed:
        _bad(f"{name}: type {x.dtype}")
    return got


def _ints(x, shape, name: str, dev) -> int:
    """Address of a dense int32 tensor of this shape on this device."""
    if not (x.dtype == _torch.int32 and x.shape == shape and x.device == dev and x.is_contiguous()):
        _bad(f"{name}: int32 {tuple(shape)}, dense, on {dev}; got {x.dtype} {tuple(x.shape)} on {x.device}")
    return x.data_ptr()


def _table(x, name: str, dev):
    st = x.stride()
    if not (x.dtype == _torch.int32 and len(st) == 2 and x.device == dev and (st[1] == 1 or x.shape[1] == 1)):
        _bad(f"{name}: int32 [sequences, columns] with contiguous rows on {dev}")
    return x.data_ptr(), st[0]


def _scales(x, heads: int, name: str, dev):
    if x is None:
        return 0
    if not (x.dtype == _torch.float32 and x.shape == (heads,) and x.device == dev and x.is_contiguous()):
        _bad(f"{name}: float32 [{heads}], dense, on {dev}")
    if x.requires_grad:
        _differentiable(name)
    if _forward._current_level >= 0:
        _no_tangents(**{name: x})
    return x.data_ptr()


def _view(c, name: str, dev) -> tuple:
    """Fields of an argus_page_view."""
    st = c.stride()
    if not (len(st) == 4 and c.device == dev and (st[3] == 1 or c.shape[3] == 1)):
        _bad(f"{name}: [pages, kv_heads, page_size, head_dim] with contiguous rows on {dev}")
    return c.data_ptr(), st[0], st[1], st[2]


def _planes(caches, num_pages: int, dev, out) -> None:
    if len(caches) > MAX_CACHES:
        _bad(f"at most {MAX_CACHES} caches")
    for i, c in enumerate(caches):
        st, shape, e = c.stride(), c.shape, c.element_size()
        if not (c.device == dev and len(shape) >= 3 and shape[1] == num_pages):
            _bad(f"caches[{i}]: [layers, {num_pages} pages, ...] on {dev}")
        if c.requires_grad:
            _differentiable(f"caches[{i}]")
        if _forward._current_level >= 0:
            _no_tangents(**{f"caches[{i}]": c})
        # a page is one run of memory, in whatever order its dimensions lie
        run = 1
        for step, n in sorted(zip(st[2:], shape[2:])):
            if n != 1:
                if step != run:
                    _bad(f"caches[{i}]: a page's elements do not lie in one run of memory")
                run *= n
        if run * e >= 1 << 32:
            _bad(f"caches[{i}]: a page of {run * e} bytes")
        p = out[i]
        p.base, p.plane_stride, p.page_stride = c.data_ptr(), st[0] * e, st[1] * e
        p.planes, p.page_bytes = shape[0], run * e


def _caches(caches, num_pages: int, dev) -> bytes:
    if len(caches) == 0:
        return b""
    out = _CACHES()
    _planes(caches, num_pages, dev, out)
    return bytes(out)


class MarkerBuffer:
    """Marker records that the operators write of their own regions: give it as
    `markers` to the calls of one stream, then `records()` to
    RegionAttribution(num_regions=region_base + NUM_REGIONS).run (NUM_ALL_REGIONS, where operators of a
    prompt's pass write too).  Contexts are waves, time is in ticks of 10 ns.  Four contexts (group_shift 2)
    are a block, save of a step that is one launch (few sequences and pages): its blocks have sixteen waves,
    four such groups each; and of a prompt's operators as their header says."""

    def __init__(self, capacity: int, ctx_base: int = 0, region_base: int = 0, device="cuda"):
        t = _t()
        self.buffer = t.empty((capacity, 16), dtype=t.uint8, device=device)
        self.c = argus_markers(self.buffer.data_ptr(), capacity, 0, ctx_base, region_base)

    @property
    def used(self) -> int:
        return int(self.c.used)

    def records(self):
        return self.buffer[:self.used]

    def clear(self) -> None:
        self.c.used = 0


class _on:
    """A call on another stream than the current one, or on another device: allocations belong to
    that stream, so that the allocator hands their memory on in its order, and the memory of
    the tensors that the call uses is not handed on before the stream is done with them."""

    def __init__(self, stream, dev, *used):
        t = _torch
        self.ctx = t.cuda.stream(stream) if stream is not None else t.cuda.device(dev)
        if stream is not None:
            for x in used:
                if x is not None and x.is_cuda:
                    x.record_stream(stream)

    def __enter__(self):
        return self.ctx.__enter__()

    def __exit__(self, *exc):
        return self.ctx.__exit__(*exc)


def _elsewhere(stream, dev) -> bool:
    """Whether the call leaves the current stream or device."""
    if dev.type != "cuda":
        _bad(f"tensors on a GPU, not on {dev}")
    if stream is None:
        return dev.index != _device()
    if stream.device != dev:
        _bad(f"a stream of {stream.device} for tensors on {dev}")
    return True


def _workspace(need: int, ints):
    """(tensor, address on 256 bytes); `ints`: an int32 tensor of the device."""
    if need == _NO_SIZE:
        raise ArgusError(-1, argus_decode_last_error())
    if need == 0:
        return None, None
    ws = ints.new_empty((need + 259) // 4)
    return ws, (ws.data_ptr() + 255) & ~255


_NO_SIZE = (1 << 64) - 1


def _done(rc: int, call: str) -> None:
    if rc != 0:
        raise ArgusError(rc, f"{call}: {argus_decode_last_error()}")


def _buffer(markers):
    return None if markers is None else markers.buffer


def _marks(markers, dev):
    if markers is None:
        return None
    if markers.buffer.device != dev:
        _bad(f"a MarkerBuffer on {markers.buffer.device} for tensors on {dev}")
    return ctypes.byref(markers.c)


def attend_pages(q, k_cache, v_cache, table, lens, scale: float | None = None, window: int = 0,
                 sinks: int = 0, k_scale=None, v_scale=None, lse: bool = False, out=None,
                 markers=None, stream=None) -> dict:
    """Attention of one new token per sequence over a paged cache.

    q: [seqs, heads, head_dim] bf16 or fp16, contiguous rows; k_cache, v_cache: [pages,
    kv_heads, page_size, head_dim] of q's type or float8_e4m3fn (any order of the first
    three dimensions in memory); table: int32 [seqs, columns]; lens: int32 [seqs], the
    new token included; k_scale, v_scale: float32 [kv_heads].  With a window, a
    sequence's last `window` and first `sinks` tokens are visible.  Entries of the
    table outside [0, pages) are pages that are not held: not visible.  Returns out
    (like q, dense) and, if asked, lse (float32 [seqs, heads]); a row that sees
    nothing answers zeros and -inf."""
    t = _t()
    dev = q.device
    if _elsewhere(stream, dev):
        with _on(stream, dev, q, k_cache, v_cache, table, lens, k_scale, v_scale, out, _buffer(markers)):
            return attend_pages(q, k_cache, v_cache, table, lens, scale, window, sinks, k_scale, v_scale, lse,
                                out, markers)
    qs = q.stride()
    if not (len(qs) == 3 and (qs[2] == 1 or q.shape[2] == 1)):
        _bad("q: [seqs, heads, head_dim], contiguous rows")
    S, heads, D = q.shape
    qt = _type(q, (BF16, FP16), "q")
    ct = _type(k_cache, (qt, FP8), "k_cache")
    if q.requires_grad or k_cache.requires_grad or v_cache.requires_grad:
        _differentiable("q, k_cache or v_cache")
    if _forward._current_level >= 0:
        _no_tangents(q=q, k_cache=k_cache, v_cache=v_cache, out=out)
    k, v = _view(k_cache, "k_cache", dev), _view(v_cache, "v_cache", dev)
    N, H, ps, kd = k_cache.shape
    if not (v_cache.shape == k_cache.shape and v_cache.dtype == k_cache.dtype and kd == D):
        _bad(f"k_cache {tuple(k_cache.shape)} {k_cache.dtype}, v_cache {tuple(v_cache.shape)} {v_cache.dtype}, head_dim {D}")
    if H == 0 or heads % H:
        _bad(f"{heads} heads over {H} of the cache")
    tab, tab_stride = _table(table, "table", dev)
    tS, P = table.shape
    if tS != S:
        _bad(f"table of {tS} sequences, q of {S}")
    if not (0 <= window < 2 ** 31 and 0 <= sinks < 2 ** 31):
        _bad(f"window {window}, sinks {sinks}")
    cfg = _pack(_ATTEND_CONFIG, ABI_VERSION, qt, ct, S, H, heads // H if heads else 1, D, ps, N, P, window, sinks,
                              D ** -0.5 if scale is None else scale, 0)
    given = out is not None
    if not given:
        out = q.new_empty((S, heads, D))
    elif not (out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.is_contiguous()):
        _bad("out: like q, dense")
    elif out.requires_grad:
        _differentiable("out")
    res = dict(out=out)
    l_ptr = 0
    if lse:
        res["lse"] = t.empty((S, heads), dtype=t.float32, device=dev)
        l_ptr = res["lse"].data_ptr()
    io = _pack(_ATTEND_IO, q.data_ptr(), qs[0], qs[1], *k, *v, tab, tab_stride, _ints(lens, (S,), "lens", dev),
               _scales(k_scale, H, "k_scale", dev), _scales(v_scale, H, "v_scale", dev), out.data_ptr(), l_ptr)
    need = _lib_attend_bytes(cfg)
    ws, ws_ptr = _workspace(need, table)
    _done(_lib_attend(cfg, io, ws_ptr, need, _marks(markers, dev), _raw_stream(dev.index)), "argus_decode_attend")
    if given:
        _written((out,))
    return res


def append_tokens(new_k, new_v, k_cache, v_cache, table, starts, offsets=None, k_scale=None,
                  v_scale=None, markers=None, stream=None) -> None:
    """Writes new tokens' keys and values into their pages.

    new_k, new_v: [rows, kv_heads, head_dim] bf16 or fp16, contiguous rows (views of a
    fused projection's result do); k_cache, v_cache: [pages, kv_heads, page_size,
    head_dim] of that type, or float8_e4m3fn, which takes x / scale[head] limited to
    +-448.  Row r of sequence s (offsets[s] <= r < offsets[s + 1]; without offsets one
    row per sequence) goes to position starts[s] + r - offsets[s]; rows without a held
    page are left out."""
    _t()
    dev = k_cache.device
    if _elsewhere(stream, dev):
        with _on(stream, dev, new_k, new_v, k_cache, v_cache, table, starts, offsets, k_scale, v_scale, _buffer(markers)):
            return append_tokens(new_k, new_v, k_cache, v_cache, table, starts, offsets, k_scale, v_scale, markers)
    ks, vs = new_k.stride(), new_v.stride()
    k, v = _view(k_cache, "k_cache", dev), _view(v_cache, "v_cache", dev)
    N, H, ps, D = k_cache.shape
    rows = new_k.shape[0]
    if not (len(ks) == len(vs) == 3 and (ks[2] == vs[2] == 1 or D == 1) and new_k.device == dev and new_v.device == dev):
        _bad(f"new_k, new_v: [rows, kv_heads, head_dim] with contiguous rows on {dev}")
    st = _type(new_k, (BF16, FP16), "new_k")
    if new_k.requires_grad or new_v.requires_grad or k_cache.requires_grad or v_cache.requires_grad:
        _differentiable("new_k, new_v, k_cache or v_cache")
    if _forward._current_level >= 0:
        _no_tangents(new_k=new_k, new_v=new_v, k_cache=k_cache, v_cache=v_cache)
    ct = _type(k_cache, (st, FP8), "k_cache")
    if not (v_cache.shape == k_cache.shape and v_cache.dtype == k_cache.dtype):
        _bad("k_cache and v_cache differ")
    if not (new_k.shape == (rows, H, D) and new_v.shape == (rows, H, D) and new_v.dtype == new_k.dtype):
        _bad(f"new_k {tuple(new_k.shape)}, new_v {tuple(new_v.shape)} for a cache of {H} heads of {D}")
    tab, tab_stride = _table(table, "table", dev)
    S, P = table.shape
    cfg = _pack(_APPEND_CONFIG, ABI_VERSION, st, ct, S, H, D, ps, N, P, rows)
    io = _pack(_APPEND_IO, new_k.data_ptr(), new_v.data_ptr(), ks[0], ks[1], vs[0], vs[1], *k, *v, tab,
               tab_stride, _ints(starts, (S,), "starts", dev),
               0 if offsets is None else _ints(offsets, (S + 1,), "offsets", dev),
               _scales(k_scale, H, "k_scale", dev), _scales(v_scale, H, "v_scale", dev))
    _done(_lib_append(cfg, io, _marks(markers, dev), _raw_stream(dev.index)), "argus_decode_append")
    _written((k_cache, v_cache))


def step_pages(table, lens, parents, grow, page_size: int, held=None, num_pages: int | None = None,
               caches=(), window: int = 0, sinks: int = 0, markers=None, stream=None) -> dict:
    """Page tables of one decode step from those of the last.

    New sequence s goes on from sequence parents[s] (-1: empty; None: itself) and gets
    room for grow[s] tokens (None: 0).  A page that a sequence would write on beside
    others is copied in every cache ([layers, pages, ...] tensors, a page of a layer in
    one run of memory); copies and growth take the free pages in ascending order;
    pages that a window has left behind are let go.  held: int32 [pages], holds that
    others have on pages (a prefix cache); without it num_pages or a cache gives the
    size of the pool.  Returns table [new, columns], lens [new], refs [pages] and
    counters [8] (STEP_COUNTER_NAMES), int32; an entry without a page is -1."""
    t = _t()
    dev = table.device
    if _elsewhere(stream, dev):
        with _on(stream, dev, table, lens, parents, grow, held, *caches, _buffer(markers)):
            return step_pages(table, lens, parents, grow, page_size, held, num_pages, caches, window, sinks, markers)
    if num_pages is None:
        if held is None and len(caches) == 0:
            _bad("num_pages, held or a cache gives the number of pages")
        num_pages = held.shape[0] if held is not None else caches[0].shape[1]
    N = num_pages
    tab, tab_stride = _table(table, "table", dev)
    S0, P = table.shape
    S = S0 if parents is None else parents.shape[0]
    if not (0 <= window < 2 ** 31 and 0 <= sinks < 2 ** 31 and 1 <= N <= 2 ** 28 and 0 < page_size <= 65536):
        _bad(f"window {window}, sinks {sinks}, num_pages {N}, page_size {page_size}")
    cfg = _pack(_STEP_CONFIG, ABI_VERSION, S0, S, P, N, page_size, window, sinks, len(caches), 0)
    new = table.new_empty
    out = dict(table=new((S, P)), lens=new(S), refs=new(N), counters=new(8))
    io = _pack(_STEP_IO, tab, tab_stride, _ints(lens, (S0,), "lens", dev),
               0 if parents is None else _ints(parents, (S,), "parents", dev),
               0 if grow is None else _ints(grow, (S,), "grow", dev),
               0 if held is None else _ints(held, (N,), "held", dev),
               out["table"].data_ptr(), out["lens"].data_ptr(), out["refs"].data_ptr(),
               out["counters"].data_ptr(), _caches(caches, N, dev))
    need = argus_decode_step_workspace_bytes(S, N)
    ws, ws_ptr = _workspace(need, table)
    _done(_lib_step(cfg, io, ws_ptr, need, _marks(markers, dev), _raw_stream(dev.index)), "argus_decode_step")
    _written(caches)
    return out


def compact_pages(table, refs, caches=(), markers=None, stream=None) -> dict:
    """Moves the pages with refs > 0 to the front of the pool, in every cache ([layers,
    pages, ...] tensors).  Returns table, refs, map (int32 [pages]: a page's new number,
    -1 for a free one) and counters (COMPACT_COUNTER_NAMES)."""
    t = _t()
    dev = table.device
    if _elsewhere(stream, dev):
        with _on(stream, dev, table, refs, *caches, _buffer(markers)):
            return compact_pages(table, refs, caches, markers)
    tab, tab_stride = _table(table, "table", dev)
    S, P = table.shape
    N = refs.shape[0]
    if not 1 <= N <= 2 ** 28:
        _bad(f"{N} pages")
    cfg = _pack(_COMPACT_CONFIG, ABI_VERSION, S, P, N, len(caches), 0)
    new = table.new_empty
    out = dict(table=new((S, P)), refs=new(N), map=new(N), counters=new(8))
    io = _pack(_COMPACT_IO, tab, tab_stride, _ints(refs, (N,), "refs", dev), out["table"].data_ptr(),
               out["refs"].data_ptr(), out["map"].data_ptr(), out["counters"].data_ptr(), _caches(caches, N, dev))
    need = argus_decode_compact_workspace_bytes(N)
    ws, ws_ptr = _workspace(need, table)
    _done(_lib_compact(cfg, io, ws_ptr, need, _marks(markers, dev), _raw_stream(dev.index)), "argus_decode_compact")
    _written(caches)
    return out


def select_beams(logits, scores, k: int, finished=None, eos: int = -1, markers=None, stream=None) -> dict:
    """Beam search's selection: the k best of each group's beams and tokens.

    logits: [groups, beams, vocab] bf16, fp16 or fp32, contiguous rows; scores: float32
    [groups, beams]; finished: bool [groups, beams] or None: such a beam stands for
    itself, with token `eos`.  Returns scores float32, parents int32 (beams numbered over
    the whole batch, as step_pages takes them), tokens int32 and finished bool, [groups,
    k] each, in falling order of the score; places without a candidate have -inf, -1,
    -1, False."""
    t = _t()
    dev = logits.device
    if _elsewhere(stream, dev):
        with _on(stream, dev, logits, scores, finished, _buffer(markers)):
            return select_beams(logits, scores, k, finished, eos, markers)
    lt = _type(logits, (BF16, FP16, FP32), "logits")
    ls = logits.stride()
    if not (len(ls) == 3 and (ls[2] == 1 or logits.shape[2] == 1)):
        _bad("logits: [groups, beams, vocab], contiguous rows")
    G, W, V = logits.shape
    if not (scores.dtype == t.float32 and scores.shape == (G, W) and scores.device == dev and scores.is_contiguous()):
        _bad(f"scores: float32 {(G, W)}, dense, on {dev}")
    if logits.requires_grad or scores.requires_grad:
        _differentiable("logits or scores")
    if _forward._current_level >= 0:
        _no_tangents(logits=logits, scores=scores)
    done = 0
    if finished is not None:
        if not (finished.dtype in (t.bool, t.uint8) and finished.shape == (G, W) and finished.device == dev
                and finished.is_contiguous()):
            _bad(f"finished: bool {(G, W)}, dense, on {dev}")
        done = finished.data_ptr()
    if not (0 < k <= 64 and -2 ** 31 <= eos < 2 ** 31):
        _bad(f"k {k} (1..64), eos {eos}")
    cfg = _pack(_SELECT_CONFIG, ABI_VERSION, lt, G, W, V, k, eos, 0)
    shape = (G, k)
    parents = t.empty(shape, dtype=t.int32, device=dev)
    out = dict(scores=scores.new_empty(shape), parents=parents, tokens=parents.new_empty(shape),
               finished=t.empty(shape, dtype=t.bool, device=dev))
    io = _pack(_SELECT_IO, logits.data_ptr(), ls[0], ls[1], scores.data_ptr(), done, out["scores"].data_ptr(),
               parents.data_ptr(), out["tokens"].data_ptr(), out["finished"].data_ptr())
    need = _lib_select_bytes(cfg)
    ws, ws_ptr = _workspace(need, parents)
    _done(_lib_select(cfg, io, ws_ptr, need, _marks(markers, dev), _raw_stream(dev.index)), "argus_decode_select")
    return out
