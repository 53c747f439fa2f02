"""Python binding of the decode-step operators (include/argus_decode.h).

The functions named ``argus_decode_*`` are one-to-one wrappers (argument
marshalling only).  The others take torch CUDA tensors: they check what the C
side cannot see (types, shapes, devices), allocate outputs and the workspace,
and enqueue on the current torch stream or the one given.  Every step of the
computation runs in the HIP kernels of libargus_attr.so; there is no fallback.
"""
from __future__ import annotations

import ctypes

from .attr import ABI_VERSION, ArgusError, load_library

BF16, FP16, FP32, FP8 = 0, 1, 2, 3
MAX_CACHES = 4
NUM_COUNTERS_STEP = 8
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

_torch = None
_types = {}


def _t():
    global _torch
    if _torch is None:
        import torch
        _types.update({torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32,
                       torch.float8_e4m3fn: FP8})
        _torch = torch
    return _torch


def _need(ok: bool, why: str) -> None:
    if not ok:
        raise ArgusError(-1, why)


def _type(x, allowed, name: str) -> int:
    got = _types.get(x.dtype)
    _need(got in allowed, f"{name}: type {x.dtype}")
    return got


def _ints(x, shape, name: str, dev) -> int:
    """Address of a dense int32 tensor of this shape on this device."""
    t = _torch
    _need(x.dtype == t.int32 and x.shape == shape and x.device == dev and x.is_contiguous(),
          f"{name}: int32 {tuple(shape)}, dense, on {dev}; got {x.dtype} {tuple(x.shape)} on {x.device}")
    return x.data_ptr()


def _table(x, name: str, dev):
    _need(x.dtype == _torch.int32 and x.dim() == 2 and x.device == dev and (x.stride(1) == 1 or x.shape[1] == 1),
          f"{name}: int32 [sequences, columns] with contiguous rows on {dev}")
    return x.data_ptr(), x.stride(0)


def _scales(x, heads: int, name: str, dev):
    if x is None:
        return None
    _need(x.dtype == _torch.float32 and x.shape == (heads,) and x.device == dev and x.is_contiguous(),
          f"{name}: float32 [{heads}], dense, on {dev}")
    return x.data_ptr()


def _view(c, name: str, dev) -> argus_page_view:
    _need(c.dim() == 4 and c.device == dev and (c.stride(3) == 1 or c.shape[3] == 1),
          f"{name}: [pages, kv_heads, page_size, head_dim] with contiguous rows on {dev}")
    st = c.stride()
    return argus_page_view(c.data_ptr(), st[0], st[1], st[2])


def _planes(caches, num_pages: int, dev):
    _need(len(caches) <= MAX_CACHES, f"at most {MAX_CACHES} caches")
    out = (argus_page_planes * MAX_CACHES)()
    for i, c in enumerate(caches):
        _need(c.device == dev and c.dim() >= 3 and c.shape[1] == num_pages,
              f"caches[{i}]: [layers, {num_pages} pages, ...] on {dev}")
        e = c.element_size()
        one = c[0, 0] if c.shape[0] else c
        # a page is one run of memory, in whatever order its dimensions lie
        run = 1
        for st, n in sorted(zip(one.stride(), one.shape)):
            if n != 1:
                _need(st == run, f"caches[{i}]: a page's elements do not lie in one run of memory")
                run *= n
        out[i] = argus_page_planes(c.data_ptr(), c.stride(0) * e, c.stride(1) * e, c.shape[0], run * e)
    return out


class MarkerBuffer:
    """Marker records that the operators write of their own regions: give it as
    `markers` to the calls of one stream, then `records()` to
    RegionAttribution(num_regions=region_base + NUM_REGIONS).run.  Contexts are waves
    (group_shift 2: blocks), time is in ticks of 10 ns."""

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
    """The stream of a call: allocations belong to it, so that the allocator hands their memory on in
    its order."""

    def __init__(self, stream, dev):
        self.dev, self.stream, self.ctx = dev, stream, None

    def __enter__(self):
        t = _torch
        cur = t.cuda.current_stream(self.dev)
        if self.stream is not None and self.stream != cur:
            self.ctx = t.cuda.stream(self.stream)
            self.ctx.__enter__()
            cur = self.stream
        elif self.dev.index is not None and self.dev.index != t.cuda.current_device():
            self.ctx = t.cuda.device(self.dev)
            self.ctx.__enter__()
        return cur.cuda_stream

    def __exit__(self, *exc):
        if self.ctx is not None:
            self.ctx.__exit__(*exc)


def _workspace(need: int, dev):
    """(tensor, address): 256-byte aligned, as the allocator's blocks are."""
    if need == (1 << 64) - 1:
        raise ArgusError(-1, argus_decode_last_error())
    if need == 0:
        return None, None
    ws = _torch.empty(need + 256, dtype=_torch.uint8, device=dev)
    return ws, (ws.data_ptr() + 255) & ~255


def _done(rc: int, call: str) -> None:
    if rc != 0:
        raise ArgusError(rc, f"{call}: {argus_decode_last_error()}")


def _marks(markers):
    return None if markers is None else ctypes.byref(markers.c)


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
    _need(q.dim() == 3 and (q.stride(2) == 1 or q.shape[2] == 1), "q: [seqs, heads, head_dim], contiguous rows")
    S, heads, D = q.shape
    qt = _type(q, (BF16, FP16), "q")
    ct = _type(k_cache, (qt, FP8), "k_cache")
    k, v = _view(k_cache, "k_cache", dev), _view(v_cache, "v_cache", dev)
    N, H, ps, _ = k_cache.shape
    _need(v_cache.shape == k_cache.shape and v_cache.dtype == k_cache.dtype and k_cache.shape[3] == D,
          f"k_cache {tuple(k_cache.shape)} {k_cache.dtype}, v_cache {tuple(v_cache.shape)} {v_cache.dtype}, head_dim {D}")
    _need(H > 0 and heads % H == 0, f"{heads} heads over {H} of the cache")
    tab, tab_stride = _table(table, "table", dev)
    _need(table.shape[0] == S, f"table of {table.shape[0]} sequences, q of {S}")
    _need(0 <= window < 2 ** 31 and 0 <= sinks < 2 ** 31, f"window {window}, sinks {sinks}")
    cfg = argus_attend_config(ABI_VERSION, qt, ct, S, H, heads // H if heads else 1, D, ps, N, table.shape[1],
                              int(window), int(sinks), D ** -0.5 if scale is None else float(scale), 0)
    with _on(stream, dev) as s:
        if out is None:
            out = t.empty((S, heads, D), dtype=q.dtype, device=dev)
        else:
            _need(out.shape == q.shape and out.dtype == q.dtype and out.device == dev and out.is_contiguous(),
                  "out: like q, dense")
        res = dict(out=out)
        if lse:
            res["lse"] = t.empty((S, heads), dtype=t.float32, device=dev)
        need = argus_decode_attend_workspace_bytes(cfg)
        ws, ws_ptr = _workspace(need, dev)
        io = argus_attend_io(q.data_ptr(), q.stride(0), q.stride(1), k, v, tab, tab_stride,
                             _ints(lens, (S,), "lens", dev), _scales(k_scale, H, "k_scale", dev),
                             _scales(v_scale, H, "v_scale", dev), out.data_ptr(),
                             res["lse"].data_ptr() if lse else None)
        _done(argus_decode_attend(cfg, io, ws_ptr, need, _marks(markers), s), "argus_decode_attend")
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
    t = _t()
    dev = k_cache.device
    for x, name in ((new_k, "new_k"), (new_v, "new_v")):
        _need(x.dim() == 3 and x.device == dev and (x.stride(2) == 1 or x.shape[2] == 1),
              f"{name}: [rows, kv_heads, head_dim] with contiguous rows on {dev}")
    st = _type(new_k, (BF16, FP16), "new_k")
    ct = _type(k_cache, (st, FP8), "k_cache")
    k, v = _view(k_cache, "k_cache", dev), _view(v_cache, "v_cache", dev)
    N, H, ps, D = k_cache.shape
    rows = new_k.shape[0]
    _need(v_cache.shape == k_cache.shape and v_cache.dtype == k_cache.dtype, "k_cache and v_cache differ")
    _need(new_k.shape == (rows, H, D) and new_v.shape == (rows, H, D) and new_v.dtype == new_k.dtype,
          f"new_k {tuple(new_k.shape)}, new_v {tuple(new_v.shape)} for a cache of {H} heads of {D}")
    tab, tab_stride = _table(table, "table", dev)
    S = table.shape[0]
    cfg = argus_append_config(ABI_VERSION, st, ct, S, H, D, ps, N, table.shape[1], rows)
    ks, vs = new_k.stride(), new_v.stride()
    io = argus_append_io(new_k.data_ptr(), new_v.data_ptr(), ks[0], ks[1], vs[0], vs[1], k, v, tab,
                         tab_stride, _ints(starts, (S,), "starts", dev),
                         None if offsets is None else _ints(offsets, (S + 1,), "offsets", dev),
                         _scales(k_scale, H, "k_scale", dev), _scales(v_scale, H, "v_scale", dev))
    with _on(stream, dev) as s:
        _done(argus_decode_append(cfg, io, _marks(markers), s), "argus_decode_append")


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
    if num_pages is None:
        _need(held is not None or len(caches) > 0, "num_pages, held or a cache gives the number of pages")
        num_pages = held.shape[0] if held is not None else caches[0].shape[1]
    N = int(num_pages)
    tab, tab_stride = _table(table, "table", dev)
    S0, P = table.shape
    S = S0 if parents is None else parents.shape[0]
    _need(0 <= window < 2 ** 31 and 0 <= sinks < 2 ** 31, f"window {window}, sinks {sinks}")
    _need(1 <= N <= 2 ** 28 and 0 < page_size <= 65536, f"num_pages {N}, page_size {page_size}")
    cfg = argus_step_config(ABI_VERSION, S0, S, P, N, int(page_size), int(window), int(sinks), len(caches), 0)
    with _on(stream, dev) as s:
        out = dict(table=t.empty((S, P), dtype=t.int32, device=dev), lens=t.empty(S, dtype=t.int32, device=dev),
                   refs=t.empty(N, dtype=t.int32, device=dev),
                   counters=t.empty(NUM_COUNTERS_STEP, dtype=t.int32, device=dev))
        io = argus_step_io(tab, tab_stride, _ints(lens, (S0,), "lens", dev),
                           None if parents is None else _ints(parents, (S,), "parents", dev),
                           None if grow is None else _ints(grow, (S,), "grow", dev),
                           None if held is None else _ints(held, (N,), "held", dev),
                           out["table"].data_ptr(), out["lens"].data_ptr(), out["refs"].data_ptr(),
                           out["counters"].data_ptr(), _planes(caches, N, dev))
        need = argus_decode_step_workspace_bytes(S, N)
        ws, ws_ptr = _workspace(need, dev)
        _done(argus_decode_step(cfg, io, ws_ptr, need, _marks(markers), s), "argus_decode_step")
    return out


def compact_pages(table, refs, caches=(), markers=None, stream=None) -> dict:
    """Moves the pages with refs > 0 to the front of the pool, in every cache ([layers,
    pages, ...] tensors).  Returns table, refs, map (int32 [pages]: a page's new number,
    -1 for a free one) and counters (COMPACT_COUNTER_NAMES)."""
    t = _t()
    dev = table.device
    tab, tab_stride = _table(table, "table", dev)
    S, P = table.shape
    N = refs.shape[0]
    _need(1 <= N <= 2 ** 28, f"{N} pages")
    cfg = argus_compact_config(ABI_VERSION, S, P, N, len(caches), 0)
    with _on(stream, dev) as s:
        out = dict(table=t.empty((S, P), dtype=t.int32, device=dev), refs=t.empty(N, dtype=t.int32, device=dev),
                   map=t.empty(N, dtype=t.int32, device=dev), counters=t.empty(8, dtype=t.int32, device=dev))
        io = argus_compact_io(tab, tab_stride, _ints(refs, (N,), "refs", dev), out["table"].data_ptr(),
                              out["refs"].data_ptr(), out["map"].data_ptr(), out["counters"].data_ptr(),
                              _planes(caches, N, dev))
        need = argus_decode_compact_workspace_bytes(N)
        ws, ws_ptr = _workspace(need, dev)
        _done(argus_decode_compact(cfg, io, ws_ptr, need, _marks(markers), s), "argus_decode_compact")
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
    lt = _type(logits, (BF16, FP16, FP32), "logits")
    _need(logits.dim() == 3 and (logits.stride(2) == 1 or logits.shape[2] == 1),
          "logits: [groups, beams, vocab], contiguous rows")
    G, W, V = logits.shape
    _need(scores.dtype == t.float32 and scores.shape == (G, W) and scores.device == dev and scores.is_contiguous(),
          f"scores: float32 {(G, W)}, dense, on {dev}")
    if finished is not None:
        _need(finished.dtype in (t.bool, t.uint8) and finished.shape == (G, W) and finished.device == dev
              and finished.is_contiguous(), f"finished: bool {(G, W)}, dense, on {dev}")
    _need(0 < k <= 64, f"k {k} (1..64)")
    _need(-2 ** 31 <= eos < 2 ** 31, f"eos {eos}")
    cfg = argus_select_config(ABI_VERSION, lt, G, W, V, int(k), int(eos), 0)
    with _on(stream, dev) as s:
        out = dict(scores=t.empty((G, k), dtype=t.float32, device=dev), parents=t.empty((G, k), dtype=t.int32, device=dev),
                   tokens=t.empty((G, k), dtype=t.int32, device=dev), finished=t.empty((G, k), dtype=t.bool, device=dev))
        io = argus_select_io(logits.data_ptr(), logits.stride(0), logits.stride(1), scores.data_ptr(),
                             None if finished is None else finished.data_ptr(), out["scores"].data_ptr(),
                             out["parents"].data_ptr(), out["tokens"].data_ptr(), out["finished"].data_ptr())
        need = argus_decode_select_workspace_bytes(cfg)
        ws, ws_ptr = _workspace(need, dev)
        _done(argus_decode_select(cfg, io, ws_ptr, need, _marks(markers), s), "argus_decode_select")
    return out
