"""Decode-step operators without a GPU: the library exports what include/argus_decode.h declares,
layouts agree, and bad arguments are refused with their codes before any HIP call."""
from __future__ import annotations

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "argus_decode.h")
FAKE = 0x100000  # never read: every call fails its checks first


@pytest.fixture(scope="module")
def dec():
    from paper_2609_12299_amd import attr, decode
    if not os.path.exists(attr.LIB_PATH):
        from paper_2609_12299_amd import build
        build.build()
    decode._library()
    return decode


def test_exports_every_declared_function(dec):
    names = sorted(set(re.findall(r"\b(argus_decode_[a-z_]+)\s*\(", open(HEADER).read())))
    assert len(names) == 10
    so = dec._library()
    for n in names:
        assert hasattr(so, n), n
        assert callable(getattr(dec, n)), f"{n} has no wrapper"


def test_regions(dec):
    text = open(HEADER).read()
    regions = re.findall(r"ARGUS_REGION_([A-Z_]+) = (\d+)", text)
    assert [int(i) for _, i in regions] == list(range(len(regions)))
    assert [n.lower().replace("_", ".") for n, _ in regions] == dec.REGION_NAMES
    assert re.search(r"ARGUS_NUM_REGIONS = (\d+)", text).group(1) == str(dec.NUM_REGIONS)


def test_struct_sizes_are_the_compilers(dec, tmp_path):
    """The sizes that the C compiler gives the structs of the header."""
    import subprocess
    names = ["markers", "page_view", "attend_config", "attend_io", "append_config", "append_io", "page_planes",
             "step_config", "step_io", "compact_config", "compact_io", "select_config", "select_io"]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "argus_decode.h"\nint main(void) {\n'
                   + "".join(f'  printf("{n} %zu\\n", sizeof(argus_{n}));\n' for n in names) + "  return 0;\n}\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines():
        n, s = line.split()
        assert ctypes.sizeof(getattr(dec, "argus_" + n)) == int(s), n


def view(dec, **kw):
    v = dec.argus_page_view(FAKE, 4096, 1024, 64)
    for k, x in kw.items():
        setattr(v, k, x)
    return v


# ---------------------------------------------------------------- attend

def attend(dec, io_kw=None, ws=FAKE, room=None, markers=None, **kw):
    cfg = dec.argus_attend_config(1, dec.BF16, dec.BF16, 4, 2, 4, 64, 16, 100, 512, 0, 0, 0.125, 0)
    for k, x in kw.items():
        setattr(cfg, k, x)
    io = dec.argus_attend_io(FAKE, 512, 64, view(dec), view(dec), FAKE, 512, FAKE, None, None, FAKE, FAKE)
    for k, x in (io_kw or {}).items():
        setattr(io, k, x)
    need = dec.argus_decode_attend_workspace_bytes(cfg)
    room = (need if need < 1 << 60 else 0) if room is None else room
    return dec.argus_decode_attend(cfg, io, ws, room, markers, None)


@pytest.mark.parametrize("field,value,code", [
    ("abi_version", 2, -2), ("q_type", 2, -1), ("q_type", 3, -1), ("cache_type", 1, -1), ("cache_type", 2, -1),
    ("seqs", (1 << 20) + 1, -4), ("kv_heads", 0, -1), ("kv_heads", 1025, -1), ("group", 0, -1), ("group", 257, -1),
    ("head_dim", 0, -1), ("head_dim", 12, -1), ("head_dim", 264, -1), ("head_dim", 136, -1), ("page_size", 4, -1),
    ("page_size", 24, -1), ("page_size", 131072, -1), ("num_pages", 0, -4), ("num_pages", 1 << 31, -4),
    ("columns", 0, -4), ("columns", 1 << 27, -4), ("window", 1 << 31, -4), ("sinks", 1 << 31, -4)])
def test_attend_refuses_configurations(dec, field, value, code):
    assert attend(dec, **{field: value}) == code
    assert dec.argus_decode_last_error()
    cfg = dec.argus_attend_config(1, dec.BF16, dec.BF16, 4, 2, 4, 64, 16, 100, 512, 0, 0, 0.125, 0)
    setattr(cfg, field, value)
    assert dec.argus_decode_attend_workspace_bytes(cfg) == (1 << 64) - 1


def test_attend_refuses_head_sizes_of_eight_in_8_bits(dec):
    assert attend(dec, cache_type=dec.FP8, head_dim=72) == -1
    assert "multiple of 16" in dec.argus_decode_last_error()


@pytest.mark.parametrize("io,code", [
    (dict(d_q=None), -1), (dict(d_q=FAKE + 8), -3), (dict(q_seq_stride=4), -3), (dict(q_head_stride=12), -3),
    (dict(d_table=None), -1), (dict(d_table=FAKE + 2), -3), (dict(table_stride=511), -1), (dict(d_lens=None), -1),
    (dict(d_lens=FAKE + 1), -3), (dict(d_out=None), -1), (dict(d_out=FAKE + 8), -3), (dict(d_k_scale=FAKE + 2), -3),
    (dict(d_lse=FAKE + 2), -3)])
def test_attend_refuses_pointers(dec, io, code):
    assert attend(dec, io) == code


@pytest.mark.parametrize("kw,code", [
    (dict(base=None), -1), (dict(base=FAKE + 8), -3), (dict(page_stride=4), -3), (dict(head_stride=4), -3),
    (dict(token_stride=68), -3), (dict(page_stride=-4096), -4), (dict(token_stride=-64), -4),
    (dict(token_stride=1 << 30), -4), (dict(page_stride=1 << 36), -4)])
def test_attend_refuses_views(dec, kw, code):
    assert attend(dec, dict(k=view(dec, **kw))) == code
    assert attend(dec, dict(v=view(dec, **kw))) == code


def test_attend_refuses_workspaces_and_markers(dec):
    assert attend(dec, ws=None) == -1
    assert attend(dec, ws=FAKE + 16) == -3
    assert attend(dec, room=4096) == -4 and "workspace" in dec.argus_decode_last_error()
    assert attend(dec, markers=dec.argus_markers(FAKE, 10, 0, 0, 0)) == -4
    m = dec.argus_markers(FAKE, 1 << 30, (1 << 30) - 5, 0, 0)
    assert attend(dec, markers=m) == -4 and m.used == (1 << 30) - 5
    assert attend(dec, markers=dec.argus_markers(FAKE + 8, 1 << 30, 0, 0, 0)) == -1
    assert attend(dec, markers=dec.argus_markers(FAKE, 1 << 30, 0, 0, 65530)) == -1
    assert dec.argus_decode_attend(None, None, None, 0, None, None) == -1


def test_attend_workspace_sizes(dec):
    """None where a block takes a whole sequence; else by the shares, never by the lengths."""
    cfg = lambda **kw: dec.argus_attend_config(*[{**dict(v=1, q=0, c=0, seqs=4, h=2, g=4, d=64, ps=16, n=100, cols=32,
                                                       w=0, s=0, scale=1.0, pad=0), **kw}[k] for k in
                                                 ("v", "q", "c", "seqs", "h", "g", "d", "ps", "n", "cols", "w", "s", "scale", "pad")])
    size = lambda **kw: dec.argus_decode_attend_workspace_bytes(cfg(**kw))
    assert size() == 0 and size(cols=64) == 0 and size(cols=65) > 0 and size(cols=4096, w=400) == 0
    assert size(d=256) == 0 and size(cols=33, d=256) > 0
    most = 1024 * 2 * 32 * (128 + 2) * 4 + 1024 * 16 + 1024
    for seqs in (1, 7, 300, 1 << 20):
        for cols in (65, 4096, 1 << 26):
            assert 0 < size(seqs=seqs, cols=cols, g=32, d=128) <= most
    assert size(seqs=0, cols=4096) == 0


# ---------------------------------------------------------------- append

def append(dec, io_kw=None, **kw):
    cfg = dec.argus_append_config(1, dec.BF16, dec.BF16, 4, 2, 64, 16, 100, 512, 4)
    for k, x in kw.items():
        setattr(cfg, k, x)
    io = dec.argus_append_io(FAKE, FAKE, 128, 64, 128, 64, view(dec), view(dec), FAKE, 512, FAKE, None, None, None)
    for k, x in (io_kw or {}).items():
        setattr(io, k, x)
    return dec.argus_decode_append(cfg, io, None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=0), -2), (dict(source_type=2), -1), (dict(cache_type=1), -1), (dict(seqs=(1 << 20) + 1), -4),
    (dict(kv_heads=0), -1), (dict(head_dim=20), -1), (dict(head_dim=512), -1), (dict(cache_type=3, head_dim=72), -1),
    (dict(page_size=48), -1), (dict(num_pages=0), -4), (dict(columns=0), -4), (dict(rows=1 << 31), -4), (dict(rows=5), -1)])
def test_append_refuses_configurations(dec, kw, code):
    assert append(dec, **kw) == code


@pytest.mark.parametrize("io,code", [
    (dict(d_new_k=None), -1), (dict(d_new_v=None), -1), (dict(d_new_v=FAKE + 4), -3), (dict(k_row_stride=4), -3),
    (dict(v_head_stride=2), -3), (dict(d_table=None), -1), (dict(table_stride=1), -1), (dict(d_starts=None), -1),
    (dict(d_starts=FAKE + 1), -3), (dict(d_offsets=FAKE + 1), -3), (dict(d_k_scale=FAKE + 1), -3)])
def test_append_refuses_pointers(dec, io, code):
    assert append(dec, io) == code
    assert append(dec, dict(k=view(dec, base=None))) == -1
    assert append(dec, dict(v=view(dec, token_stride=4))) == -3


# ------------------------------------------------------------ step, compact

def step(dec, io_kw=None, ws=FAKE, room=None, cache=None, **kw):
    cfg = dec.argus_step_config(1, 4, 4, 32, 100, 16, 0, 0, 0 if cache is None else 1, 0)
    for k, x in kw.items():
        setattr(cfg, k, x)
    io = dec.argus_step_io(FAKE, 32, FAKE, FAKE, FAKE, FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE)
    if cache is not None:
        io.caches[0] = dec.argus_page_planes(*cache)
    for k, x in (io_kw or {}).items():
        setattr(io, k, x)
    if room is None:
        room = dec.argus_decode_step_workspace_bytes(4, 100)
    return dec.argus_decode_step(cfg, io, ws, room, None, None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=3), -2), (dict(old_seqs=(1 << 20) + 1), -4), (dict(new_seqs=(1 << 20) + 1), -4),
    (dict(num_pages=0), -4), (dict(num_pages=(1 << 28) + 1), -4), (dict(page_size=0), -1), (dict(page_size=12), -1),
    (dict(columns=0), -4), (dict(columns=1 << 27), -4), (dict(window=1 << 31), -4), (dict(num_caches=5), -1)])
def test_step_refuses_configurations(dec, kw, code):
    assert step(dec, **kw) == code


@pytest.mark.parametrize("io,code", [
    (dict(d_table=None), -1), (dict(d_lens=None), -1), (dict(d_new_table=None), -1), (dict(d_new_lens=None), -1),
    (dict(d_refs=None), -1), (dict(d_counters=None), -1), (dict(d_new_table=FAKE), -1), (dict(d_new_lens=FAKE), -1),
    (dict(d_refs=FAKE), -1), (dict(d_table=FAKE + 2), -3), (dict(d_refs=4 * FAKE + 1), -3), (dict(table_stride=31), -1)])
def test_step_refuses_pointers(dec, io, code):
    assert step(dec, io) == code


def test_step_refuses_the_rest(dec):
    assert step(dec, dict(d_parents=None), new_seqs=5, room=1 << 20) == -1
    assert step(dec, cache=(None, 1600, 16, 2, 16)) == -1
    assert step(dec, cache=(FAKE, 1600, 16, 0, 16)) == -1
    assert step(dec, cache=(FAKE, 1600, 16, 2, 8)) == -1
    assert step(dec, cache=(FAKE, 1600, 24, 2, 16)) == -3
    assert step(dec, cache=(FAKE + 8, 1600, 16, 2, 16)) == -3
    assert step(dec, ws=None) == -1 and step(dec, ws=FAKE + 4) == -3 and step(dec, room=100) == -4
    assert dec.argus_decode_step_workspace_bytes(1, 0) == (1 << 64) - 1
    assert dec.argus_decode_step_workspace_bytes(1, (1 << 28) + 1) == (1 << 64) - 1


def test_compact_refuses(dec):
    def compact(io_kw=None, ws=FAKE, room=1 << 20, **kw):
        cfg = dec.argus_compact_config(1, 4, 32, 100, 0, 0)
        for k, x in kw.items():
            setattr(cfg, k, x)
        io = dec.argus_compact_io(FAKE, 32, FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE)
        for k, x in (io_kw or {}).items():
            setattr(io, k, x)
        return dec.argus_decode_compact(cfg, io, ws, room, None, None)

    for kw, code in ((dict(abi_version=0), -2), (dict(seqs=(1 << 20) + 1), -4), (dict(columns=0), -4),
                     (dict(num_pages=0), -4), (dict(num_caches=9), -1)):
        assert compact(**kw) == code, kw
    for io, code in ((dict(d_table=None), -1), (dict(d_refs=None), -1), (dict(d_new_refs=None), -1),
                     (dict(d_map=None), -1), (dict(d_counters=None), -1), (dict(d_new_table=FAKE), -1),
                     (dict(d_new_refs=FAKE), -1), (dict(d_map=FAKE), -1), (dict(d_map=3 * FAKE), -1),
                     (dict(d_map=FAKE + 2), -3), (dict(table_stride=3), -1)):
        assert compact(io) == code, io
    assert compact(ws=None) == -1 and compact(ws=FAKE + 8) == -3 and compact(room=64) == -4
    assert dec.argus_decode_compact_workspace_bytes(0) == (1 << 64) - 1


# ----------------------------------------------------------------- select

def test_select_refuses(dec):
    def select(io_kw=None, ws=FAKE, room=1 << 20, **kw):
        cfg = dec.argus_select_config(1, dec.BF16, 2, 4, 1000, 4, -1, 0)
        for k, x in kw.items():
            setattr(cfg, k, x)
        io = dec.argus_select_io(FAKE, 4000, 1000, FAKE, FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE, 5 * FAKE)
        for k, x in (io_kw or {}).items():
            setattr(io, k, x)
        return dec.argus_decode_select(cfg, io, ws, room, None, None)

    for kw, code in ((dict(abi_version=9), -2), (dict(type=3), -1), (dict(beams=0), -1), (dict(beams=65), -1),
                     (dict(k=0), -1), (dict(k=65), -1), (dict(vocab=0), -1), (dict(vocab=(1 << 24) + 1), -1),
                     (dict(groups=(1 << 20) + 1), -4)):
        assert select(**kw) == code, kw
    for io, code in ((dict(d_logits=None), -1), (dict(d_logits=FAKE + 1), -3), (dict(d_scores=None), -1),
                     (dict(d_new_scores=None), -1), (dict(d_parents=None), -1), (dict(d_tokens=None), -1),
                     (dict(d_new_finished=None), -1), (dict(d_new_finished=FAKE), -1), (dict(d_new_scores=FAKE), -1),
                     (dict(d_tokens=4 * FAKE + 2), -3)):
        assert select(io) == code, io
    assert select(ws=None) == -1 and select(ws=FAKE + 128) == -3 and select(room=16) == -4


def test_wrappers_check_types_and_shapes():
    """What the C side cannot see is refused in Python, before any launch (tensors on the CPU here)."""
    import torch

    from paper_2609_12299_amd import ArgusError, MarkerBuffer, decode
    decode._t()
    dev = torch.device("cpu")
    i32 = torch.zeros(4, dtype=torch.int32)
    for bad in (i32.long(), i32[:3], torch.zeros(8, dtype=torch.int32)[::2]):
        with pytest.raises(ArgusError):
            decode._ints(bad, (4,), "x", dev)
    with pytest.raises(ArgusError):
        decode._table(torch.zeros(4, 4, dtype=torch.int32).t()[:, :3].t().t(), "t", dev)
    with pytest.raises(ArgusError):
        decode._type(torch.zeros(1, dtype=torch.float64), (0, 1), "q")
    with pytest.raises(ArgusError):
        decode._view(torch.zeros(2, 2, 8, 16).transpose(2, 3), "k", dev)
    with pytest.raises(ArgusError):
        decode._scales(torch.zeros(3), 2, "s", dev)
    out = (decode.argus_page_planes * 4)()
    pool = torch.zeros(2, 5, 3, 8, 16)
    decode._planes((pool, pool.transpose(3, 4)), 5, dev, out)
    assert out[0].page_bytes == 3 * 8 * 16 * 4 and out[0].planes == 2 and out[1].page_bytes == out[0].page_bytes
    for bad in (pool[:, :, :, :4], pool[:, :4], pool[0, 0], pool[:, :, ::2]):
        with pytest.raises(ArgusError):
            decode._planes((bad,), 5, dev, out)
    with pytest.raises(ArgusError):
        decode._planes((pool,) * 5, 5, dev, out)
    m = MarkerBuffer(100, ctx_base=7, region_base=20, device="cpu")
    assert m.used == 0 and m.records().shape == (0, 16)


def test_tensors_on_the_cpu_are_refused():
    import torch

    from paper_2609_12299_amd import ArgusError, append_tokens, attend_pages, compact_pages, select_beams, step_pages
    q, c = torch.zeros(1, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    one = torch.zeros(1, dtype=torch.int32)
    tab = torch.zeros(1, 2, dtype=torch.int32)
    for call in (lambda: attend_pages(q, c, c, tab, one), lambda: append_tokens(q[:, :2], q[:, :2], c, c, tab, one),
                 lambda: step_pages(tab, one, None, None, 16, num_pages=3), lambda: compact_pages(tab, one),
                 lambda: select_beams(torch.zeros(1, 2, 50), torch.zeros(1, 2), 2)):
        with pytest.raises(ArgusError, match="on a GPU"):
            call()


def test_launches_stay_within_their_limits(dec):
    """Calls of more threads than a launch can have: refused, or in another form."""
    many = dec.argus_append_config(dec.ABI_VERSION, 0, 0, 1, 1, 8, 8, 10, 10, 1 << 29)
    io = dec.argus_append_io(FAKE, FAKE, 8, 8, 8, 8, view(dec), view(dec), FAKE, 10, FAKE, FAKE, None, None)
    assert dec.argus_decode_append(many, io, None, None) == -4  # ARGUS_E_CAPACITY
    assert "rows" in dec.argus_decode_last_error()
    cfg = dec.argus_select_config(dec.ABI_VERSION, 0, 1 << 20, 64, 8, 1, -1, 0)
    assert dec.argus_decode_select_workspace_bytes(cfg) == (1 << 64) - 1
    cfg.beams = 32
    assert dec.argus_decode_select_workspace_bytes(cfg) < 1 << 40
    # 2^24 segments of one page: shared out, as a block for each would be too many
    a = dec.argus_attend_config(dec.ABI_VERSION, 0, 0, 1 << 20, 8, 1, 8, 8, 10, 1, 0, 0, 1.0, 0)
    assert dec.argus_decode_attend_workspace_bytes(a) == 0
    a.kv_heads = 16
    assert 0 < dec.argus_decode_attend_workspace_bytes(a) < 1 << 32


def test_page_bytes_beyond_32_bits():
    torch = pytest.importorskip("torch")
    from paper_2609_12299_amd import decode
    from paper_2609_12299_amd.attr import ArgusError
    out = (decode.argus_page_planes * decode.MAX_CACHES)()
    fine, wide = (torch.empty((1, 2, n), dtype=torch.uint8, device="meta") for n in ((1 << 32) - 16, 1 << 32))
    decode._planes([fine], 2, fine.device, out)
    assert out[0].page_bytes == (1 << 32) - 16
    with pytest.raises(ArgusError):
        decode._planes([wide], 2, wide.device, out)


def test_packed_layouts_are_the_structures(dec):
    """What the wrappers pack as bytes is what the structures hold, field by field."""
    view1, view2 = dec.argus_page_view(1, 2, 3, 4), dec.argus_page_view(5, 6, 7, 8)
    caches = dec._CACHES(*(dec.argus_page_planes(i + 1, 2, 3, 4, 5 + i) for i in range(dec.MAX_CACHES)))
    flat = [1, 2, 3, 4, 5, 6, 7, 8]
    for layout, struct, packed, fields in (
            (dec._ATTEND_CONFIG, dec.argus_attend_config, [*range(12), 0.25, 13], None),
            (dec._ATTEND_IO, dec.argus_attend_io, [11, -2, 3, *flat, *range(20, 27)], [11, -2, 3, view1, view2, *range(20, 27)]),
            (dec._APPEND_CONFIG, dec.argus_append_config, [*range(10)], None),
            (dec._APPEND_IO, dec.argus_append_io, [*range(6), *flat, *range(20, 26)], [*range(6), view1, view2, *range(20, 26)]),
            (dec._STEP_CONFIG, dec.argus_step_config, [*range(10)], None),
            (dec._STEP_IO, dec.argus_step_io, [*range(10), bytes(caches)], [*range(10), caches]),
            (dec._COMPACT_CONFIG, dec.argus_compact_config, [*range(6)], None),
            (dec._COMPACT_IO, dec.argus_compact_io, [*range(7), bytes(caches)], [*range(7), caches]),
            (dec._SELECT_CONFIG, dec.argus_select_config, [*range(6), -1, 7], None),
            (dec._SELECT_IO, dec.argus_select_io, [*range(9)], None)):
        assert layout.pack(*packed) == bytes(struct(*(fields or packed))), struct
        assert layout.size == ctypes.sizeof(struct)


def test_step_of_no_sequences_passes_its_checks(dec):
    """0 old and 0 new sequences, all tables NULL as empty tensors give them: only the workspace is refused."""
    none = dict.fromkeys(("d_table", "d_lens", "d_parents", "d_grow", "d_new_table", "d_new_lens"))
    for held in (None, FAKE):
        assert step(dec, dict(none, d_held=held), old_seqs=0, new_seqs=0, room=0) == -4
        assert "workspace" in dec.argus_decode_last_error()
    assert step(dec, dict(none, d_refs=FAKE), old_seqs=0, new_seqs=0, room=0) == -1


def test_streams_of_another_device_are_refused():
    """Such a stream cannot run the call, and another one in its place would not be what was asked for."""
    from types import SimpleNamespace

    import torch

    from paper_2609_12299_amd import ArgusError, decode
    decode._t()
    first, second = torch.device("cuda", 0), torch.device("cuda", 1)
    assert decode._elsewhere(SimpleNamespace(device=first), first)
    assert decode._elsewhere(SimpleNamespace(device=second), second)
    with pytest.raises(ArgusError, match="stream of cuda:1"):
        decode._elsewhere(SimpleNamespace(device=second), first)


def test_marker_buffers_of_another_device_are_refused():
    """The kernels of one device do not write into the memory of another, or of the host."""
    import torch

    from paper_2609_12299_amd import ArgusError, MarkerBuffer, decode
    m = MarkerBuffer(10, device="cpu")
    assert decode._marks(None, torch.device("cuda", 0)) is None
    assert decode._marks(m, torch.device("cpu")) is not None
    with pytest.raises(ArgusError, match="MarkerBuffer on cpu"):
        decode._marks(m, torch.device("cuda", 0))


def test_tensors_that_require_gradients_are_refused():
    """There is no backward pass: a result without history would be taken for one of constants."""
    import torch

    from paper_2609_12299_amd import ArgusError, decode
    decode._t()
    dev = torch.device("cpu")
    out = (decode.argus_page_planes * 4)()
    cache = torch.zeros(2, 2, 8, 16, dtype=torch.bfloat16, requires_grad=True)
    scale = torch.zeros(2, requires_grad=True)
    for call in (lambda: decode._differentiable("q"), lambda: decode._scales(scale, 2, "k_scale", dev),
                 lambda: decode._planes((cache,), 2, dev, out)):
        with pytest.raises(ArgusError, match="no_grad"):
            call()
        with torch.no_grad():
            call()
