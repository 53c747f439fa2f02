"""The operators of a prompt's pass without a GPU: the library exports what include/argus_prompt.h declares,
layouts agree, and bad arguments are refused with their codes before any HIP call."""
from __future__ import annotations

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "argus_prompt.h")
FAKE = 0x100000  # never read: every call fails its checks first


@pytest.fixture(scope="module")
def pr():
    from paper_2609_12299_amd import attr, prompt
    if not os.path.exists(attr.LIB_PATH):
        from paper_2609_12299_amd import build
        build.build()
    prompt._library()
    return prompt


def test_exports_every_declared_function(pr):
    names = sorted(set(re.findall(r"\b(argus_prompt_[a-z_]+)\s*\(", open(HEADER).read())))
    assert len(names) == 5
    import paper_2609_12299_amd as fw
    so = pr._library()
    for n in names:
        assert hasattr(so, n), n
        assert callable(getattr(fw, n)), f"{n} has no wrapper"


def test_regions(pr):
    text = open(HEADER).read()
    regions = re.findall(r"ARGUS_REGION_([A-Z_]+) = (\d+)", text)
    assert [int(i) for _, i in regions] == list(range(pr.NUM_REGIONS, pr.NUM_ALL_REGIONS))
    assert [n.lower().replace("_", ".") for n, _ in regions] == pr.PROMPT_REGION_NAMES
    assert re.search(r"ARGUS_NUM_ALL_REGIONS = (\d+)", text).group(1) == str(pr.NUM_ALL_REGIONS)
    assert len(set(pr.ALL_REGION_NAMES)) == pr.NUM_ALL_REGIONS


def test_struct_sizes_are_the_compilers(pr, tmp_path):
    """The sizes that the C compiler gives the structs of the header."""
    import subprocess
    names = ["chunk_config", "chunk_io", "rotate_config", "rotate_io", "score_config", "score_io"]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "argus_prompt.h"\nint main(void) {\n'
                   + "".join(f'  printf("{n} %zu\\n", sizeof(argus_{n}));\n' for n in names) + "  return 0;\n}\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines():
        n, s = line.split()
        assert ctypes.sizeof(getattr(pr, "argus_" + n)) == int(s), n


def test_packed_layouts_are_the_structures(pr):
    """What the wrappers pack as bytes is what the structures hold, field by field."""
    v1, v2 = pr.argus_page_view(1, 2, 3, 4), pr.argus_page_view(5, 6, 7, 8)
    flat = [1, 2, 3, 4, 5, 6, 7, 8]
    for layout, struct, packed, fields in (
            (pr._CHUNK_CONFIG, pr.argus_chunk_config, [*range(13), 0.25], None),
            (pr._CHUNK_IO, pr.argus_chunk_io, [11, -2, 3, *flat, *range(20, 28)], [11, -2, 3, v1, v2, *range(20, 28)]),
            (pr._ROTATE_CONFIG, pr.argus_rotate_config, [*range(13), 1.5], None),
            (pr._ROTATE_IO, pr.argus_rotate_io, [*range(12), *flat, *range(20, 27)], [*range(12), v1, v2, *range(20, 27)]),
            (pr._SCORE_CONFIG, pr.argus_score_config, [*range(6)], None),
            (pr._SCORE_IO, pr.argus_score_io, [*range(8)], None)):
        assert layout.pack(*packed) == bytes(struct(*(fields or packed))), struct
        assert layout.size == ctypes.sizeof(struct)


def view(pr, **kw):
    v = pr.argus_page_view(FAKE, 4096, 1024, 64)
    for k, x in kw.items():
        setattr(v, k, x)
    return v


# ---------------------------------------------------------------- attend

CHUNK = dict(abi_version=1, q_type=0, cache_type=0, seqs=4, rows=100, kv_heads=2, group=4, head_dim=64, page_size=16,
             num_pages=100, columns=512, window=0, sinks=0, scale=0.125)


def attend(pr, io_kw=None, ws=FAKE, room=None, markers=None, **kw):
    cfg = pr.argus_chunk_config(*{**CHUNK, **kw}.values())
    io = pr.argus_chunk_io(FAKE, 512, 64, view(pr), view(pr), FAKE, 512, FAKE, FAKE, None, None, FAKE, FAKE)
    for k, x in (io_kw or {}).items():
        setattr(io, k, x)
    need = pr.argus_prompt_attend_workspace_bytes(cfg)
    room = (need if need < 1 << 60 else 0) if room is None else room
    return pr.argus_prompt_attend(cfg, io, ws, room, markers, None)


@pytest.mark.parametrize("field,value,code", [
    ("abi_version", 2, -2), ("q_type", 2, -1), ("q_type", 3, -1), ("cache_type", 1, -1), ("cache_type", 2, -1),
    ("seqs", (1 << 20) + 1, -4), ("rows", 1 << 28, -4), ("kv_heads", 0, -1), ("kv_heads", 1025, -1), ("group", 0, -1),
    ("group", 257, -1), ("head_dim", 0, -1), ("head_dim", 12, -1), ("head_dim", 264, -1), ("head_dim", 136, -1),
    ("page_size", 4, -1), ("page_size", 24, -1), ("page_size", 131072, -1), ("num_pages", 0, -4), ("num_pages", 1 << 31, -4),
    ("columns", 0, -4), ("columns", 1 << 26, -4), ("window", 1 << 30, -4), ("sinks", 1 << 30, -4)])
def test_attend_refuses_configurations(pr, field, value, code):
    from paper_2609_12299_amd import argus_decode_last_error
    assert attend(pr, **{field: value}) == code
    assert argus_decode_last_error()
    assert pr.argus_prompt_attend_workspace_bytes(pr.argus_chunk_config(*{**CHUNK, field: value}.values())) == (1 << 64) - 1


def test_attend_refuses_head_sizes_of_eight_in_8_bits(pr):
    assert attend(pr, cache_type=pr.FP8, head_dim=72) == -1


@pytest.mark.parametrize("io,code", [
    (dict(d_q=None), -1), (dict(d_q=FAKE + 8), -3), (dict(q_row_stride=4), -3), (dict(q_head_stride=12), -3),
    (dict(d_table=None), -1), (dict(d_table=FAKE + 2), -3), (dict(table_stride=511), -1), (dict(d_lens=None), -1),
    (dict(d_lens=FAKE + 1), -3), (dict(d_offsets=None), -1), (dict(d_offsets=FAKE + 2), -3), (dict(d_out=None), -1),
    (dict(d_out=FAKE + 8), -3), (dict(d_k_scale=FAKE + 2), -3), (dict(d_v_scale=FAKE + 2), -3), (dict(d_lse=FAKE + 2), -3)])
def test_attend_refuses_pointers(pr, io, code):
    assert attend(pr, io) == code


@pytest.mark.parametrize("kw,code", [
    (dict(base=None), -1), (dict(base=FAKE + 8), -3), (dict(page_stride=4), -3), (dict(head_stride=4), -3),
    (dict(token_stride=68), -3), (dict(page_stride=-4096), -4), (dict(token_stride=-64), -4),
    (dict(token_stride=1 << 30), -4), (dict(page_stride=1 << 36), -4)])
def test_attend_refuses_views(pr, kw, code):
    assert attend(pr, dict(k=view(pr, **kw))) == code
    assert attend(pr, dict(v=view(pr, **kw))) == code


def test_attend_refuses_workspaces_and_markers(pr):
    long = dict(columns=1 << 20, rows=4, seqs=1)
    if pr.argus_prompt_attend_workspace_bytes(pr.argus_chunk_config(*{**CHUNK, **long}.values())):
        assert attend(pr, ws=None, **long) == -1
        assert attend(pr, ws=FAKE + 16, **long) == -3
        assert attend(pr, room=4096, **long) == -4
    assert attend(pr, markers=pr.argus_markers(FAKE, 3, 0, 0, 0)) == -4
    m = pr.argus_markers(FAKE, 1 << 30, (1 << 30) - 5, 0, 0)
    assert attend(pr, markers=m) == -4 and m.used == (1 << 30) - 5
    assert attend(pr, markers=pr.argus_markers(FAKE + 8, 1 << 30, 0, 0, 0)) == -1
    # (fewer regions would fit)
    assert attend(pr, markers=pr.argus_markers(FAKE, 1 << 30, 0, 0, 65536 - pr.NUM_ALL_REGIONS + 1)) == -1
    assert pr.argus_prompt_attend(None, None, None, 0, None, None) == -1


# ---------------------------------------------------------------- rotate

ROTATE = dict(abi_version=1, source_type=0, cache_type=0, seqs=4, rows=100, heads=8, kv_heads=2, head_dim=64, pairs=32,
              interleaved=0, page_size=16, num_pages=100, columns=512, amplitude=1.0)


def rotate(pr, io_kw=None, markers=None, **kw):
    cfg = pr.argus_rotate_config(*{**ROTATE, **kw}.values())
    io = pr.argus_rotate_io(FAKE, 512, 64, FAKE, 512, 64, FAKE, FAKE, 128, 64, 128, 64, view(pr), view(pr), FAKE, 512, FAKE, FAKE,
                            FAKE, None, None)
    for k, x in (io_kw or {}).items():
        setattr(io, k, x)
    return pr.argus_prompt_rotate(cfg, io, markers, None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=0), -2), (dict(source_type=2), -1), (dict(cache_type=1), -1), (dict(seqs=(1 << 20) + 1), -4),
    (dict(rows=1 << 24), -4), (dict(heads=65536), -1), (dict(kv_heads=1025), -1), (dict(heads=0, kv_heads=0), -1),
    (dict(head_dim=20), -1), (dict(head_dim=264), -1), (dict(cache_type=3, head_dim=72), -1), (dict(pairs=0), -1),
    (dict(pairs=33), -1), (dict(interleaved=2), -1), (dict(page_size=48), -1), (dict(num_pages=0), -4), (dict(columns=0), -4),
    (dict(columns=1 << 27), -4)])
def test_rotate_refuses_configurations(pr, kw, code):
    assert rotate(pr, **kw) == code


@pytest.mark.parametrize("io,code", [
    (dict(d_q=None), -1), (dict(d_out=None), -1), (dict(d_q=FAKE + 8), -3), (dict(d_out=FAKE + 8), -3), (dict(q_row_stride=4), -3),
    (dict(out_head_stride=2), -3), (dict(d_new_k=None), -1), (dict(d_new_v=None), -1), (dict(d_new_v=FAKE + 4), -3),
    (dict(k_row_stride=4), -3), (dict(v_head_stride=2), -3), (dict(d_table=None), -1), (dict(table_stride=1), -1),
    (dict(d_starts=None), -1), (dict(d_starts=FAKE + 1), -3), (dict(d_offsets=FAKE + 1), -3), (dict(d_offsets=None), -1),
    (dict(d_frequencies=None), -1), (dict(d_frequencies=FAKE + 4), -3), (dict(d_k_scale=FAKE + 1), -3)])
def test_rotate_refuses_pointers(pr, io, code):
    assert rotate(pr, io) == code


def test_rotate_refuses_views_and_markers(pr):
    assert rotate(pr, dict(k=view(pr, base=None))) == -1
    assert rotate(pr, dict(v=view(pr, token_stride=4))) == -3
    assert rotate(pr, markers=pr.argus_markers(FAKE, 3, 0, 0, 0)) == -4
    assert rotate(pr, markers=pr.argus_markers(FAKE, 1 << 30, 0, 0, 65536 - pr.NUM_ALL_REGIONS + 1)) == -1
    assert pr.argus_prompt_rotate(None, None, None, None) == -1


# ----------------------------------------------------------------- score

def score(pr, io_kw=None, ws=FAKE, room=1 << 20, markers=None, **kw):
    cfg = pr.argus_score_config(*{**dict(abi_version=1, type=0, rows=3, vocab=1000, top=5, pad=0), **kw}.values())
    io = pr.argus_score_io(FAKE, 1000, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE)
    for k, x in (io_kw or {}).items():
        setattr(io, k, x)
    return pr.argus_prompt_score(cfg, io, ws, room, markers, None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=9), -2), (dict(type=3), -1), (dict(rows=(1 << 22) + 1), -4), (dict(vocab=0), -1),
    (dict(vocab=(1 << 24) + 1), -1), (dict(top=65), -1)])
def test_score_refuses_configurations(pr, kw, code):
    assert score(pr, **kw) == code
    cfg = pr.argus_score_config(*{**dict(abi_version=1, type=0, rows=3, vocab=1000, top=5, pad=0), **kw}.values())
    assert pr.argus_prompt_score_workspace_bytes(cfg) == (1 << 64) - 1


@pytest.mark.parametrize("io,code", [
    (dict(d_logits=None), -1), (dict(d_logits=FAKE + 1), -3), (dict(d_tokens=None), -1), (dict(d_tokens=FAKE + 2), -3),
    (dict(d_logprobs=None), -1), (dict(d_entropy=None), -1), (dict(d_entropy=FAKE + 1), -3), (dict(d_ranks=None), -1),
    (dict(d_top_logprobs=None), -1), (dict(d_top_tokens=None), -1), (dict(d_top_tokens=FAKE + 2), -3)])
def test_score_refuses_pointers(pr, io, code):
    assert score(pr, io) == code


def test_score_refuses_workspaces_and_markers(pr):
    big = dict(rows=1, vocab=1 << 20)
    need = pr.argus_prompt_score_workspace_bytes(pr.argus_score_config(1, 0, 1, 1 << 20, 5, 0))
    assert need > 0
    assert score(pr, ws=None, **big) == -1 and score(pr, ws=FAKE + 128, **big) == -3 and score(pr, room=need - 1, **big) == -4
    assert score(pr, markers=pr.argus_markers(FAKE, 3, 0, 0, 0)) == -4
    assert score(pr, markers=pr.argus_markers(FAKE, 1 << 30, 0, 0, 65536 - pr.NUM_ALL_REGIONS + 1)) == -1
    assert pr.argus_prompt_score(None, None, None, 0, None, None) == -1
    # a workspace never depends on what device memory holds, and stays small
    for rows in (1, 3, 767, 768, 1 << 22):
        for top in (0, 1, 64):
            assert pr.argus_prompt_score_workspace_bytes(pr.argus_score_config(1, 0, rows, 1 << 24, top, 0)) < 1 << 23


# --------------------------------------------------------------- wrappers

def tensors():
    import torch
    q, c = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    one, two = torch.zeros(1, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32)
    return q, c, one, two, torch.zeros(1, 2, dtype=torch.int32), torch.ones(32, dtype=torch.float64)


def test_tensors_on_the_cpu_are_refused():
    import torch

    from paper_2609_12299_amd import ArgusError, attend_chunks, rotate_tokens, score_tokens
    q, c, one, two, tab, f = tensors()
    for call in (lambda: attend_chunks(q, c, c, tab, one, two), lambda: rotate_tokens(q, q[:, :2], q[:, :2], c, c, tab, one, f, two),
                 lambda: rotate_tokens(q, None, None, None, None, None, one, f, two),
                 lambda: score_tokens(torch.zeros(3, 50), torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ArgusError, match="on a GPU"):
            call()


def test_wrappers_check_what_the_c_side_cannot_see(monkeypatch):
    """Types, shapes, parts that go together, gradients: before any launch (tensors on the CPU here)."""
    import torch

    from paper_2609_12299_amd import ArgusError, attend_chunks, prompt, rotary_frequencies, rotate_tokens, score_tokens
    prompt._t()
    monkeypatch.setattr(prompt, "_elsewhere", lambda stream, dev: False)
    q, c, one, two, tab, f = tensors()
    k = q[:, :2]
    x, t = torch.zeros(3, 50), torch.zeros(3, dtype=torch.int32)
    for call in (
            lambda: attend_chunks(q[0], c, c, tab, one, two), lambda: attend_chunks(q.float(), c, c, tab, one, two),
            lambda: attend_chunks(q, c.half(), c.half(), tab, one, two), lambda: attend_chunks(q, c, c[:2], tab, one, two),
            lambda: attend_chunks(q[:, :3], c, c, tab, one, two), lambda: attend_chunks(q, c, c, tab.long(), one, two),
            lambda: attend_chunks(q, c, c, tab, two, two), lambda: attend_chunks(q, c, c, tab, one, one),
            lambda: attend_chunks(q, c, c, tab, one, two.long()), lambda: attend_chunks(q, c, c, tab, one, two, window=-1),
            lambda: attend_chunks(q, c, c, tab, one, two, out=torch.zeros(3, 4, 32, dtype=torch.bfloat16)),
            lambda: attend_chunks(q, c, c, tab, one, two, k_scale=torch.ones(3)),
            lambda: attend_chunks(q.clone().requires_grad_(), c, c, tab, one, two),
            lambda: rotate_tokens(None, None, None, None, None, None, one, f, two),
            lambda: rotate_tokens(q, k, None, c, c, tab, one, f, two), lambda: rotate_tokens(q, None, k, None, None, None, one, f, two),
            lambda: rotate_tokens(q, None, None, c, None, None, one, f, two), lambda: rotate_tokens(q, k, k, c, c, None, one, f, two),
            lambda: rotate_tokens(q, k, k, c, c, tab, one, f.float(), two), lambda: rotate_tokens(q, k, k[:2], c, c, tab, one, f, two),
            lambda: rotate_tokens(q, k.half(), k, c, c, tab, one, f, two), lambda: rotate_tokens(None, k, k, c, c, tab, one, f, two, out=q),
            lambda: rotate_tokens(q, k, k, c, c, tab, one, f, two, out=q.half()), lambda: rotate_tokens(q[0], k, k, c, c, tab, one, f, two),
            lambda: rotate_tokens(q, k, k, c, c, tab, one[:0], f, two), lambda: rotate_tokens(q, k, k.clone().requires_grad_(), c, c, tab, one, f, two),
            lambda: rotate_tokens(q, k, k, c, c, tab, one, f.clone().requires_grad_(), two),
            lambda: score_tokens(x[0], t), lambda: score_tokens(x.double(), t), lambda: score_tokens(x, t.long()),
            lambda: score_tokens(x, t[:2]), lambda: score_tokens(x, t, top=65), lambda: score_tokens(x, t, top=-1),
            lambda: score_tokens(x.t().contiguous().t(), t), lambda: score_tokens(x.clone().requires_grad_(), t),
            lambda: rotary_frequencies(7, device="cpu"), lambda: rotary_frequencies(8, factor=0.0, device="cpu"),
            lambda: rotary_frequencies(8, slow=3.0, fast=2.0, device="cpu")):
        with pytest.raises(ArgusError):
            call()


def test_frequencies_on_the_cpu():
    import torch

    from paper_2609_12299_amd import rotary_frequencies
    f = rotary_frequencies(8, device="cpu")
    assert f.dtype == torch.float64 and f.tolist() == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-14)
    assert rotary_frequencies(8, factor=4.0, device="cpu").tolist() == pytest.approx([0.25, 0.025, 0.0025, 0.00025], rel=1e-14)
