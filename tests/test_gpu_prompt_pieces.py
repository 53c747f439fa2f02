"""Attention of chunks where the batch is planned: what the plan left, which rows were cut, and the answers, against
plain arithmetic in 64 bits. Through the C entry, so that the workspace can be looked at."""
from __future__ import annotations

import numpy as np
import pytest

import test_gpu_prompt_attend as attend
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def call(a, scale=None, window=0, sinks=0, k_scale=None, v_scale=None, markers=None):
    """argus_prompt_attend in a workspace of just the size that it asks for: (answers, the plan's head: pieces of a
    head, row tiles that are cut, steps of their pieces, those pieces; None without a plan)."""
    from paper_2609_12299_amd import prompt as pr
    q, k, v, table = a["q"], a["k_cache"], a["v_cache"], a["table"]
    T, heads, D = q.shape
    N, H, ps, _ = k.shape
    prompt_types = {torch.bfloat16: pr.BF16, torch.float16: pr.FP16, torch.float8_e4m3fn: pr.FP8}
    cfg = pr.argus_chunk_config(1, prompt_types[q.dtype], prompt_types[k.dtype], len(a["lens"]), T, H, heads // H, D, ps, N,
                                table.shape[1], window, sinks, D ** -0.5 if scale is None else scale)
    out = torch.empty((T, heads, D), dtype=q.dtype, device="cuda")
    lse = torch.empty((T, heads), dtype=torch.float32, device="cuda")
    views = [pr.argus_page_view(c.data_ptr(), c.stride(0), c.stride(1), c.stride(2)) for c in (k, v)]
    address = lambda x: None if x is None else x.data_ptr()  # noqa: E731
    io = pr.argus_chunk_io(q.data_ptr(), q.stride(0), q.stride(1), *views, table.data_ptr(), table.stride(0), address(a["lens"]),
                           address(a["offsets"]), address(k_scale), address(v_scale), address(out), address(lse))
    need = pr.argus_prompt_attend_workspace_bytes(cfg)
    room = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    ws = (room.data_ptr() + 255) & ~255
    rc = pr.argus_prompt_attend(cfg, io, ws if need else None, need, markers, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0
    at = ws - room.data_ptr()
    assert (room[:at] == 0xA5).all() and (room[at + need:] == 0xA5).all()  # nothing beside the workspace
    head = room[at:at + 32].cpu().numpy().view(np.uint64).tolist() if need else None
    return dict(out=out, lse=lse), head


def some_heads(a, got, heads, **kw):
    """Some key/value heads of the answers against the reference (which takes its time)."""
    H = a["k_cache"].shape[1]
    G = a["q"].shape[1] // H
    scale = {n: x for n, x in kw.items() if n in ("scale", "window", "sinks")}
    for h in heads:
        mine = slice(h * G, (h + 1) * G)
        part = {n: kw[n][h:h + 1] for n in ("k_scale", "v_scale") if kw.get(n) is not None}
        attend.check(dict(a, q=a["q"][:, mine], k_cache=a["k_cache"][:, h:h + 1], v_cache=a["v_cache"][:, h:h + 1]),
                     what=f"head {h}", got={n: x[:, mine] for n, x in got.items()}, **scale, **part)


KINDS = [("bf16", 128, False), ("bf16", 128, True), ("fp16", 96, True), ("fp8", 128, True), ("fp8", 96, False), ("bf16", 80, False),
         ("fp16", 128, False), ("half over fp8", 128, False), ("half over fp8", 96, False)]


def build(kind, **kw):
    a = attend.build("fp8" if kind == "half over fp8" else kind, **kw)
    if kind == "half over fp8":
        a["q"] = a["q"].half()
    H = a["k_cache"].shape[1]
    gen = torch.Generator(device="cuda").manual_seed(3)
    scales = {n: torch.rand(H, generator=gen, device="cuda") + 0.5 for n in ("k_scale", "v_scale")} if "fp8" in kind else {}
    return a, scales


def spoil(a, kind):
    """Pages that are not held, values that are not finite: some that all rows see, some that not all do."""
    N = a["k_cache"].shape[0]
    a["table"][0, 7:12] = -1
    a["table"][0, 40] = N
    a["table"][-1, 3:90:7] = -9
    v, tab = a["v_cache"].float(), a["table"]
    inf = float("inf") if "fp8" not in kind else float("nan")
    for s, j, d, x in ((0, 900, 3, inf), (0, 1010, 3, -inf), (0, 5, 9, float("nan")), (0, 1030, 70, -inf), (-1, 500, 1, inf)):
        n = int(a["lens"][s])
        if j < n and 0 <= int(tab[s, j // 16]) < N:
            v[tab[s, j // 16].long(), :, j % 16, d] = x
    a["v_cache"] = v.to(a["v_cache"].dtype)


def same_bits(x, y):
    return all(torch.equal(x[n].view(torch.uint8), y[n].view(torch.uint8)) for n in x)


@pytest.mark.parametrize("kind,D,spoiled", KINDS)
def test_many_row_tiles_in_a_plan(kind, D, spoiled):
    """256 rows a tile, none of them cut: a wide table over a modest length. And with a window wider than what goes
    without a plan."""
    a, scales = build(kind, D=D, G=1, H=128, ps=16, sizes=[(1101, 149)], columns=400)
    if spoiled:
        spoil(a, kind)
    for kw in ({}, dict(window=900, sinks=3), dict(window=2500, sinks=70)):
        got, head = call(a, **kw, **scales)
        assert (head is None) == (kw.get("window") == 900)
        assert head is None or head[:2] == [5, 0]  # (five tiles of 1101 rows; nine if they were of 128)
        some_heads(a, got, (61, 127) if kw.get("window") != 900 else (0,), **kw, **scales)


@pytest.mark.parametrize("kind,D,spoiled", KINDS)
def test_many_row_tiles_in_pieces(kind, D, spoiled):
    """256 rows a tile, those of one long context cut and joined."""
    a, scales = build(kind, D=D, G=1, H=64, ps=16, sizes=[(2101, 0), (30, 20003)])
    if spoiled:
        spoil(a, kind)
    for kw in ({}, dict(window=16001, sinks=5)):
        got, head = call(a, **kw, **scales)
        assert head[1] == 1 and head[3] >= 2 and head[0] == 9 + head[3], head
        some_heads(a, got, (40,) if kw else (0, 63), **kw, **scales)
        assert same_bits(got, call(a, **kw, **scales)[0])


@pytest.mark.parametrize("kind,D,G", [("bf16", 64, 4), ("half over fp8", 64, 3), ("fp16", 128, 8), ("bf16", 256, 2), ("half over fp8", 256, 1),
                                      ("fp8", 128, 5)])
def test_pieces_of_four_waves(kind, D, G):
    """128 rows a tile, cut: pages that are not held among the pieces, odd lengths, a piece that sees nothing."""
    a, scales = build(kind, D=D, G=G, H=2, ps=16, sizes=[(17, 20011), (1, 9001), (3, 0)])
    got, head = call(a, **scales)
    assert head[1] >= 1
    some_heads(a, got, (0, 1), **scales)
    a["table"][0, :700] = -1
    a["table"][1, 5::3] = -1
    got, head = call(a, **scales)
    some_heads(a, got, (0, 1), **scales)


def test_lengths_in_a_plan():
    """More row tiles than two rounds of blocks, of all lengths, some cut, with a window and a plan."""
    a = attend.build("fp16", D=96, G=1, H=4, ps=32, sizes=[(1, 97 * i % 3000) for i in range(260)] + [(2, 30000)], junk=False)
    for kw in (dict(window=2900, sinks=2), {}):
        got, head = call(a, **kw)
        assert head is not None and head[0] >= 261 and (head[1] > 0) == (not kw), head
        some_heads(a, got, (0, 3), **kw)
