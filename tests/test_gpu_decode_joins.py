"""Attention whose segments lie in many, some or few pieces: every form of the join, with pieces in which
no token is visible."""
from __future__ import annotations

import pytest

from gpu_util import log
from test_gpu_decode_attend import check, make, on_gpu

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# sequences, heads, query heads of each: one segment in hundreds of pieces; a few rows; many
SHAPES = [([20011], 1, 3), ([9000, 1], 1, 20), ([6000] * 3, 2, 5), ([2100] * 10, 2, 24), ([4000, 0, 77, 9000], 2, 33)]


def run(a, **kw):
    from paper_2609_12299_amd import attend_pages
    got = attend_pages(**on_gpu(a), lse=True, **kw)
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("lens,H,G", SHAPES)
@pytest.mark.parametrize("kind,D", [("bf16", 64), ("fp16", 80), ("fp8", 128), ("bf16", 256), ("fp8", 144)])
def test_forms(lens, H, G, kind, D):
    log(f"[gpu] attend joins {lens} {H} {G} {kind} {D}")
    a = make(kind, lens, H, G, D, 32, q_kind="bf16" if kind == "fp8" else None, seed=len(lens) + D)
    check(a, run(a))


@pytest.mark.parametrize("lens,H,G", SHAPES)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_pieces_without_a_visible_token(lens, H, G, D):
    """Pages given back in the middle, at the front, or all of them."""
    log(f"[gpu] attend empty pieces {lens} {H} {G} {D}")
    a = make("bf16", lens, H, G, D, 16, seed=D)
    columns = a["table"].shape[1]
    a["table"][:, columns // 5:columns * 4 // 5] = -1
    check(a, run(a))
    a["table"][0] = -1
    check(a, run(a))
    a["table"][:] = -1
    got = run(a)
    assert (got["out"] == 0).all() and (got["lse"] == -float("inf")).all()
