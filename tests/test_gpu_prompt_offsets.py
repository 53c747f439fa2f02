"""Offsets outside [0, rows]: taken as the nearer end, alike by rotary positions and attention."""
from __future__ import annotations

import pytest

import test_gpu_prompt_attend as attend
import test_gpu_prompt_rotate as rotate
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ints = rotate.ints

# what is given, what it stands for (49 rows)
OFFSETS = [([-5, 5, 5, 6, 46, 49], [0, 5, 5, 6, 46, 49]),
           ([-9, -9, -2, 6, 46, 49], [0, 0, 0, 6, 46, 49]),
           ([-2 ** 31, 5, 5, 6, 46, 2 ** 31 - 1], [0, 5, 5, 6, 46, 49]),
           ([0, 5, 5, 6, 90, 2 ** 31 - 1], [0, 5, 5, 6, 49, 49])]


@pytest.mark.parametrize("cache", [None, "fp8"])
@pytest.mark.parametrize("given,meant", OFFSETS)
def test_rotate(cache, given, meant):
    from paper_2609_12299_amd import rotate_tokens
    log(f"[gpu] rotate offsets {given} {cache}")
    a, b = rotate.build(cache=cache, starts=(16, 16, 16, 16, 16)), rotate.build(cache=cache, starts=(16, 16, 16, 16, 16))
    for x in (a, b):  # every place is held, a page by one sequence
        x["table"] = torch.arange(5 * 8, dtype=torch.int32, device="cuda").view(5, 8)
        for n in ("k_cache", "v_cache"):
            x[n] = torch.full((40, *x[n].shape[1:]), 3.0, device="cuda").to(x[n].dtype)
    want = rotate_tokens(**dict(a, offsets=ints(meant)))["out"]
    got = rotate_tokens(**dict(b, offsets=ints(given)))["out"]
    assert torch.equal(got, want)
    for n in ("k_cache", "v_cache"):
        assert torch.equal(a[n].float(), b[n].float())


@pytest.mark.parametrize("given,meant", OFFSETS)
def test_attend(given, meant):
    from paper_2609_12299_amd import attend_chunks
    log(f"[gpu] attend offsets {given}")
    a = attend.build(sizes=[(5, 16), (0, 16), (1, 16), (40, 16), (3, 16)])
    a["lens"] = ints([70, 70, 70, 70, 70])
    a["table"] = torch.arange(5 * 5, dtype=torch.int32, device="cuda").view(5, 5) % a["k_cache"].shape[0]
    a["k_cache"], a["v_cache"] = (torch.nan_to_num(a[n]) for n in ("k_cache", "v_cache"))
    want = attend_chunks(**dict(a, offsets=ints(meant)), lse=True)
    got = attend_chunks(**dict(a, offsets=ints(given)), lse=True)
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


def test_rows_of_falling_offsets_stay_in_bounds():
    """Which sequence a row counts to is not defined then; nothing but rows of the call is written."""
    from paper_2609_12299_amd import rotate_tokens
    log("[gpu] rotate falling offsets")
    a = rotate.build()
    guard = torch.full((300, 6, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    for bad in ([0, 30, 20, 10, 40, 49], [49, 30, 20, 10, 5, 0], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0, 7, 49]):
        a["offsets"] = ints(bad)
        rotate_tokens(**a, out=guard[100:149])
        torch.cuda.synchronize()
        assert (guard[:100] == 3).all() and (guard[149:] == 3).all()
