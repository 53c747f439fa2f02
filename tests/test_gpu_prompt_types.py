"""Queries in fp16 over a cache in 8 bits, against plain arithmetic in 64 bits."""
from __future__ import annotations

import pytest

import test_gpu_prompt_attend as attend

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def build(**kw):
    a = attend.build("fp8", **kw)
    return dict(a, q=a["q"].half())


def scales(H):
    gen = torch.Generator(device="cuda").manual_seed(9)
    return {n: torch.rand(H, generator=gen, device="cuda") * 2 + 0.2 for n in ("k_scale", "v_scale")}


@pytest.mark.parametrize("D,G,ps", [(64, 4, 16), (128, 8, 64), (128, 1, 8), (96, 5, 32), (80, 3, 8), (256, 2, 16), (16, 7, 128),
                                    (176, 16, 32), (32, 40, 16)])
def test_ragged_batch(D, G, ps):
    a = build(D=D, G=G, ps=ps)
    attend.check(a, what=f"half over 8 bits {D} {G} {ps}")
    attend.check(a, what=f"half over 8 bits {D} {G} {ps}", **scales(2))


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("window,sinks", [(1, 1), (64, 4), (100, 300), (400, 1000)])
def test_windows(D, window, sinks):
    a = build(D=D, G=3, ps=16, sizes=[(70, 0), (1, 900), (33, 450), (150, 280), (5, 63)])
    a["table"][3, 4:9] = -1
    attend.check(a, window=window, sinks=sinks, **scales(2))


@pytest.mark.parametrize("n,past", [(1, 0), (2, 0), (33, 0), (63, 1), (64, 0), (65, 63), (1, 64), (1, 65), (7, 2000)])
def test_lengths(n, past):
    for D, G in ((128, 1), (64, 8), (256, 2)):
        attend.check(build(sizes=[(n, past)], H=1, G=G, D=D, ps=8), what=f"{n} {past}", **scales(1))


def test_long_sequences_and_many_heads():
    attend.check(build(D=64, G=4, ps=64, sizes=[(3, 30000), (300, 100), (1, 9000)]), **scales(2))
    attend.check(build(D=128, G=8, ps=64, sizes=[(16, 20000)]), window=5000, sinks=70, **scales(2))
    attend.check(build(D=96, G=1, H=128, ps=16, sizes=[(1100, 0)]), window=300, **scales(128))


def test_what_is_not_seen_may_be_nan():
    for D in (64, 128, 256):
        a = build(D=D, G=2, sizes=[(90, 20), (40, 200)], ps=16)
        v, tab = a["v_cache"].float(), a["table"]
        v[tab[0, 3].long(), 0, 12, 3] = float("nan")
        v[tab[1, 13].long(), 1, 7, D - 1] = float("nan")
        a["v_cache"] = v.to(a["v_cache"].dtype)
        got = attend.check(a, what=f"NaN {D}")
        assert not torch.isnan(got["out"][:40]).any() and torch.isnan(got["out"][40:90, :2, 3]).all()
