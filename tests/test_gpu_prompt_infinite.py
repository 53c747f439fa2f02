"""Values that are not finite where a row sees them: the same answer whatever their weight is, wherever they lie
among the tokens, and in however many pieces the tokens are looked at."""
from __future__ import annotations

import pytest

import test_gpu_prompt_attend as attend
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

INF, NAN = float("inf"), float("nan")


def ladder(kind, D, H, G, sizes, scores, columns=None):
    """A batch all of whose rows have the score scores(j) for token j (scale 1)."""
    a = attend.build(kind, D=D, H=H, G=G, ps=16, sizes=sizes, columns=columns, junk=False)
    k, tab = torch.zeros(a["k_cache"].shape, device="cuda"), a["table"]
    for s, n in enumerate(a["lens"].tolist()):
        j = torch.arange(n, device="cuda")
        x = torch.tensor([scores(i) for i in range(n)], device="cuda") / 8
        k[tab[s, j // 16].long(), :, j % 16, 0] = x[:, None]
    a["k_cache"] = k.to(a["k_cache"].dtype)
    a["q"] = torch.zeros_like(a["q"])
    a["q"][..., 0] = 8.0
    return a


def put(a, s, j, h, d, x):
    a["v_cache"][a["table"][s, j // 16].long(), h, j % 16, d] = x


SHAPES = [(64, 2, 3, None), (128, 2, 4, None), (256, 1, 2, None), (96, 2, 2, None), (128, 2, 4, 1000), (64, 1, 8, 1000)]


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("low", [-8.0, -32.0, -96.0, -160.0, -400.0])
@pytest.mark.parametrize("D,H,G,columns", SHAPES)
def test_small_weights(kind, low, D, H, G, columns):
    """Token 100's score lies far below the others': its values have a part as large as that of any other token."""
    a = ladder(kind, D, H, G, [(200, 300), (9, 700)], lambda j: low if j in (100, 101) else 0.0, columns)
    put(a, 0, 100, 0, 3, INF)
    put(a, 0, 100, H - 1, D - 1, -INF)
    put(a, 0, 101, 0, 9, INF)
    put(a, 0, 350, 0, 9, -INF)  # rows from there on: both
    put(a, 1, 100, 0, 0, NAN)
    attend.check(a, scale=1.0, what=f"{kind} {low}")


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("D,H,G,columns", SHAPES)
def test_maxima_that_climb(kind, D, H, G, columns):
    """Infinite values first, then scores that lie ever higher."""
    a = ladder(kind, D, H, G, [(200, 300)], lambda j: float(j // 64) * 24.0, columns)
    put(a, 0, 20, 0, 3, INF)
    put(a, 0, 200, H - 1, D - 1, -INF)
    attend.check(a, scale=1.0, what=kind)


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("D,G", [(64, 8), (128, 4), (256, 2), (96, 8)])
def test_pieces_far_apart(kind, D, G):
    """Maxima of pieces that lie more than 104 apart: the weight of the lower one is none in 32 bits."""
    a = ladder(kind, D, 1, G, [(16, 20000)], lambda j: -130.0 if j < 11000 else 0.0)
    put(a, 0, 300, 0, 3, INF)
    put(a, 0, 9000, 0, 5, -INF)
    put(a, 0, 15000, 0, 6, INF)
    put(a, 0, 20010, 0, 7, INF)  # some of the rows
    attend.check(a, scale=1.0, what=kind)


def test_no_score_at_all():
    """Scores of minus infinity alone: zeros, whatever the values are."""
    from paper_2609_12299_amd import attend_chunks
    log("[gpu] no score")
    for D, columns in ((64, None), (128, None), (128, 1000)):
        a = ladder("bf16", D, 1, 2, [(70, 200)], lambda j: -INF, columns)
        put(a, 0, 20, 0, 3, INF)
        put(a, 0, 240, 0, 3, INF)
        got = attend_chunks(**a, scale=1.0, lse=True)
        assert (got["out"] == 0).all() and torch.isneginf(got["lse"]).all()


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp8"])
@pytest.mark.parametrize("D,H,G,columns", SHAPES)
def test_rows_without_a_score(kind, D, H, G, columns):
    """Queries of minus infinity beside others, over values that are not finite: zeros for them alone."""
    from paper_2609_12299_amd import attend_chunks
    log(f"[gpu] rows without a score {kind} {D} {columns}")
    a = ladder(kind, D, H, G, [(60, 300), (40, 0)], lambda j: 8.0, columns)
    none = torch.arange(100, device="cuda") % 3 == 1
    a["q"][none, :, 0] = -INF
    for j in (5, 200, 350):
        put(a, 0, j, 0, 3, NAN)
        put(a, 0, j + 1, 0, 4, NAN if kind == "fp8" else INF)
    got = attend_chunks(**a, scale=1.0, lse=True)
    assert (got["out"][none] == 0).all() and torch.isneginf(got["lse"][none]).all()
    rest = got["out"][~none].float()
    mine = torch.arange(100, device="cuda")[~none] < 60
    assert torch.isnan(rest[mine][:, :G, 3]).all() and (~torch.isfinite(rest[mine][:, :G, 4])).all()
    rest[:, :G, 3:5] = 0
    assert torch.isfinite(rest).all() and torch.isfinite(got["lse"][~none]).all()


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("fp16", 96), ("bf16", 80)])
def test_many_row_tiles(kind, D):
    """The same with eight waves to a block, planned and not."""
    for columns in (None, 300):
        a = ladder(kind, D, 128, 1, [(1100, 150)], lambda j: -40.0 if j == 100 else 0.0, columns)
        for h in (0, 70, 127):
            put(a, 0, 100, h, 3, INF)
            put(a, 0, 1100, h, 4, -INF)
            put(a, 0, 30, h, 5, NAN)
        from paper_2609_12299_amd import attend_chunks
        got = attend_chunks(**a, scale=1.0, lse=True)
        for h in (0, 1, 70, 127):
            attend.check(dict(a, q=a["q"][:, h:h + 1], k_cache=a["k_cache"][:, h:h + 1], v_cache=a["v_cache"][:, h:h + 1]), scale=1.0,
                         what=kind, got={n: x[:, h:h + 1] for n, x in got.items()})
