"""Attention of one new token over a paged cache against its definition in 64 bits."""
from __future__ import annotations

import math

import numpy as np
import pytest

import decode_ref as ref
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn}


def make(kind, lens, H, G, D, ps, q_kind=None, columns=None, window=0, sinks=0, seed=0, layout="heads", junk=True):
    gen = torch.Generator().manual_seed(seed)
    S = len(lens)
    columns = columns or max(1, -(-max(lens + [1]) // ps))
    pages = S * columns + 3
    dt = TYPES[kind]
    qd = TYPES[q_kind or kind]
    perm = torch.randperm(pages, generator=gen)[:S * columns].reshape(S, columns).int()
    k, v = (torch.randn(pages, H, ps, D, generator=gen).to(dt) for _ in range(2))
    if junk:  # what no sequence can see holds anything
        seen = torch.zeros(pages, ps, dtype=torch.bool)
        for s, n in enumerate(lens):
            for j in range(min(max(n, 0), columns * ps)):
                seen[perm[s, j // ps], j % ps] = True
        for c, x in ((k, math.nan), (v, math.nan)):
            f = c.float()
            f[~seen[:, None, :].expand(-1, H, -1)] = x
            c.copy_(f.to(dt))
    if layout == "tokens":  # a token's heads side by side in memory
        k, v = (c.transpose(1, 2).contiguous().transpose(1, 2) for c in (k, v))
    q = torch.randn(S, H * G, D, generator=gen).to(qd)
    a = dict(q=q, k_cache=k, v_cache=v, table=perm, lens=torch.tensor(lens, dtype=torch.int32),
             scale=D ** -0.5, window=window, sinks=sinks)
    if kind == "fp8":
        a.update(k_scale=torch.rand(H, generator=gen) + 0.5, v_scale=torch.rand(H, generator=gen) + 0.5)
    return a


def on_gpu(a):
    out = {}
    for n, x in a.items():
        if isinstance(x, torch.Tensor):
            y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda")
            y.copy_(x)
            x = y
        out[n] = x
    return out


def check(a, got, what=""):
    want = ref.attend(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lens"], a["scale"], a.get("window", 0),
                      a.get("sinks", 0), a.get("k_scale"), a.get("v_scale"))
    o, l = got["out"].double().cpu().numpy(), got["lse"].double().cpu().numpy()
    for x, y, tol, name in ((o, want[0], want[2], "out"), (l, want[1], want[3], "lse")):
        fine = np.isfinite(y)
        assert np.array_equal(x[~fine], y[~fine], equal_nan=True), f"{what} {name}: {x[~fine][:4]} {y[~fine][:4]}"
        off = np.abs(x[fine] - y[fine])
        assert np.isfinite(x[fine]).all(), f"{what} {name}: not finite"
        assert (off <= tol[fine]).all(), f"{what} {name}: off {off.max()}, {np.max(off / tol[fine])} of the tolerance"


def run(a, **kw):
    from paper_2609_12299_amd import attend_pages
    return attend_pages(**on_gpu(a), lse=True, **kw)


LENS = [0, 1, 7, 8, 31, 32, 33, 63, 129, 200]


@pytest.mark.parametrize("kind,q_kind", [("bf16", None), ("fp16", None), ("fp8", "bf16"), ("fp8", "fp16")])
@pytest.mark.parametrize("D", [64, 128, 256, 16, 80, 96, 144])
def test_types_and_head_sizes(kind, q_kind, D):
    log(f"[gpu] attend {kind} {q_kind} D={D}")
    a = make(kind, LENS, 2, 3, D, 16, q_kind)
    check(a, run(a), f"{kind} {D}")


@pytest.mark.parametrize("D", [8, 24, 40, 72, 120])
def test_head_sizes_of_eight(D):
    log(f"[gpu] attend D={D}")
    a = make("bf16", LENS, 1, 5, D, 8)
    check(a, run(a), f"{D}")


@pytest.mark.parametrize("G", [1, 2, 7, 8, 16, 17, 24, 32, 33, 71])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_groups(G, D):
    log(f"[gpu] attend G={G} D={D}")
    a = make("bf16", [1, 33, 100], 2, G, D, 16)
    check(a, run(a), f"{G} {D}")


@pytest.mark.parametrize("ps", [8, 16, 32, 64, 128, 1024])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_pages_and_layouts(ps, layout):
    log(f"[gpu] attend page {ps} {layout}")
    a = make("fp16", LENS + [ps - 1, ps, ps + 1], 2, 4, 64, ps, layout=layout)
    check(a, run(a), f"{ps} {layout}")


@pytest.mark.parametrize("lens", [[3000], [1, 5000, 0, 17], [700] * 9, [0, 0, 0], [4097, 3, 3, 3, 3, 3, 3, 3, 3000],
                                  [40] * 300, [20000, 1]])
@pytest.mark.parametrize("kind,D,G", [("bf16", 128, 8), ("fp8", 64, 20)])
def test_shared_over_blocks(lens, kind, D, G):
    """Tables long enough that segments are cut wherever the shares end."""
    log(f"[gpu] attend shares {lens[:4]} {kind} {D}")
    a = make(kind, lens, 2, G, D, 16, "bf16", columns=1300, junk=False)
    check(a, run(a), f"{lens[:4]} {kind}")


@pytest.mark.parametrize("kind,q_kind", [("bf16", None), ("fp16", None), ("fp8", "bf16"), ("fp8", "fp16")])
@pytest.mark.parametrize("D", [16, 64, 80, 96, 128, 144, 256])
@pytest.mark.parametrize("columns", [64, 130])
def test_head_sizes_over_longer_tables(kind, q_kind, D, columns):
    """A block per sequence up to 1024 tokens, shared over the waves beyond; 8 bits and 16, whole rows and parts."""
    log(f"[gpu] attend {kind} {q_kind} D={D} columns {columns}")
    a = make(kind, [1, 997, 0, 17, 513, columns * 16], 2, 5, D, 16, q_kind, columns=columns, window=0 if D % 32 else 900, sinks=3)
    check(a, run(a), f"{kind} {D} {columns}")


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (33, 64), (100, 5), (128, 31), (5000, 7), (64, 5000)])
@pytest.mark.parametrize("columns", [20, 200])
def test_window_and_sinks(window, sinks, columns):
    log(f"[gpu] attend window {window} sinks {sinks} columns {columns}")
    a = make("bf16", [0, 1, 5, 64, 65, 130, 320, 257], 2, 4, 64, 16, columns=columns, window=window, sinks=sinks)
    check(a, run(a), f"{window} {sinks}")


def test_pages_not_held_and_lengths_out_of_range():
    log("[gpu] attend holes")
    a = make("bf16", [100, 150, 64, 90, 40], 2, 4, 64, 16, columns=12)
    t, N = a["table"], a["k_cache"].shape[0]
    t[0, 1] = -1
    t[0, 6] = N
    t[1, :] = -7
    t[2, 0] = 2 ** 31 - 1
    t[2, 3] = -2 ** 31
    a["lens"][3] = -5
    a["lens"][4] = 40
    check(a, run(a), "holes")
    b = make("bf16", [64, 64], 1, 1, 64, 16, columns=4)
    b["lens"][0] = 2 ** 31 - 1  # beyond the table: as long as it
    want = dict(b, lens=torch.tensor([64, 64], dtype=torch.int32))
    check(want, run(b), "length beyond the table")


def test_infinities_nan_and_lowest_values():
    log("[gpu] attend extremes")
    for kind in ("bf16", "fp16"):
        a = make(kind, [70, 70, 70, 70, 70], 1, 2, 64, 16, seed=3)
        k, v, t = a["k_cache"], a["v_cache"], a["table"]
        big = torch.finfo(TYPES[kind]).max

        def put(c, s, j, x):
            c[t[s, j // 16], :, j % 16] = x
        put(v, 0, 5, math.inf)  # a visible infinite value, whatever its weight
        put(v, 0, 41, math.inf)
        put(k, 1, 9, math.nan)  # a visible NaN
        put(k, 2, 33, 0.0)
        a["q"][2] = 0.0
        a["q"][2, :, 0] = 1.0
        for j in range(70):  # scores at the type's lowest value, but one
            row = torch.zeros(64)
            row[0] = -big if j != 33 else 0.0
            put(k, 2, j, row.to(TYPES[kind]))
        a["q"][3] = 0.0
        a["q"][3, :, 0] = 1.0
        for j in range(70):  # every score minus infinity
            row = torch.zeros(64)
            row[0] = -math.inf
            put(k, 3, j, row.to(TYPES[kind]))
        got = run(a)
        o, l = got["out"].float().cpu(), got["lse"].cpu()
        assert torch.isinf(o[0]).all() and (o[0] > 0).all()
        assert torch.isnan(o[1]).all() and torch.isnan(l[1]).all()
        assert torch.equal(o[2], v[t[2, 2], :, 1].expand(2, 64).float())
        assert (l[2] == 0).all()
        assert (o[3] == 0).all() and (l[3] == -math.inf).all()
        last = {n: (x[4:5] if n in ("q", "table", "lens") else x) for n, x in a.items()}
        check(last, dict(out=got["out"][4:5], lse=got["lse"][4:5]), "the row beside them")


def test_weights_far_apart():
    """Scores that climb along the sequence: the running maximum moves all the time; and one token
    that outweighs all others."""
    log("[gpu] attend climbing scores")
    for kind in ("bf16", "fp16", "fp8"):
        a = make(kind, [600, 600], 1, 4, 64, 16, "bf16" if kind == "fp8" else None, columns=64, junk=False)
        k, t = a["k_cache"], a["table"]
        a["q"] = torch.zeros_like(a["q"])
        a["q"][:, :, 0] = 8.0
        for j in range(600):
            for s, x in ((0, j / 8.0), (1, 200.0 if j == 311 else -100.0)):
                row = torch.zeros(1, 64)
                row[:, 0] = x
                k[t[s, j // 16], :, j % 16] = row.to(TYPES[kind])
        check(a, run(a), kind)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-33, 1e31, 40.0, -40.0])
def test_scales(scale):
    """None, negative ones, and such that the differences of scores have to come before the exponential."""
    log(f"[gpu] attend scale {scale}")
    for kind in ("bf16", "fp16"):
        a = make(kind, [1, 100, 333], 2, 4, 64, 16, seed=9)
        a["scale"] = scale
        if abs(scale) > 1:  # scores a few units apart
            a["q"] = (a["q"].float() / abs(scale)).to(a["q"].dtype) if scale < 1e30 else a["q"] * 0
        check(a, run(a), f"{kind} {scale}")


def test_scores_beyond_a_million():
    """The maximum lies where a product's rounding would show in a weight."""
    log("[gpu] attend far scores")
    a = make("bf16", [400, 400], 1, 2, 64, 16, columns=40, junk=False)
    k, t = a["k_cache"], a["table"]
    a["q"] = torch.zeros_like(a["q"])
    a["q"][:, :, 0], a["q"][:, :, 1] = 1.0, 1.0
    a["scale"] = 1.0
    for s, big in ((0, 2.0 ** 22), (1, -2.0 ** 30)):
        for j in range(400):
            row = torch.zeros(64)
            row[0], row[1] = big, float(j % 4) / 2 if s == 0 else 0.0
            k[t[s, j // 16], :, j % 16] = row.to(torch.bfloat16)
    got = run(a)
    w = torch.exp(torch.arange(400) % 4 / 2.0).double()
    v = a["v_cache"]
    for s, weights in ((0, w), (1, torch.ones(400).double())):
        vv = torch.stack([v[t[s, j // 16], 0, j % 16] for j in range(400)]).double()
        want = (weights[:, None] * vv).sum(0) / weights.sum()
        # scores of 2^22 hold halves exactly
        off = (got["out"][s].double().cpu() - want).abs()
        assert (off <= 2.0 ** -8 * 1.01 * want.abs() + 2.0 ** -14 * vv.abs().mean()).all(), off.max()


def test_tables_of_more_than_2_31_units():
    """Work is shared out in groups of tiles where all tables could hold so much."""
    log("[gpu] attend huge tables")
    from paper_2609_12299_amd import attend_pages
    H, ps, D, S, P = 64, 32, 8, 64, 1 << 20
    a = make("bf16", [0, 1, 3000, 95, 700, 33], H, 1, D, ps, columns=96, junk=False)
    g = on_gpu(a)
    table = torch.full((S, P), -1, dtype=torch.int32, device="cuda")
    table[:6, :96] = g["table"]
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    lens[:6] = g["lens"]
    q = torch.zeros((S, H, D), dtype=torch.bfloat16, device="cuda")
    q[:6] = g["q"]
    got = attend_pages(q, g["k_cache"], g["v_cache"], table, lens, scale=a["scale"], lse=True)
    check(a, dict(out=got["out"][:6], lse=got["lse"][:6]), "huge tables")
    assert (got["out"][6:] == 0).all() and (got["lse"][6:] == -math.inf).all()


def test_strided_inputs():
    log("[gpu] attend strides")
    from paper_2609_12299_amd import attend_pages
    a = make("bf16", LENS, 2, 4, 64, 16)
    g = on_gpu(a)
    S, heads, D = g["q"].shape
    fused = torch.full((S, heads + 5, D + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    fused[:, 3:3 + heads, :D] = g["q"]
    wide = torch.full((S, g["table"].shape[1] + 3), 10 ** 9, dtype=torch.int32, device="cuda")
    wide[:, :-3] = g["table"]
    N, H, ps, _ = g["k_cache"].shape
    both = torch.empty((N, 2, H, ps, D), dtype=torch.bfloat16, device="cuda")
    both[:, 0], both[:, 1] = g["k_cache"], g["v_cache"]
    g.update(q=fused[:, 3:3 + heads, :D], table=wide[:, :-3], k_cache=both[:, 0], v_cache=both[:, 1])
    out = torch.full((S, heads, D), math.nan, dtype=torch.bfloat16, device="cuda")
    got = attend_pages(**g, lse=True, out=out)
    assert got["out"].data_ptr() == out.data_ptr()
    check(a, got, "strides")


def test_offsets_beyond_32_bits():
    log("[gpu] attend far pages")
    H, ps, D, pages = 4, 64, 128, 80000  # 5.2 GB: offsets pass 2^31 elements and 2^32 bytes
    k, v = (torch.empty((pages, H, ps, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    a = make("bf16", [300, 1000], H, 2, D, ps, columns=16)
    small = a["k_cache"].shape[0]
    far = torch.arange(small, dtype=torch.int64) * 2 + pages - 2 * small
    k[far.cuda()], v[far.cuda()] = a["k_cache"].cuda(), a["v_cache"].cuda()
    g = on_gpu({n: x for n, x in a.items() if n not in ("k_cache", "v_cache", "table")})
    from paper_2609_12299_amd import attend_pages
    got = attend_pages(k_cache=k, v_cache=v, table=far[a["table"].long()].int().cuda(), lse=True, **g)
    check(a, got, "far pages")


def test_repeats_streams_and_graph():
    """The same bits from call to call, on another stream, and replayed from a graph beside other work."""
    log("[gpu] attend repeats")
    from paper_2609_12299_amd import attend_pages
    a = make("bf16", [1, 3000, 0, 170, 900], 2, 8, 128, 16, columns=200, junk=False)
    g = on_gpu(a)
    first = {n: x.clone() for n, x in attend_pages(**g, lse=True).items()}
    torch.cuda.synchronize()
    check(a, first, "first")
    side = torch.cuda.Stream()
    for _ in range(3):
        got = attend_pages(**g, lse=True, stream=side)
        side.synchronize()
        assert torch.equal(got["out"], first["out"]) and torch.equal(got["lse"], first["lse"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = attend_pages(**g, lse=True)
    scratch = torch.empty(1 << 20, device="cuda")
    for rep in range(3):
        res["out"].fill_(7.0)
        res["lse"].fill_(7.0)
        scratch.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(res["out"], first["out"]) and torch.equal(res["lse"], first["lse"]), rep


def test_no_sequences():
    from paper_2609_12299_amd import attend_pages
    a = on_gpu(make("bf16", [5], 2, 4, 64, 16))
    a.update(q=a["q"][:0], table=a["table"][:0], lens=a["lens"][:0])
    assert attend_pages(**a, lse=True)["out"].shape == (0, 8, 64)


def test_more_segments_than_blocks():
    """2^24 sequences by heads: more than a launch of a block each could have."""
    from paper_2609_12299_amd import attend_pages
    log("[gpu] attend 2^24 segments")
    S, H, N, D = 1 << 20, 16, 1000, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    v = torch.randn((N, H, 8, D), generator=gen, device="cuda").bfloat16()
    k = torch.randn((N, H, 8, D), generator=gen, device="cuda").bfloat16()
    q = torch.randn((S, H, D), generator=gen, device="cuda").bfloat16()
    table = torch.randint(0, N, (S, 1), generator=gen, device="cuda").int()
    lens = torch.ones(S, dtype=torch.int32, device="cuda")
    lens[::7] = 0
    got = attend_pages(q, k, v, table, lens, lse=True)
    want = v[table[:, 0].long(), :, 0]
    want[::7] = 0
    # one weight over itself: the value, rounded once
    assert ((got["out"].float() - want.float()).abs() <= want.float().abs() * 2.0 ** -8).all()
    assert (got["lse"][::7] == -math.inf).all() and torch.isfinite(got["lse"][1::7]).all()


@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("big", [2.0 ** 9, 2.0 ** 12, 2.0 ** 15, 2.0 ** 19, -2.0 ** 19])
@pytest.mark.parametrize("tokens,columns", [(400, 40), (4000, 400)])
def test_large_scores_that_climb(kind, big, tokens, columns):
    """Large scores, exact in 32 bits, whose maximum moves from tile to tile and from wave to wave: a block
    for all of them, and pieces that are joined.  What is left is the rounding of the result, the
    exponentials (2^-22 each) and the weights' own (2^-16), with the maximum's below 2^-13."""
    log(f"[gpu] attend climbing scores near {big} {kind} {tokens}")
    a = make(kind, [tokens], 1, 2, 64, 16, columns=columns, junk=False)
    k, t = a["k_cache"], a["table"]
    a["scale"] = 1.0
    a["q"] = torch.zeros_like(a["q"])
    a["q"][:, :, 0], a["q"][:, :, 1] = 16.0, 1.0
    j = torch.arange(tokens)
    small = (j * 13.0 / tokens * 4).round() / 4 + (j % 4) / 4.0  # climbs by 13, in quarters
    rows = torch.zeros(tokens, 64)
    rows[:, 0], rows[:, 1] = big / 16, small
    k[t[0, j // 16].long(), 0, j % 16] = rows.to(TYPES[kind])
    got = run(a)
    w = torch.exp((small - small.max()).double())
    v = a["v_cache"][t[0, j // 16].long(), 0, j % 16].double()
    want = (w[:, None] * v).sum(0) / w.sum()
    mean = (w[:, None] * v.abs()).sum(0) / w.sum()
    off = (got["out"][0].double().cpu() - want).abs()
    assert (off <= ref.ROUND[TYPES[kind]] * 1.01 * want.abs() + 2.0 ** -13 * mean).all(), (off / mean).max()
    lse = big + small.max().double() + torch.log(w.sum())
    assert ((got["lse"][0].double().cpu() - lse).abs() <= 2.0 ** -23 * lse.abs() + 2.0 ** -13).all()
