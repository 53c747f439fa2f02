"""Attention of chunks of new tokens over a paged cache, against plain arithmetic in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest

import prompt_ref as ref
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn}
RAGGED = [(1, 0), (37, 91), (0, 50), (5, 1000), (130, 3), (1, 640), (64, 64), (2, 0)]  # new, past


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def build(kind="bf16", sizes=RAGGED, H=2, G=4, D=64, ps=16, seed=0, spare=0, columns=None, junk=True):
    """Tensors of a batch; what no sequence has is NaN."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[kind]
    qt = torch.bfloat16 if kind == "fp8" else t
    lens = [n + p for n, p in sizes]
    columns = columns or max(1, max(-(-x // ps) for x in lens)) + 1
    need = [-(-x // ps) for x in lens]
    N = sum(need) + 3
    perm = torch.randperm(N, generator=gen, device="cuda").int()
    table = torch.full((len(sizes), columns), -1, dtype=torch.int32, device="cuda")
    caches = [torch.full((N, H, ps, D), float("nan") if junk else 0.0, device="cuda") for _ in range(2)]
    at = 0
    for s, n in enumerate(need):
        ids = perm[at:at + n]
        table[s, :n] = ids
        at += n
        for c in caches:
            rows = torch.randn((n * ps, H, D), generator=gen, device="cuda")
            rows[lens[s]:] = float("nan") if junk else 0.0
            c[ids.long()] = rows.view(n, ps, H, D).transpose(1, 2)
    k, v = (c.to(t) for c in caches)
    T = sum(n for n, _ in sizes)
    fused = torch.randn((T + spare, H * G + 2 * H, D), generator=gen, device="cuda").to(qt)
    ends = np.cumsum([0] + [n for n, _ in sizes])
    return dict(q=fused[:, :H * G], k_cache=k, v_cache=v, table=table, lens=ints(lens), offsets=ints(ends.tolist()))


def check(a, scale=None, what="", got=None, **kw):
    from paper_2609_12299_amd import attend_chunks
    log(f"[gpu] chunks {what} {tuple(a['q'].shape)} {tuple(a['k_cache'].shape)} {kw}")
    if got is None:
        got = attend_chunks(**a, scale=scale, lse=True, **kw)
    torch.cuda.synchronize()
    D = a["q"].shape[2]
    o, l, to, tl, real = ref.attend(a["q"], a["k_cache"], a["v_cache"], a["table"], a["lens"], a["offsets"],
                                    D ** -0.5 if scale is None else scale, kw.get("window", 0), kw.get("sinks", 0),
                                    kw.get("k_scale"), kw.get("v_scale"))
    out, lse = got["out"].double().cpu().numpy()[real], got["lse"].double().cpu().numpy()[real]
    o, l, to, tl = o[real], l[real], to[real], tl[real]
    np.testing.assert_array_equal(np.isnan(out), np.isnan(o))
    fine = np.isfinite(o)
    np.testing.assert_array_equal(out[~fine & ~np.isnan(o)], o[~fine & ~np.isnan(o)])
    far = np.abs(out[fine] - o[fine]) - to[fine]
    assert far.size == 0 or far.max() <= 0, f"out is off by {far.max()} more than it may, {(far > 0).sum()} of {far.size}"
    np.testing.assert_array_equal(np.isneginf(lse), np.isneginf(l))
    seen = np.isfinite(l)
    assert (np.abs(lse[seen] - l[seen]) <= tl[seen]).all(), np.abs(lse[seen] - l[seen]).max()
    return got


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("D,G,ps", [(64, 4, 16), (128, 8, 64), (128, 1, 8), (96, 5, 32), (80, 3, 8), (256, 2, 16), (16, 7, 128),
                                    (176, 16, 32), (32, 40, 16)])
def test_ragged_batch(kind, D, G, ps):
    a = build(kind, D=D, G=G, ps=ps)
    kw = {}
    if kind == "fp8":
        kw = dict(k_scale=torch.tensor([0.7, 1.9], device="cuda"), v_scale=torch.tensor([3.0, 0.25], device="cuda"))
    check(a, what=f"{kind} {D} {G} {ps}", **kw)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 0), (64, 4), (65, 64), (100, 300), (129, 1), (100000, 5), (400, 1000)])
@pytest.mark.parametrize("kind,D", [("bf16", 64), ("fp16", 128), ("fp8", 128), ("bf16", 256)])
def test_windows(kind, D, window, sinks):
    a = build(kind, D=D, G=3, ps=16, sizes=[(70, 0), (1, 900), (33, 450), (150, 280), (5, 63)])
    check(a, what=kind, window=window, sinks=sinks)


@pytest.mark.parametrize("n,past", [(1, 0), (2, 0), (31, 0), (32, 0), (33, 0), (63, 1), (64, 0), (65, 63), (128, 0), (129, 127), (1, 63),
                                    (1, 64), (1, 65), (300, 0), (7, 2000)])
def test_lengths(n, past):
    for kind, D, G in (("bf16", 128, 1), ("fp8", 64, 8), ("fp16", 256, 2)):
        check(build(kind, sizes=[(n, past)], H=1, G=G, D=D, ps=8), what=f"{n} {past}")


def test_group_of_one_and_many_heads():
    check(build(sizes=[(200, 10), (3, 300)], H=5, G=1, D=128, ps=16))
    check(build(sizes=[(9, 10), (3, 300)], H=1, G=256, D=64, ps=16))
    check(build(sizes=[(40, 0)], H=16, G=2, D=8, ps=16))


def test_pages_that_are_not_held():
    a = build(D=128, sizes=[(100, 200), (3, 500), (40, 0)])
    a["table"][0, 3:9] = -1
    a["table"][0, 11] = a["k_cache"].shape[0]  # beyond the pool
    a["table"][1, ::2] = -5
    a["table"][2, :] = -1                      # nothing at all
    got = check(a)
    assert (got["out"][103:] == 0).all() and torch.isneginf(got["lse"][103:]).all()
    check(a, window=50, sinks=4)
    f = build("fp8", D=64, sizes=[(100, 200), (3, 500)])
    f["table"][0, 3:9] = -1
    check(f)


def test_lengths_out_of_their_range():
    """More new tokens than tokens, lengths below 0 and beyond the table."""
    a = build(D=64, sizes=[(20, 10), (30, 40), (10, 100), (5, 60)], columns=8, junk=False)
    a["lens"] = ints([7, -3, 1000, 0])
    a["table"].clamp_(min=0)
    check(a)
    check(a, window=5)


def test_rows_of_no_sequence_are_left_alone():
    from paper_2609_12299_amd import attend_chunks
    a = build(sizes=[(5, 3), (40, 100)], D=64, spare=20)
    a["offsets"] += 7
    a["q"][:7] = float("nan")
    a["q"][52:] = float("nan")
    out = torch.full(a["q"].shape, 3.0, dtype=torch.bfloat16, device="cuda")
    got = attend_chunks(**a, lse=True, out=out)
    assert got["out"] is out and (out[:7] == 3).all() and (out[52:] == 3).all()
    check(a, got=got)


def test_offsets_out_of_order_stay_in_bounds():
    """What they say is undefined then; nothing outside the rows is touched."""
    from paper_2609_12299_amd import attend_chunks
    a = build(sizes=[(50, 30), (40, 10), (8, 0)], D=64)
    guard = torch.full((300, 8, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    for bad in ([0, 60, 20, 98], [-5, 50, 90, 98], [0, 50, 2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, 0, 0, 2 ** 31 - 1], [98, 90, 50, 0]):
        a["offsets"] = ints(bad)
        attend_chunks(**a, out=guard[100:198])
        torch.cuda.synchronize()
        assert (guard[:100] == 3).all() and (guard[198:] == 3).all()


def test_what_is_not_seen_may_be_anything():
    """NaN and infinities among the new tokens: the rows before them do not know."""
    for kind, D in (("bf16", 128), ("fp16", 64), ("fp8", 128), ("bf16", 256)):
        a = build(kind, D=D, G=2, sizes=[(90, 20), (40, 200)], ps=16)
        k, v, tab = a["k_cache"].float(), a["v_cache"].float(), a["table"]
        inf = float("inf") if kind != "fp8" else float("nan")

        def put(c, s, j, h, d, x):
            c[tab[s, j // 16].long(), h, j % 16, d] = x
        put(v, 0, 60, 0, 3, float("nan"))
        put(v, 0, 80, 0, 3, inf)
        put(v, 0, 75, 1, 7, inf)
        put(v, 0, 100, 1, 7, -inf)
        put(v, 1, 215, 0, D - 1, -inf)
        put(v, 1, 216, 0, D - 2, inf)
        put(v, 1, 2, 1, 0, float("nan"))  # everybody sees this one
        a["v_cache"] = v.to(TYPES[kind])
        got = check(a, what=kind)
        assert not torch.isnan(got["out"][:40].float()).any()
        check(a, what=kind, window=30, sinks=3)
        put(k, 0, 70, 0, 5, float("nan"))
        put(k, 1, 230, 1, 6, inf)
        a["k_cache"] = k.to(TYPES[kind])
        out = check_hidden_keys(a)
        assert not torch.isnan(out[:50]).any() and torch.isnan(out[50:90, :2]).all()


def check_hidden_keys(a):
    from paper_2609_12299_amd import attend_chunks
    b = dict(a, v_cache=torch.nan_to_num(a["v_cache"].float(), 0, 0, 0).to(a["v_cache"].dtype))
    return attend_chunks(**b)["out"].float()


def test_scores_of_minus_infinity_and_large_ones():
    a = build("bf16", D=64, G=1, H=1, sizes=[(100, 30)])
    q = a["q"].clone()
    check(dict(a, q=q * 200), what="large")
    check(dict(a, q=q * 2000), what="larger")
    check(dict(a, q=q), scale=-0.125, what="negative scale")
    check(dict(a, q=q), scale=0.0, what="scale 0")
    k = a["k_cache"].clone()
    k[..., 0] = -float("inf")
    q[..., 0] = 1.0
    got = check_no_score(dict(a, q=q, k_cache=k))
    assert (got["out"] == 0).all() and torch.isneginf(got["lse"]).all()


def check_no_score(a):
    from paper_2609_12299_amd import attend_chunks
    return attend_chunks(**a, lse=True)


def test_scores_that_climb():
    """Maxima that move at every step."""
    a = build("fp16", D=64, G=1, H=1, sizes=[(200, 300)], ps=16, junk=False)
    k = torch.zeros_like(a["k_cache"])
    for j in range(500):
        k[a["table"][0, j // 16].long(), 0, j % 16, 0] = j * 0.25
    q = torch.zeros_like(a["q"])
    q[..., 0] = 8.0
    check(dict(a, q=q, k_cache=k), scale=1.0)
    check(dict(a, q=-q, k_cache=k), scale=1.0)


@pytest.mark.parametrize("order", [(0, 1, 2), (1, 0, 2), (0, 2, 1), (2, 1, 0)])
def test_strides(order):
    """Any order of the cache's dimensions, rows of q with room between them, tables that are views."""
    a = build("bf16", D=80, G=2, ps=16)
    for n in ("k_cache", "v_cache"):
        c = a[n]
        shape = [c.shape[i] for i in order] + [96]
        back = [order.index(i) for i in range(3)] + [3]
        wide = torch.full(shape, float("nan"), dtype=c.dtype, device="cuda").permute(back)[..., 8:88]
        wide.copy_(c)
        a[n] = wide
    table = torch.full((a["table"].shape[0], a["table"].shape[1] + 9), 7, dtype=torch.int32, device="cuda")
    table[:, 5:-4] = a["table"]
    a["table"] = table[:, 5:-4]
    q = torch.empty((a["q"].shape[1], a["q"].shape[0], 88), dtype=torch.bfloat16, device="cuda").transpose(0, 1)[..., :80]
    q.copy_(a["q"])
    check(dict(a, q=q))


def test_far_offsets_in_the_cache():
    """Pages that lie more than 2^32 bytes behind the first."""
    H, ps, D = 1, 16, 128
    n = 70000
    k, v = (torch.empty((n, 40, ps, D), dtype=torch.bfloat16, device="cuda")[:, 7:8] for _ in range(2))
    a = build(H=H, G=4, D=D, ps=ps, sizes=[(50, 120)])
    ids = torch.tensor([n - 1 - 5000 * i for i in range(a["k_cache"].shape[0])], device="cuda")
    k[ids], v[ids] = a["k_cache"], a["v_cache"]
    table = torch.where(a["table"] >= 0, ids[a["table"].clamp(min=0).long()].int(), -1).int()
    got = check(a)
    from paper_2609_12299_amd import attend_chunks
    far = attend_chunks(**dict(a, k_cache=k, v_cache=v, table=table), lse=True)
    assert torch.equal(far["out"], got["out"]) and torch.equal(far["lse"], got["lse"])


def test_empty_batches():
    from paper_2609_12299_amd import attend_chunks
    a = build(sizes=[(0, 40), (0, 0)], D=64)
    assert attend_chunks(**a, lse=True)["out"].shape == (0, 8, 64)
    b = build(D=64)
    none = dict(b, q=b["q"][:0], table=b["table"][:0], lens=b["lens"][:0], offsets=ints([0]))
    assert attend_chunks(**none)["out"].shape == (0, 8, 64)


def test_one_token_is_attend_pages():
    from paper_2609_12299_amd import attend_chunks, attend_pages
    a = build("bf16", sizes=[(1, p) for p in (0, 5, 63, 64, 700, 1500)], D=128)
    got = check(a)
    b = {n: a[n] for n in ("q", "k_cache", "v_cache", "table", "lens")}
    want = attend_pages(**b, lse=True)
    # each is off by half a step of the result, this one by half a step of its weights too
    assert ((got["out"].float() - want["out"].float()).abs() <= 4 * 2.0 ** -8 * a["v_cache"].float().nan_to_num().abs().max()).all()
    assert torch.allclose(got["lse"], want["lse"], atol=1e-4)


def test_graph_replays():
    """A captured call gives each replay's own answer, with eager calls between the replays."""
    from paper_2609_12299_amd import attend_chunks
    a = build("bf16", D=128, sizes=[(60, 3000), (1, 9000), (200, 0)], ps=64)
    out = torch.empty(a["q"].shape, dtype=torch.bfloat16, device="cuda")
    a["q"] = a["q"].contiguous()
    attend_chunks(**a, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend_chunks(**a, out=out)
    for i in range(4):
        a["q"].mul_(-1.5 if i % 2 else 0.7)
        want = attend_chunks(**a)["out"]
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_the_same_bits_every_time():
    from paper_2609_12299_amd import attend_chunks
    a = build("fp16", D=64, sizes=[(300, 5000), (17, 20000), (1, 12000)], ps=32)
    first = attend_chunks(**a, lse=True)
    for _ in range(5):
        again = attend_chunks(**a, lse=True)
        assert torch.equal(first["out"], again["out"]) and torch.equal(first["lse"], again["lse"])


@pytest.mark.parametrize("kind,D,G,sizes", [
    ("bf16", 128, 8, [(16, 20000)]), ("fp8", 64, 4, [(3, 30000), (700, 100), (1, 9000)]), ("fp16", 256, 2, [(40, 9000)]),
    ("bf16", 64, 16, [(600, 1200), (2, 0), (0, 3), (90, 7000)]), ("bf16", 96, 3, [(1, 16000)])])
def test_long_sequences(kind, D, G, sizes):
    """Lengths that several blocks share."""
    kw = {}
    if kind == "fp8":
        kw = dict(k_scale=torch.tensor([0.7, 1.9], device="cuda"), v_scale=torch.tensor([3.0, 0.25], device="cuda"))
    a = build(kind, D=D, G=G, ps=64, sizes=sizes)
    check(a, what=kind, **kw)
    check(a, what=kind, window=5000, sinks=70, **kw)


@pytest.mark.parametrize("kind,D,kw", [("bf16", 128, {}), ("fp8", 96, {}), ("fp16", 80, dict(window=300, sinks=5)), ("bf16", 120, dict(window=1000))])
def test_many_row_tiles(kind, D, kw):
    """Long chunks of many heads: more waves share what is read."""
    a = build(kind, D=D, G=1, H=128, ps=16, sizes=[(1100, 150)])
    if kind == "fp8":
        kw = dict(kw, k_scale=torch.rand(128, device="cuda") + 0.5, v_scale=torch.rand(128, device="cuda") + 0.5)
    check(a, what=kind, **kw)


def test_batches_of_many_lengths():
    """More row tiles than two rounds of blocks, of all lengths: some cut, the others in classes."""
    check(build("bf16", D=64, G=2, H=8, ps=16, sizes=[(1 + 37 * i % 90, 61 * i % 700) for i in range(150)] + [(3, 9000), (70, 4000)]))
    check(build("fp16", D=96, G=1, H=4, ps=32, sizes=[(1, 97 * i % 3000) for i in range(260)]), window=700, sinks=2)
