"""New tokens into their pages, page tables from step to step, and compaction, against their definitions."""
from __future__ import annotations

import random

import numpy as np
import pytest

import decode_ref as ref
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- append

def append_case(kind, source, counts, starts, H, D, ps, columns, seed=0, layout="heads"):
    gen = torch.Generator().manual_seed(seed)
    S, T = len(counts), sum(counts)
    pages = S * columns + 2
    table = torch.randperm(pages, generator=gen)[:S * columns].reshape(S, columns).int()
    fused = torch.randn(max(T, 1), 3, H, D, generator=gen).mul_(8).to(TYPES[source])[:T]
    caches = [torch.randn(pages, H, ps, D, generator=gen).to(TYPES[kind]) for _ in range(2)]
    if layout == "tokens":
        caches = [c.transpose(1, 2).contiguous().transpose(1, 2) for c in caches]
    scales = [torch.rand(H, generator=gen) * 0.05 + 0.01 for _ in range(2)] if kind == "fp8" else [None, None]
    return table, fused, caches, scales


def append_want(cache, new, table, counts, starts, scale):
    """Bytes of the cache afterwards, row after row."""
    N, H, ps, D = cache.shape
    want, r = cache.clone(), 0
    for s, n in enumerate(counts):
        for i in range(n):
            pos = starts[s] + i
            if 0 <= pos < table.shape[1] * ps and 0 <= int(table[s, pos // ps]) < N:
                x = new[r]
                if scale is not None:
                    x = (x.float() / scale[:, None]).clamp(-448, 448)
                want[int(table[s, pos // ps]), :, pos % ps] = x.to(cache.dtype)
            r += 1
    return want


def bits(x):
    return x.contiguous().view(torch.uint8)


@pytest.mark.parametrize("kind,source", [("bf16", "bf16"), ("fp16", "fp16"), ("fp8", "bf16"), ("fp8", "fp16")])
@pytest.mark.parametrize("H,D,ps,layout", [(1, 64, 8, "heads"), (8, 128, 16, "heads"), (3, 80, 32, "tokens"), (2, 256, 64, "heads")])
@pytest.mark.parametrize("counts", [[1] * 5, [0, 3, 0, 40, 1, 17, 0], [5000, 1]])
def test_append(kind, source, H, D, ps, layout, counts):
    from paper_2609_12299_amd import append_tokens
    log(f"[gpu] append {kind} {source} {H} {D} {ps} {counts}")
    rnd = random.Random(1)
    starts = [rnd.randrange(40) for _ in counts]
    columns = -(-(max(counts) + 40) // ps)
    table, fused, caches, scales = append_case(kind, source, counts, starts, H, D, ps, columns, layout=layout)
    table[0, 0] = -1  # not held: left out
    k, v = (torch.empty_strided(c.shape, c.stride(), dtype=c.dtype, device="cuda").copy_(c) for c in caches)
    f = fused.cuda()
    offsets = None if counts == [1] * len(counts) else ints(np.concatenate([[0], np.cumsum(counts)]).tolist())
    append_tokens(f[:, 0], f[:, 2], k, v, table.cuda(), ints(starts), offsets,
                  *[None if x is None else x.cuda() for x in scales])
    for c, new, cache, scale in ((k, fused[:, 0], caches[0], scales[0]), (v, fused[:, 2], caches[1], scales[1])):
        assert torch.equal(bits(c.cpu()), bits(append_want(cache, new, table, counts, starts, scale)))


def test_append_extremes_and_rows_left_out():
    from paper_2609_12299_amd import append_tokens
    log("[gpu] append extremes")
    H, D, ps = 1, 16, 8
    x = torch.zeros(4, H, D, dtype=torch.bfloat16)
    x[0, 0, :8] = torch.tensor([float("inf"), -float("inf"), float("nan"), 3.38e38, -3.38e38, 1e-38, -0.0, 449.0])
    x[1, 0, :6] = torch.tensor([0.009765625, 0.0029296875, 17.0, 18.0, 464.0, -500.0])
    scale = torch.tensor([0.01])
    for sc in (scale, torch.tensor([1.0]), torch.tensor([3.0])):
        k, v = (torch.ones(3, H, ps, D).to(TYPES["fp8"]).cuda() for _ in range(2))
        table = ints([[2], [1], [0], [7]])
        # row 2 lies before its sequence, row 3 in a page out of range
        append_tokens(x.cuda(), x.cuda(), k, v, table, ints([0, 7, -1, 0]), None, sc.cuda(), sc.cuda())
        want = append_want(torch.ones(3, H, ps, D).to(TYPES["fp8"]), x, table.cpu(), [1] * 4, [0, 7, -1, 0], sc)
        for c in (k, v):
            c = c.float().cpu()
            w = want.float()
            assert torch.equal(torch.isnan(c), torch.isnan(w)) and torch.equal(c.nan_to_num(0), w.nan_to_num(0))
    # offsets that leave rows before the first and behind the last
    k, v = (torch.zeros(3, H, ps, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    append_tokens(x.nan_to_num(1.0).cuda(), x.cuda(), k, v, ints([[2], [1]]), ints([0, 3]), ints([1, 2, 3]))
    assert torch.equal(k[2, 0, 0].cpu(), x.nan_to_num(1.0)[1, 0]) and torch.equal(k[1, 0, 3].cpu(), x.nan_to_num(1.0)[2, 0])
    k[2, 0, 0], k[1, 0, 3] = 0, 0
    assert (k == 0).all()


def test_append_every_quotient():
    """All bf16 numbers over some scales: the quotient is rounded as a division's."""
    from paper_2609_12299_amd import append_tokens
    log("[gpu] append quotients")
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).reshape(256, 1, 256)
    for sc in (0.01, 0.3, 1.0 / 3.0, 7.0, 0.0123456, 1e-3, 100.0):
        s = torch.tensor([sc])
        k, v = (torch.zeros(32, 1, 8, 256, dtype=torch.uint8, device="cuda").view(TYPES["fp8"]) for _ in range(2))
        append_tokens(every.cuda(), every.cuda(), k, v, torch.arange(32, dtype=torch.int32, device="cuda")[None],
                      ints([0]), ints([0, 256]), s.cuda(), s.cuda())
        want = (every.float() / s).clamp(-448, 448).to(TYPES["fp8"]).float().reshape(-1)
        got = k.float().cpu().reshape(-1)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.nan_to_num(0), want.nan_to_num(0)), sc


# ------------------------------------------------------------------- step

def check_step(table, lens, parents, grow, ps, N, held=None, window=0, sinks=0, layers=2, layout="dense", **kw):
    from paper_2609_12299_amd import step_pages
    table, lens = np.asarray(table, np.int32), np.asarray(lens, np.int32)
    want = ref.step(table, lens, parents, grow, ps, N, held, window, sinks)
    gen = torch.Generator().manual_seed(5)
    k = torch.randn(layers, N, 2, max(ps, 8), 8, generator=gen).to(torch.bfloat16).cuda()
    v = torch.randn(layers, N, max(ps, 8), 24, generator=gen).cuda()
    if layout == "pages first":  # a page's layers side by side
        k = k.transpose(0, 1).contiguous().transpose(0, 1)
    before = [c.clone() for c in (k, v)]
    wide = torch.full((max(len(lens), 1), table.shape[1] + 2), 7, dtype=torch.int32, device="cuda")[:len(lens)]
    wide[:, :-2] = torch.from_numpy(table).cuda()
    got = step_pages(wide[:, :-2], ints(lens.tolist()), None if parents is None else ints(list(parents)),
                     None if grow is None else ints(list(grow)), ps, held=None if held is None else ints(list(held)),
                     num_pages=N, caches=(k, v), window=window, sinks=sinks, **kw)
    torch.cuda.synchronize()
    for name, w in zip(("table", "lens", "refs", "counters"), want):
        np.testing.assert_array_equal(got[name].cpu().numpy(), w, err_msg=name)
    for c, b in zip((k, v), before):
        for src, dst in want[4]:
            b[:, dst] = b[:, src]
        assert torch.equal(c, b)
    return got


def random_step(rnd, ps, S0, P, N, S, share=0.5):
    """Old tables with shared pages, lengths of all kinds, some entries that are none."""
    table = np.full((S0, P), -1, np.int32)
    lens = np.zeros(S0, np.int32)
    for s in range(S0):
        n = rnd.choice([0, 1, rnd.randrange(P * ps + 1), rnd.randrange(P * ps + 1)])
        lens[s] = n
        src = rnd.randrange(s) if s and rnd.random() < share else None
        for c in range(-(-n // ps)):
            table[s, c] = table[src, c] if src is not None and rnd.random() < 0.9 else rnd.randrange(N)
            if rnd.random() < 0.03:
                table[s, c] = rnd.choice([-1, N, -9])
        if rnd.random() < 0.05:
            lens[s] = rnd.choice([-3, P * ps + 100])
    parents = [rnd.choice([-1, rnd.randrange(max(S0, 1)) if S0 else -1, rnd.randrange(-3, S0 + 3)]) for _ in range(S)]
    grow = [rnd.choice([0, 1, 1, rnd.randrange(2 * ps + 1), -2]) for _ in range(S)]
    return table, lens, parents, grow


@pytest.mark.parametrize("seed", range(12))
def test_step_random(seed):
    rnd = random.Random(seed)
    ps = rnd.choice([1, 8, 16])
    S0, S, P, N = rnd.randrange(1, 12), rnd.randrange(1, 14), rnd.randrange(1, 20), rnd.randrange(20, 400)
    log(f"[gpu] step seed {seed}: {S0} -> {S} sequences, {P} columns of {ps}, {N} pages")
    table, lens, parents, grow = random_step(rnd, ps, S0, P, N, S)
    held = [rnd.choice([0, 0, 0, 1, 2, -1]) for _ in range(N)] if seed % 2 else None
    window = rnd.choice([0, 1, rnd.randrange(1, P * ps + 1)])
    check_step(table, lens, parents, grow, ps, N, held, window, rnd.choice([0, 1, ps, 3 * ps]) if window else 0,
               layout=rnd.choice(["dense", "pages first"]))


@pytest.mark.parametrize("S,P,N", [(600, 40, 9000), (3, 700, 5000), (1, 1, 1), (257, 3, 20001)])
def test_step_sizes(S, P, N):
    log(f"[gpu] step {S} {P} {N}")
    rnd = random.Random(S)
    table, lens, parents, grow = random_step(rnd, 8, S, P, N, S + 3)
    check_step(table, lens, parents, grow, 8, N, layers=1)


def test_step_beams():
    """Four beams of one prompt: who writes on, who copies, who is let go."""
    log("[gpu] step beams")
    P, ps = 8, 16
    table = np.full((4, P), -1, np.int32)
    table[:, 0] = 5
    table[:, 1] = [6, 7, 8, 9]
    lens = [20, 20, 20, 20]
    got = check_step(table, lens, [1, 1, 1, 3], [1] * 4, ps, 16)
    assert got["table"][:, 1].tolist() == [7, 0, 1, 9]  # the first writes on; 6 and 8 come free after the copies
    check_step(table, lens, [0, 1, 2, 3], [1] * 4, ps, 16)
    check_step(table, lens, None, None, ps, 16)           # nothing moves
    check_step(table, lens, None, [13] * 4, ps, 16)       # every beam into a page of its own
    check_step(table, lens, [-1] * 4, [0] * 4, ps, 16)    # all let go
    check_step(table, lens, [2, 2], [0, 4], ps, 16)       # one stands still, one grows
    check_step(table, lens, [0, 1, 2, 3], [1] * 4, ps, 16, held=[0] * 7 + [1] + [0] * 8)
    check_step(table, lens, [3, 3, 3, 3], [1] * 4, ps, 9)  # no page left for all copies
    # a page that ends inside for one and is whole for another
    table[1, :3] = [5, 6, 10]
    check_step(table, [20, 40, 20, 20], [0, 1, 0], [1, 1, 1], ps, 16)


def test_step_of_nothing():
    log("[gpu] step empty")
    check_step(np.zeros((0, 4), np.int32), [], [-1, -1], [5, 0], 8, 32)
    check_step(np.full((2, 4), -1, np.int32), [0, 0], [], [], 8, 32)


def test_step_repeats_and_graph():
    from paper_2609_12299_amd import step_pages
    log("[gpu] step graph")
    rnd = random.Random(3)
    table, lens, parents, grow = random_step(rnd, 16, 40, 30, 3000, 50)
    want = ref.step(table, lens, parents, grow, 16, 3000)
    args = (torch.from_numpy(table).cuda(), ints(lens.tolist()), ints(parents), ints(grow), 16)
    step_pages(*args, num_pages=3000)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step_pages(*args, num_pages=3000)
    for _ in range(3):
        for x in res.values():
            x.fill_(77)
        torch.randn(1 << 18, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, w in zip(("table", "lens", "refs", "counters"), want):
            np.testing.assert_array_equal(res[name].cpu().numpy(), w, err_msg=name)


# ---------------------------------------------------------------- compact

@pytest.mark.parametrize("N,S,P,live", [(1, 1, 1, 1.0), (64, 3, 5, 0.5), (5000, 7, 90, 0.3), (4096, 2, 8, 0.0),
                                        (4097, 2, 8, 1.0), (20000, 300, 20, 0.7)])
def test_compact(N, S, P, live):
    from paper_2609_12299_amd import compact_pages
    log(f"[gpu] compact {N} {S} {P} {live}")
    rnd = np.random.default_rng(N)
    refs = np.where(rnd.random(N) < live, rnd.integers(1, 5, N), rnd.choice([0, 0, -1], N)).astype(np.int32)
    table = rnd.integers(-3, N + 3, (S, P)).astype(np.int32)
    want = ref.compact(table, refs)
    gen = torch.Generator().manual_seed(1)
    k = torch.randn(3, N, 16, generator=gen).cuda()
    v = torch.randn(1, N, 2, 8, 40, generator=gen).to(torch.bfloat16).cuda()
    before = [c.clone() for c in (k, v)]
    got = compact_pages(torch.from_numpy(table).cuda(), ints(refs.tolist()), caches=(k, v))
    torch.cuda.synchronize()
    for name, w in zip(("table", "refs", "map", "counters"), want):
        np.testing.assert_array_equal(got[name].cpu().numpy(), w, err_msg=name)
    for c, b in zip((k, v), before):
        if want[4]:
            src, dst = (torch.tensor(x, device="cuda") for x in zip(*want[4]))
            b[:, dst] = b[:, src]
        assert torch.equal(c, b)


@pytest.mark.parametrize("N", [32, 5000])
@pytest.mark.parametrize("parents", [None, []])
@pytest.mark.parametrize("hold", [False, True])
def test_step_from_no_sequences_to_none(N, parents, hold):
    """A batch that has run dry: the holds that are left are counted."""
    log(f"[gpu] step of no sequences {N} {parents} {hold}")
    held = [p % 3 - 1 for p in range(N)] if hold else None
    check_step(np.zeros((0, 4), np.int32), [], parents, None, 8, N, held)
    check_step(np.zeros((0, 4), np.int32), [], parents, [], 8, N, held)


@pytest.mark.parametrize("source", ["bf16", "fp16"])
@pytest.mark.parametrize("scale", [2.0 ** -149, 2.0 ** -140, 2.0 ** -129, 1.1 * 2.0 ** -127, 2.0 ** -126, 1.7 * 2.0 ** -119,
                                   2.0 ** -100, 1.3 * 2.0 ** -81, 1.9 * 2.0 ** -80, 1.1 * 2.0 ** 80, 1.7 * 2.0 ** 118,
                                   1.3 * 2.0 ** 127, float("inf"), 0.0, -0.5, -2.0 ** -130])
def test_append_scales_of_any_size(source, scale):
    """All numbers of 16 bits over scales whose reciprocal is no ordinary number, or whose products leave
    remainders below the least number of 32 bits."""
    from paper_2609_12299_amd import append_tokens
    log(f"[gpu] append {source} over {scale}")
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TYPES[source]).reshape(256, 1, 256)
    s = torch.tensor([scale], dtype=torch.float64).float()
    k, v = (torch.zeros(32, 1, 8, 256, dtype=torch.uint8, device="cuda").view(TYPES["fp8"]) for _ in range(2))
    append_tokens(every.cuda(), every.cuda(), k, v, torch.arange(32, dtype=torch.int32, device="cuda")[None],
                  ints([0]), ints([0, 256]), s.cuda(), s.cuda())
    want = (every.float() / s).clamp(-448, 448).to(TYPES["fp8"]).float().reshape(-1)
    for c in (k, v):
        got = c.float().cpu().reshape(-1)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got.nan_to_num(0), want.nan_to_num(0))
