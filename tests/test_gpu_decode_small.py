"""Steps and compactions on both sides of the sizes up to which a call is one launch."""
from __future__ import annotations

import numpy as np
import pytest

import decode_ref as ref
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("S,P,N", [(128, 64, 4096), (128, 65, 4096), (127, 64, 4097), (2048, 4, 4096), (2049, 3, 4096),
                                   (2048, 1, 300), (1, 8192, 4095), (3, 8, 1)])
@pytest.mark.parametrize("held", [False, True])
def test_step(S, P, N, held):
    from paper_2609_12299_amd import step_pages
    log(f"[gpu] step {S} {P} {N} {held}")
    rng = np.random.default_rng(S * P + N)
    ps = 8
    table = rng.integers(-1, N, (S, P)).astype(np.int32)
    lens = rng.integers(0, P * ps + 1, S).astype(np.int32)
    parents = rng.integers(-1, S, S).astype(np.int32)
    grow = rng.integers(0, 20, S).astype(np.int32)
    hold = (rng.integers(0, 3, N) == 0).astype(np.int32) if held else None
    want = ref.step(table, lens, parents, grow, ps, N, hold, P * ps // 2, ps)
    cache = torch.randn((3, N, ps, 24), generator=torch.Generator().manual_seed(S)).cuda()  # 768 bytes a page
    after = cache.clone()
    for src, dst in want[4]:
        after[:, dst] = cache[:, src]
    g = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    got = step_pages(g(table), g(lens), g(parents), g(grow), ps, held=g(hold) if held else None, num_pages=N,
                     caches=(cache,), window=P * ps // 2, sinks=ps)
    torch.cuda.synchronize()
    for n, w in zip(("table", "lens", "refs", "counters"), want):
        np.testing.assert_array_equal(got[n].cpu().numpy(), w, err_msg=n)
    assert torch.equal(cache, after)


@pytest.mark.parametrize("N", [1, 15, 16, 17, 2047, 4095, 4096, 4097])
@pytest.mark.parametrize("live", [0.0, 0.01, 0.5, 0.99, 1.0])
def test_compact(N, live):
    from paper_2609_12299_amd import compact_pages
    log(f"[gpu] compact {N} {live}")
    rng = np.random.default_rng(N)
    refs = np.where(rng.random(N) < live, rng.integers(1, 5, N), rng.integers(-1, 1, N)).astype(np.int32)
    table = rng.integers(-2, N + 2, (5, 33)).astype(np.int32)
    want = ref.compact(table, refs)
    cache = torch.randn((2, N, 8, 16), generator=torch.Generator().manual_seed(N)).cuda()
    after = cache.clone()
    for src, dst in want[4]:
        after[:, dst] = cache[:, src]
    got = compact_pages(torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda(), caches=(cache,))
    torch.cuda.synchronize()
    for n, w in zip(("table", "refs", "map", "counters"), want):
        np.testing.assert_array_equal(got[n].cpu().numpy(), w, err_msg=n)
    kept = torch.from_numpy(want[2][want[2] >= 0].astype(np.int64))
    assert torch.equal(cache[:, kept.cuda()], after[:, kept.cuda()])


def test_small_calls_in_a_graph():
    """One launch of many blocks that plan each for itself: replays answer as the first call."""
    from paper_2609_12299_amd import compact_pages, step_pages
    log("[gpu] small calls in a graph")
    gen = torch.Generator().manual_seed(5)
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen).int().cuda()  # noqa: E731
    table, lens, parents, grow = ints(-1, 900, 32, 40), ints(0, 320, 32), ints(-1, 32, 32), ints(0, 9, 32)
    refs = ints(0, 3, 900)
    start = torch.randn((2, 900, 8, 16), generator=gen).cuda()
    cache, pool = start.clone(), start.clone()
    run = lambda: (step_pages(table, lens, parents, grow, 8, caches=(cache,)), compact_pages(table, refs, caches=(pool,)))  # noqa: E731
    first = run()
    torch.cuda.synchronize()
    after, packed = cache.clone(), pool.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = run()
    for _ in range(3):
        cache.copy_(start)
        pool.copy_(start)
        for r in res:
            for x in r.values():
                x.zero_()
        torch.randn(1 << 16, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for r, f in zip(res, first):
            assert all(torch.equal(r[n], f[n]) for n in f)
        assert torch.equal(cache, after) and torch.equal(pool, packed)
