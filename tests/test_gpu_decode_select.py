"""Beam search's selection against its definition in 64 bits."""
from __future__ import annotations

import math

import numpy as np
import pytest

import decode_ref as ref
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def make(kind, G, W, V, seed=0, spread=2.5):
    """Logits on a grid of 1/32 and beams whose candidates lie 1/(32 W) apart, so that no choice hangs
    on rounding; equal logits within a beam are common."""
    gen = torch.Generator().manual_seed(seed)
    x = ((torch.randn(G, W, V, generator=gen) * spread * 32).round() / 32).clamp(-7.9, 7.9).to(TYPES[kind])
    lse = torch.logsumexp(x.double(), 2)
    s = lse - 9.0 - torch.randint(0, 64, (G, W), generator=gen) / 32 + torch.arange(W) / (32.0 * W)
    return x, s.float()


def check(x, s, k, finished=None, eos=-1, **kw):
    from paper_2609_12299_amd import select_beams
    want = ref.select(x, s, k, finished, eos)
    xg = kw.pop("x_gpu", None)
    got = select_beams(x.cuda() if xg is None else xg, s.cuda(), k, None if finished is None else finished.cuda(), eos, **kw)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(got["parents"].cpu().numpy(), want[1])
    np.testing.assert_array_equal(got["tokens"].cpu().numpy(), want[2])
    np.testing.assert_array_equal(got["finished"].cpu().numpy(), want[3])
    sc = got["scores"].double().cpu().numpy()
    assert np.array_equal(np.isfinite(sc), np.isfinite(want[0])) and (sc[~np.isfinite(want[0])] == -np.inf).all()
    fine = np.isfinite(want[0])
    # score and logit as they are, the logarithm to 2^-22 of its size (its sum's exponents, the sum of V
    # positive terms by threads of 32 and trees, the logarithm), two additions
    size = np.abs(want[0][fine]) + np.abs(s.numpy()[np.isfinite(s.numpy())]).max(initial=0) + 24
    assert (np.abs(sc - want[0])[fine] <= 2.0 ** -21 * size).all()
    return got


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("G,W,V,k", [(1, 1, 1, 1), (1, 1, 7, 5), (2, 3, 100, 6), (3, 4, 8191, 4), (2, 5, 8193, 10),
                                     (1, 8, 50257, 16), (2, 2, 16385, 64), (1, 64, 300, 64), (5, 1, 32000, 1)])
def test_sizes(kind, G, W, V, k):
    log(f"[gpu] select {kind} {G} {W} {V} {k}")
    x, s = make(kind, G, W, V)
    check(x, s, k)


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_finished_and_eos(kind):
    log(f"[gpu] select finished {kind}")
    x, s = make(kind, 4, 4, 3000, seed=2)
    done = torch.tensor([[0, 0, 0, 0], [1, 0, 0, 1], [1, 1, 1, 1], [0, 1, 0, 0]], dtype=torch.bool)
    s = torch.where(done, -1.0 - torch.arange(4) / 3.0, s)
    best = x[0, 0].float().argmax().item()
    for eos in (best, 0, 2999, -1):
        check(x, s, 6, done, eos)


def test_equal_values():
    """More equal values than are ranked by counting: the lowest tokens win."""
    log("[gpu] select ties")
    x, s = make("bf16", 2, 3, 20000)
    x[0] = 0.5
    x[1, :, ::2] = 1.0
    x[1, 1] = -0.0
    x[1, 1, 5::3] = 0.0
    lse = torch.logsumexp(x.double(), 2)
    s = (lse - 3.0 - torch.arange(3) / 96.0).float()
    s[0, 1] = s[0, 0]  # equal beams too
    for k in (1, 7, 64):
        check(x, s, k)


def test_few_candidates():
    """Masked tokens, dead beams, rows without any candidate."""
    log("[gpu] select few")
    x, s = make("fp32", 6, 2, 9000, seed=4)
    x[0, :, 5:] = -math.inf
    x[1] = -math.inf
    s[2, 0] = -math.inf
    s[2, 1] = math.nan
    x[3, 0, 17] = math.nan
    x[4, 1, 8500] = math.inf
    x[5, 0, 1:] = torch.finfo(torch.float32).min
    x[5, 1, :] = torch.finfo(torch.float32).min
    lse = torch.logsumexp(x[5].double(), 1)
    s[5] = (lse - 1.0 - torch.arange(2) / 64).float()
    from paper_2609_12299_amd import select_beams
    want = ref.select(x[:5], s[:5], 16)
    got = select_beams(x.cuda(), s.cuda(), 16)
    np.testing.assert_array_equal(got["parents"].cpu().numpy()[:5], want[1])
    np.testing.assert_array_equal(got["tokens"].cpu().numpy()[:5], want[2])
    assert (got["tokens"][1] == -1).all() and (got["tokens"][2] == -1).all()
    assert torch.isinf(got["scores"][1]).all()
    assert got["parents"][5, 0].item() == 10 and got["tokens"][5, 0].item() == 0


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_strides_and_alignment(kind):
    log(f"[gpu] select strides {kind}")
    x, s = make(kind, 3, 4, 5001, seed=6)
    for pad in (1, 3, 8):
        wide = torch.full((3, 5, 5001 + pad), math.nan, dtype=TYPES[kind], device="cuda")
        wide[:, 1:, pad:] = x.cuda()
        check(x, s, 5, x_gpu=wide[:, 1:, pad:])


def test_repeats_stream_and_graph():
    from paper_2609_12299_amd import select_beams
    log("[gpu] select graph")
    x, s = make("bf16", 4, 4, 30001, seed=8)
    first = check(x, s, 8, stream=torch.cuda.Stream())
    xg, sg = x.cuda(), s.cuda()
    select_beams(xg, sg, 8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = select_beams(xg, sg, 8)
    for _ in range(3):
        for y in res.values():
            y.zero_()
        torch.randn(1 << 18, device="cuda").sum()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(res[n], first[n]) for n in res)


def test_rows_beyond_32_bits():
    """Logits of more than 2^31 elements; the far rows are looked at too."""
    log("[gpu] select far rows")
    G, W, V = 9000, 2, 128000
    x = torch.zeros((G, W, V), dtype=torch.bfloat16, device="cuda")
    x[:, 0, 77], x[:, 1, V - 1] = 5.0, 3.0
    from paper_2609_12299_amd import select_beams
    got = select_beams(x, torch.zeros((G, W), device="cuda"), 2)
    assert (got["tokens"] == torch.tensor([77, V - 1], device="cuda")).all()
    assert torch.equal(got["parents"].cpu(), torch.arange(2 * G).reshape(G, 2).int())


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_logits_of_any_size(kind):
    """Rows of one value, of one that stands out, and rows whose parts lie far apart: the logarithm of
    the sum is as good for values of 10^36 as for those of 10."""
    log(f"[gpu] select sizes of logits {kind}")
    sizes = [3.0, 9e4, 5e5, 9.9e5, 1.1e6, 1e9, 1e10, 3e30, 8e36, 1.5e37, 3e38]
    V = 20000
    x = torch.zeros(2 * len(sizes) + 1, 2, V)
    for i, c in enumerate(sizes):
        x[2 * i], x[2 * i + 1] = c, -c
        x[2 * i:2 * i + 2, 1, V - 3] += c / 64
    x[-1, 0], x[-1, 1] = 100.0, -2e6
    x[-1, 0, V - 3] = 2e6
    x[-1, 1, :300] = -5.0
    x = x.to(TYPES[kind])
    s = torch.tensor([-1.0, -4.0 / 3.0]).repeat(len(x), 1)
    check(x, s, 6)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("k", [31, 32, 33, 63, 64])
def test_large_k(kind, k):
    """Lists that fill up within a step, rows that rise (every element is among the best so far) and
    rows of few values."""
    log(f"[gpu] select large k {kind} {k}")
    G, W, V = 3, 2, 30011
    gen = torch.Generator().manual_seed(k)
    x = torch.randn(G, W, V, generator=gen) * 2.5
    x[1] = torch.arange(V) / 4000.0
    x[2] = torch.randint(0, 3, (W, V), generator=gen).float()
    x = ((x * 32).round() / 32).clamp(-7.9, 7.9).to(TYPES[kind])
    s = (torch.logsumexp(x.double(), 2) - 9.0 + torch.arange(W) / (32.0 * W)).float()
    check(x, s, k)


def around_a_million(V, W, sign):
    """Rows [5, W, V] in fp32 with values on both sides of sign * 10^6, in steps of 1/16, which 32 bits hold there."""
    gen = torch.Generator().manual_seed(11)
    x = torch.empty(5, W, V)
    x[0] = sign * 1e6 - 0.0625  # of one value, one that stands out on the other side
    x[0, :, V - 3] = sign * 1e6 + 0.5
    x[1] = sign * 1e6 + 0.5     # the higher ones first
    x[1, :, V // 3:] = sign * 1e6 - 0.25
    x[2] = sign * 1e6 - 8.75 + (torch.randn(W, V, generator=gen) * 2.5 * 16).round() / 16
    x[3] = sign * 1e6 + (torch.rand(V, generator=gen) * 20 - 10).mul_(16).round_() / 16
    x[4] = sign * 1e6 - 10 + (20.0 * torch.arange(V) / V * 16).round() / 16  # and the maximum moves all the time
    return x


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("W,k,V", [(2, 6, 20000), (64, 64, 20000), (2, 3, 4096), (1, 2, 9)])
def test_logits_on_both_sides_of_a_million(sign, W, k, V):
    """Where the form of the exponentials changes: a row's parts on either side (the first shape), and the
    steps of one part (the second)."""
    log(f"[gpu] select around {sign} 10^6: {W} x {V}")
    x = around_a_million(V, W, sign)
    s = (-1.0 - torch.arange(W) / 3.0).repeat(len(x), 1)
    check(x, s, k)


def test_rows_masked_by_a_sum():
    """Beams of whose tokens all or some carry about -10^6, beside one that carries nothing."""
    log("[gpu] select masked by a sum")
    gen = torch.Generator().manual_seed(5)
    x = (torch.randn(3, 4, 32000, generator=gen) * 2.5 * 16).round() / 16
    x[:, 1] += -1e6 - 8.75
    x[:, 2, ::2] += -1e6
    x[:, 3] += 1e6 - 8.75
    check(x, (-1.0 - torch.arange(4) / 3.0).repeat(3, 1), 8)
