"""Log probabilities of given tokens, entropy, ranks and alternatives, against plain arithmetic in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest

import prompt_ref as ref
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def build(kind, rows, vocab, seed=0, scale=2.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn((rows, vocab), generator=gen, device="cuda") * scale).to(TYPES[kind])
    return x, torch.randint(0, vocab, (rows,), generator=gen, device="cuda").int()


def check(x, tokens, top=0, what=""):
    from paper_2609_12299_amd import score_tokens
    log(f"[gpu] score {what} {tuple(x.shape)} {x.dtype} top {top}")
    got = score_tokens(x, tokens, top=top)
    torch.cuda.synchronize()
    want, tol = ref.score(x, tokens, top)
    got = {n: t.cpu().numpy() for n, t in got.items()}
    np.testing.assert_array_equal(got["ranks"], want["ranks"])
    for n in ("logprobs", "entropy") + (("top_logprobs",) if top else ()):
        g, w = got[n].astype(np.float64), want[n]
        np.testing.assert_array_equal(np.isnan(g), np.isnan(w), err_msg=n)
        np.testing.assert_array_equal(np.isneginf(g), np.isneginf(w), err_msg=n)
        fine = np.isfinite(w)
        far = np.abs(g[fine] - w[fine]) - tol[n][fine]
        assert far.size == 0 or far.max() <= 0, f"{n} is off by {far.max()} more than it may"
    if top:
        np.testing.assert_array_equal(got["top_tokens"], want["top_tokens"])
    else:
        assert set(got) == {"logprobs", "entropy", "ranks"}
    return got


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 5), (7, 31, 64), (5, 64, 0), (1, 2048, 5), (2, 2047, 20), (2, 2049, 20), (9, 8193, 1),
                                            (1, 32000, 5), (3, 50257, 64), (1, 200003, 64), (900, 1003, 3), (33, 16389, 0)])
def test_sizes(kind, rows, vocab, top):
    check(*build(kind, rows, vocab), top)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("shift", range(1, 9))
def test_alignments(kind, shift):
    """Rows that begin anywhere."""
    x, t = build(kind, 4, 5003 + shift)
    check(x[:, shift:], (t - shift).clamp(min=0), 7)


@pytest.mark.parametrize("kind", list(TYPES))
def test_few_and_many_rows(kind):
    """Rows that a block reads by itself, in one step of its waves or in some, and rows in parts."""
    check(*build(kind, 140, 33001), 6)
    check(*build(kind, 2, 32768), 64)
    check(*build(kind, 257, 9001), 3)
    x, t = build(kind, 130, 33003)
    check((x[:, 1:] * 0.4).round(), t.clamp(max=33001), 20, "few values")
    x, t = build(kind, 4, 140001)
    check((x[:, 1:] * 0.4).round(), t.clamp(max=139999), 20, "few values")


def test_equal_logits():
    """The lower token comes first, in ranks and alternatives; -0 and 0 are equal."""
    for kind in TYPES:
        x, t = build(kind, 6, 9000)
        x = (x * 0.5).round()  # few values
        check(x, t, 64, "few values")
        check(torch.zeros_like(x), t, 64, "one value")
        z = torch.zeros_like(x)
        z[:, ::3] = -0.0
        check(z, t, 20, "zeros")
    x = torch.zeros((2, 300000), device="cuda")
    check(x, torch.tensor([0, 299999], dtype=torch.int32, device="cuda"), 64)


def test_ranks_of_every_place():
    x, _ = build("bf16", 1, 5000)
    x = (x * 2).round() / 2
    for part in (x[:, :4999], x[:, 1:], x[:, 3:4990]):
        n = part.shape[1]
        tokens = torch.tensor([0, 1, 2, 5, 6, 7, 8, 9, 2046, 2047, 2048, 2055, n - 9, n - 8, n - 7, n - 2, n - 1], device="cuda").int()
        check(part.expand(len(tokens), n), tokens, 2)


def test_logits_of_minus_infinity():
    for kind in TYPES:
        x, t = build(kind, 8, 40007)
        x[0, 100:] = -float("inf")       # fewer than the alternatives asked for
        x[1, ::2] = -float("inf")
        x[2] = -float("inf")
        x[2, 40006] = 3.0                # one is left
        x[3] = -float("inf")             # none
        x[4, :40000] = -float("inf")
        t[4] = 5                         # a token that may not be chosen
        x[5, 40001:] = -float("inf")
        t[5] = 40006
        x[6, 1:] = -float("inf")
        t[6] = 0
        check(x, t, 64, "-inf")
        check(x, t, 0, "-inf")


def test_rows_that_say_nothing():
    for kind in TYPES:
        for vocab in (700, 70001):
            x, t = build(kind, 9, vocab)
            x[0, 5] = float("nan")
            x[1, vocab - 1] = float("nan")
            x[2, 0] = float("inf")
            x[3, 300] = float("inf")
            x[3, 301] = float("nan")
            x[4, ::7] = float("inf")
            x[5] = float("nan")
            x[6, vocab // 2] = -float("inf")
            got = check(x, t, 5, "NaN")
            assert (got["ranks"][:6] == -1).all() and (got["ranks"][6:] >= 0).all()


def test_tokens_outside_the_vocabulary():
    x, t = build("bf16", 5, 5000)
    t[:4] = torch.tensor([-1, 5000, 2 ** 31 - 1, -2 ** 31], device="cuda").int()
    got = check(x, t, 3)
    assert np.isneginf(got["logprobs"][:4]).all() and (got["ranks"][:4] == -1).all() and np.isfinite(got["entropy"]).all()


@pytest.mark.parametrize("size", [1e3, 1e6, 1e10, 1e30])
def test_large_logits(size):
    x, t = build("fp32", 4, 30011)
    check(x * size, t, 5)
    check(x + size, t, 5)
    check(x - size, t, 5)


def test_sure_rows():
    """Entropies near 0: nothing cancels."""
    x, t = build("fp32", 5, 20011, scale=0.1)
    for i, up in enumerate((5.0, 15.0, 25.0, 60.0, 120.0)):
        x[i, 7000 * i % 20011] += up
    got = check(x, t, 2)
    assert (got["entropy"] >= 0).all()
    for order in (torch.sort(x, 1).values, torch.sort(x, 1, descending=True).values):  # maxima that move, or never
        check(order.contiguous(), t, 2)


def test_strides_and_empty():
    from paper_2609_12299_amd import score_tokens
    x, t = build("fp16", 40, 3001)
    check(x[::4, 10:2900], (t[::4] % 2890).contiguous(), 5)
    check(x[:1].expand(6, 3001), t[:6], 5)
    none = score_tokens(x[:0], t[:0], top=4)
    assert none["top_tokens"].shape == (0, 4) and none["logprobs"].shape == (0,)


def test_offsets_beyond_32_bits():
    big = torch.empty((3, 1 << 30), dtype=torch.float32, device="cuda")
    x, t = build("fp32", 3, 9001)
    view = big[:, -9001:]
    view.copy_(x)
    check(view, t, 5)


def test_graph_replays_and_the_same_bits():
    from paper_2609_12299_amd import score_tokens
    for rows in (2, 900):
        x, t = build("bf16", rows, 60001)
        score_tokens(x, t, top=9)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = score_tokens(x, t, top=9)
        for i in range(3):
            x.mul_(-0.9)
            want = score_tokens(x, t, top=9)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(got[n], want[n]) for n in want)
