"""Rotary positions of queries and of keys on their way into the pages, against plain arithmetic in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest

import prompt_ref as ref
from decode_ref import ROUND
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def build(kind="bf16", cache=None, new=(5, 0, 1, 40, 3), starts=(0, 9, 1000, 77, 130000), heads=6, H=2, D=64, pairs=32, ps=16, seed=0):
    from paper_2609_12299_amd import rotary_frequencies
    gen = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(new)
    fused = torch.randn((T, heads + 2 * H, D), generator=gen, device="cuda").to(TYPES[kind])
    columns = max(-(-(n + s) // ps) for n, s in zip(new, starts)) + 1
    N = sum(-(-n // ps) + 1 for n in new) + 2
    table = torch.full((len(new), columns), -1, dtype=torch.int32, device="cuda")
    perm, at = torch.randperm(N, generator=gen, device="cuda").int(), 0
    for s, (n, p) in enumerate(zip(new, starts)):
        c0, c1 = p // ps, -(-(p + n) // ps) if n else p // ps
        table[s, c0:c1] = perm[at:at + c1 - c0]
        at += c1 - c0
    ct = torch.float8_e4m3fn if cache == "fp8" else TYPES[kind]
    k, v = (torch.full((N, H, ps, D), 3.0, device="cuda").to(ct) for _ in range(2))
    return dict(q=fused[:, :heads], new_k=fused[:, heads:heads + H], new_v=fused[:, heads + H:], k_cache=k, v_cache=v, table=table,
                starts=ints(starts), offsets=ints(np.cumsum([0, *new]).tolist()), frequencies=rotary_frequencies(2 * pairs))


def check(a, what="", **kw):
    from paper_2609_12299_amd import append_tokens, rotate_tokens
    log(f"[gpu] rotate {what} {tuple(a['q'].shape)} {tuple(a['k_cache'].shape)} {a['k_cache'].dtype} {len(a['frequencies'])} pairs {sorted(kw)}")
    scales = {n: kw[n] for n in ("k_scale", "v_scale") if n in kw}
    k0, v0 = a["k_cache"].clone(), a["v_cache"].clone()
    q0, nk = a["q"].clone(), a["new_k"].clone()
    byte = lambda c: c.view(torch.uint8) if c.element_size() == 1 else c.view(torch.int16)  # noqa: E731
    # what the values' pages hold: as append_tokens writes them
    want_v, other = v0.clone(), v0.clone()
    append_tokens(a["new_k"], a["new_v"], other, want_v, a["table"], a["starts"], a["offsets"], **scales)
    got = rotate_tokens(**a, **kw)["out"]
    torch.cuda.synchronize()
    assert torch.equal(byte(a["v_cache"]), byte(want_v))
    T, D = got.shape[0], got.shape[2]
    seq, pos = ref.positions(a["starts"], a["offsets"], T)
    inter, amp = kw.get("interleaved", False), kw.get("amplitude", 1.0)
    half = ROUND[got.dtype]
    y, tol = ref.turn(q0, pos, a["frequencies"], inter, amp)
    mine = seq >= 0
    # (a result below the smallest normal number of 16 bits is off by half a step of those)
    off = np.abs(got.double().cpu().numpy() - y) - (half * 1.01 * np.abs(y) + tol + 2.0 ** -25)
    assert off[mine].size == 0 or off[mine].max() <= 0, off[mine].max()
    y, tol = ref.turn(nk, pos, a["frequencies"], inter, amp)
    k = a["k_cache"].double().cpu().numpy()
    tab, ps = a["table"].cpu().numpy(), k.shape[2]
    left = np.ones(k.shape[:3:2], bool)  # pages' places that nobody writes
    for r in range(T):
        if seq[r] < 0 or pos[r] < 0 or pos[r] // ps >= tab.shape[1] or not 0 <= tab[seq[r], pos[r] // ps] < len(k):
            continue
        page, place = tab[seq[r], pos[r] // ps], pos[r] % ps
        left[page, place] = False
        if a["k_cache"].element_size() == 1:
            s = kw["k_scale"].double().cpu().numpy()[:, None] if "k_scale" in kw else 1.0
            z = np.clip(y[r] / s, -448, 448)
            # three bits behind the first, or half a step of the smallest numbers
            allowed = 2.0 ** -4 * 1.01 * np.abs(z) + 2.0 ** -10 + 1.1 * tol[r] / s
        else:
            z, allowed = y[r], half * 1.01 * np.abs(y[r]) + tol[r] + 2.0 ** -25
        assert (np.abs(k[page, :, place] - z) <= allowed).all(), (r, np.abs(k[page, :, place] - z).max())
    left = torch.from_numpy(left).cuda()
    for c, c0 in ((a["k_cache"], k0), (a["v_cache"], v0)):
        assert torch.equal(byte(c).transpose(1, 2)[left], byte(c0).transpose(1, 2)[left])
    return got


@pytest.mark.parametrize("kind,cache", [("bf16", None), ("fp16", None), ("bf16", "fp8"), ("fp16", "fp8")])
@pytest.mark.parametrize("D,pairs", [(64, 32), (128, 64), (96, 48), (80, 40), (80, 20), (128, 32), (64, 1), (256, 128), (48, 21), (16, 8)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_and_parts(kind, cache, D, pairs, interleaved):
    kw = dict(k_scale=torch.tensor([0.02, 0.5], device="cuda"), v_scale=torch.tensor([0.3, 1.0], device="cuda")) if cache else {}
    check(build(kind, cache, D=D, pairs=pairs), what=f"{kind} {cache}", interleaved=interleaved, **kw)


def test_far_positions():
    """Angles of 10^6 radians and more, where 32 bits would be off by a twentieth of a turn."""
    check(build(new=(3, 4, 1), starts=(1000000, 123456, 999983), ps=64, D=128, pairs=64))
    a = build(new=(2, 3), starts=(0, 5))
    a["starts"] = ints([2 ** 31 - 5, 2 ** 31 - 3])
    check(a)  # (their pages are not held)


def test_amplitudes_and_stretched_contexts():
    from paper_2609_12299_amd import rotary_frequencies
    a = build(starts=(0, 9, 100000, 77, 130000))
    a["frequencies"] = rotary_frequencies(64, 500000.0, 8.0, original=8192)
    check(a, amplitude=1.25)
    a["frequencies"] = -rotary_frequencies(64, factor=4.0)
    check(a, amplitude=-0.5, interleaved=True)


def test_frequencies():
    from paper_2609_12299_amd import rotary_frequencies
    i = np.arange(16)
    plain = 10000.0 ** (-2 * i / 32)
    assert np.allclose(rotary_frequencies(32).cpu(), plain, rtol=1e-14)
    assert np.allclose(rotary_frequencies(32, factor=4.0).cpu(), plain / 4, rtol=1e-14)
    f = rotary_frequencies(32, factor=4.0, original=4096, slow=1, fast=32).cpu().numpy()
    turns = 4096 * plain / (2 * np.pi)
    assert np.allclose(f[turns >= 32], plain[turns >= 32]) and np.allclose(f[turns <= 1], plain[turns <= 1] / 4)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and ((f[mid] < plain[mid]) & (f[mid] > plain[mid] / 4)).all()


def test_one_row_per_sequence():
    a = build(new=(1, 1, 1, 1), starts=(0, 9, 1000, 77))
    assert a["offsets"].tolist() == [0, 1, 2, 3, 4]
    b = build(new=(1, 1, 1, 1), starts=(0, 9, 1000, 77))
    from paper_2609_12299_amd import rotate_tokens
    x = rotate_tokens(**a)["out"]
    y = rotate_tokens(**dict(b, offsets=None))["out"]
    assert torch.equal(x, y) and torch.equal(a["k_cache"], b["k_cache"]) and torch.equal(a["v_cache"], b["v_cache"])
    check(a)


@pytest.mark.parametrize("D,pairs,interleaved", [(64, 32, False), (64, 20, False), (64, 20, True), (80, 33, False)])
def test_in_place(D, pairs, interleaved):
    from paper_2609_12299_amd import rotate_tokens
    a = build(D=D, pairs=pairs)
    want = rotate_tokens(**a, interleaved=interleaved)["out"]
    got = rotate_tokens(**a, interleaved=interleaved, out=a["q"])["out"]
    assert got is a["q"] and torch.equal(got, want)


def test_queries_or_keys_alone():
    from paper_2609_12299_amd import rotate_tokens
    a, b = build(), build()
    want = rotate_tokens(**a)["out"]
    none = dict.fromkeys(("new_k", "new_v", "k_cache", "v_cache", "table"))
    assert torch.equal(rotate_tokens(**dict(b, **none))["out"], want)
    assert rotate_tokens(**dict(b, q=None)) == {}
    assert torch.equal(a["k_cache"], b["k_cache"]) and torch.equal(a["v_cache"], b["v_cache"])


def test_rows_without_a_place():
    """No sequence: not written.  No page, or a position below 0: the query alone."""
    from paper_2609_12299_amd import rotate_tokens
    a = build(new=(5, 8, 3), starts=(0, 20, 0))
    a["table"][1, 1] = -1
    a["table"][2, 0] = a["k_cache"].shape[0]
    a["starts"] = ints([-2, 20, 0])
    check(a)
    b = build(new=(5, 8, 3), starts=(0, 20, 0))
    b["offsets"] = ints([2, 5, 5, 9])
    out = torch.full_like(b["q"].contiguous(), 3.0)
    check(dict(b, out=out))
    assert (out[:2] == 3).all() and (out[9:] == 3).all()


def test_sizes_of_a_batch():
    """More rows than a block has in the small form, a sequence search over many, and none at all."""
    from paper_2609_12299_amd import rotate_tokens
    check(build(new=(4100, 7), starts=(3, 0), heads=2, H=1, D=16, pairs=8))
    check(build(new=tuple(i % 4 for i in range(300)), starts=tuple(7 * i for i in range(300)), heads=2, H=1, D=16, pairs=5))
    check(build(heads=65, H=1, D=64))
    a = build(new=(0, 0), starts=(3, 4))
    assert rotate_tokens(**a)["out"].shape == (0, 6, 64)


def test_graph_replays():
    from paper_2609_12299_amd import rotate_tokens
    a, b = build(), build()
    for x in (a, b):
        rotate_tokens(**x)
    torch.cuda.synchronize()
    out = torch.empty_like(a["q"].contiguous())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rotate_tokens(**a, out=out)
    for i in range(3):
        a["starts"].add_(1)  # the pages of the new places are partly not held: as eager
        b["starts"].add_(1)
        want = rotate_tokens(**b)["out"]
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(a["k_cache"], b["k_cache"])
