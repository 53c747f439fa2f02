"""The operators together: beam search over a paged cache, its bookkeeping against a dense forward
pass in 64 bits, and the markers that the operators write."""
from __future__ import annotations

import os
import sys

import numpy as np
import pytest

from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def dense_scores(m, tokens, first):
    """Sum of the log probabilities of tokens[first:] in a forward pass over the whole sequence, 64 bits."""
    w = lambda t: t.double()  # noqa: E731
    x = w(m.embed)[tokens]
    n = len(tokens)
    mask = torch.full((n, n), float("-inf"), dtype=torch.float64, device=tokens.device).triu(1)
    for i in range(m.layers):
        qkv = (x @ w(m.qkv[i])).view(n, -1, m.head_dim)
        q, k, v = qkv.split([m.heads, m.kv_heads, m.kv_heads], 1)
        k, v = (t.repeat_interleave(m.heads // m.kv_heads, 1) for t in (k, v))
        s = (q.transpose(0, 1) @ k.permute(1, 2, 0).contiguous()) * m.head_dim ** -0.5 + mask
        o = torch.softmax(s, 2) @ v.transpose(0, 1).contiguous()
        x = x + o.transpose(0, 1).reshape(n, -1) @ w(m.out[i])
    logp = torch.log_softmax(x @ w(m.logits), 1)
    return logp[torch.arange(first - 1, n - 1, device=tokens.device), tokens[first:]].sum().item()


@pytest.mark.parametrize("prompt,steps,beams,page", [(5, 40, 4, 16), (37, 9, 3, 8), (1, 20, 1, 32)])
def test_scores_are_those_of_the_tokens(prompt, steps, beams, page):
    """A beam's score is the sum of its own tokens' log probabilities: pages that were shared, copied
    or reordered wrongly would show."""
    from decode_loop import Model, search
    log(f"[gpu] decode loop {prompt} {steps} {beams} {page}")
    m = Model(layers=2, vocab=257)
    gen = torch.Generator(device="cuda").manual_seed(3)
    prompts = torch.randint(3, m.vocab, (3, prompt), generator=gen, device="cuda")
    tokens, scores, finished, d = search(m, prompts, beams, steps, page_size=page)
    assert torch.isfinite(scores).all() and not finished.any()
    for g in range(3):
        assert len({tuple(t) for t in tokens[g].tolist()}) == beams  # no two alike
        for b in range(beams):
            want = dense_scores(m, tokens[g, b], prompt)
            # 16-bit activations and logits: each log probability is off by about 2^-8 of logits of a few
            # units, in either direction
            assert abs(scores[g, b].item() - want) < 0.05 * steps, (g, b)
        assert (scores[g, :-1] >= scores[g, 1:]).all()
    d.compact()
    used = int((d.refs > 0).sum())
    assert (d.refs[:used] > 0).all() and (d.table < used).all()


def test_markers():
    """One properly nested pair after the other per wave, and the same answers with and without."""
    from paper_2609_12299_amd import (NUM_REGIONS, REGION_NAMES, ArgusError, MarkerBuffer, RegionAttribution,
                                      append_tokens, attend_pages, compact_pages, select_beams, step_pages, to_host)
    log("[gpu] decode markers")
    S, H, G, D, ps, P, N = 24, 2, 4, 64, 16, 80, 4500
    gen = torch.Generator(device="cuda").manual_seed(1)
    caches = [torch.randn((2, N, H, ps, D), generator=gen, device="cuda").bfloat16() for _ in range(2)]
    lens = torch.randint(0, P * ps - 1, (S,), generator=gen, device="cuda").int()
    table = torch.randint(0, 100, (S, P), generator=gen, device="cuda").int()
    parents = torch.randint(-1, S, (S,), generator=gen, device="cuda").int()
    one = torch.ones(S, dtype=torch.int32, device="cuda")
    q = torch.randn((S, H * G, D), generator=gen, device="cuda").bfloat16()
    new = torch.randn((S, 2, H, D), generator=gen, device="cuda").bfloat16()
    logits = torch.randn((6, 4, 3001), generator=gen, device="cuda")
    scores = torch.zeros((6, 4), device="cuda")

    def all_of_them(markers):
        c = [x.clone() for x in caches]
        out = step_pages(table, lens, parents, one, ps, caches=c, markers=markers)
        append_tokens(new[:, 0], new[:, 1], c[0][1], c[1][1], out["table"], out["lens"] - 1, markers=markers)
        a = attend_pages(q, c[0][1], c[1][1], out["table"], out["lens"], lse=True, markers=markers)
        short = attend_pages(q, c[0][0], c[1][0], out["table"][:, :4], out["lens"], lse=True, markers=markers)
        few = step_pages(out["table"][:4, :8], (out["lens"] % 100)[:4].contiguous(), None, one[:4], ps, num_pages=500,
                         markers=markers)
        com = compact_pages(out["table"], out["refs"], caches=c, markers=markers)
        tidy = compact_pages(few["table"], few["refs"], markers=markers)
        sel = select_beams(logits, scores, 4, markers=markers)
        return [*c, *out.values(), *a.values(), *short.values(), *few.values(), *com.values(), *tidy.values(), *sel.values()]

    plain = all_of_them(None)
    m = MarkerBuffer(1 << 20, ctx_base=100, region_base=5)
    marked = all_of_them(m)
    torch.cuda.synchronize()
    for x, y in zip(plain, marked):
        assert torch.equal(x.float().nan_to_num(), y.float().nan_to_num())
    rec = m.records()
    assert 0 < m.used < 1 << 20
    run = RegionAttribution(5 + NUM_REGIONS, max_records=m.used)
    res = to_host(run.run(rec))
    c = res["counters"]
    assert int(c[0]) == m.used and int(c[1]) == m.used and int(c[9]) == m.used // 2  # all valid, all matched
    assert int(c[10]) == int(c[11]) == int(c[12]) == int(c[13]) == int(c[31]) == 0
    assert int(c[14]) == 1 and int(c[16]) == 100
    counts = {n: int(res["region_stats"][5 + r][0]) for r, n in enumerate(REGION_NAMES)}
    assert all(counts.values()), counts
    assert counts["attend"] == counts["attend.place"] == counts["attend.tokens"]
    inner = [r for r, n in enumerate(REGION_NAMES) if "attend." in n and n != "attend.join"]
    level = res["instances"]["level"]
    assert set(np.unique(res["instances"]["region_id"][level == 1]) - 5) == set(inner)
    # a buffer that cannot take a call's records: refused, nothing written, nothing counted
    small = MarkerBuffer(m.used, region_base=0)
    small.c.used = m.used - 3
    before = small.buffer.clone()
    with pytest.raises(ArgusError, match="marker records"):
        select_beams(logits, scores, 4, markers=small)
    assert small.used == m.used - 3 and torch.equal(small.buffer, before)


def test_example_runs():
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "decode_loop.py"), "--steps", "6", "--groups", "2",
                        "--prompt", "20"], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "0 mismatched, 0 unclosed, 0 orphans" in r.stdout and "attend.tokens" in r.stdout


def test_contexts_of_a_block():
    """Four contexts are a block, sixteen in a step that is one launch."""
    from paper_2609_12299_amd import REGION_NAMES, MarkerBuffer, select_beams, step_pages
    log("[gpu] contexts of a block")
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    m = MarkerBuffer(1 << 16, ctx_base=40)

    def contexts(region):
        torch.cuda.synchronize()
        words = m.records().cpu().numpy().view(np.uint32).reshape(-1, 4)
        m.clear()
        return set(words[words[:, 3] & 0xFFFF == REGION_NAMES.index(region), 2].tolist())
    step_pages(ints(0, 1).view(2, 1), ints(3, 4), None, ints(1, 1), 16, num_pages=100, markers=m)
    assert m.used == 16 * 4 and contexts("step.plan") == set(range(40, 56))
    step_pages(ints(0, 1).view(2, 1), ints(3, 4), None, ints(1, 1), 16, num_pages=5000, markers=m)
    assert contexts("step.claim") == set(range(40, 44))
    select_beams(torch.zeros(3, 2, 100, device="cuda"), torch.zeros(3, 2, device="cuda"), 2, markers=m)
    assert contexts("select.beams") == set(range(40, 52))
