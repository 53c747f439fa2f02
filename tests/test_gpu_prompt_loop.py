"""The operators of a prompt's pass together, with those of a decode step: chunks and single tokens in one
batch, a prompt's scores, markers, streams, graphs."""
from __future__ import annotations

import os
import sys

import numpy as np
import pytest

import test_gpu_prompt_attend as attend
import test_gpu_prompt_rotate as rotate
import test_gpu_prompt_score as score
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

ints = attend.ints
H, G, D, PS = 2, 3, 64, 16


def start(seqs, most, seed=0, kind=None):
    kind = kind or torch.bfloat16
    P = -(-most // PS)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.randperm(seqs * P + 5, generator=gen, device="cuda").int()[:seqs * P].view(seqs, P)
    caches = [torch.zeros((seqs * P + 5, H, PS, D), dtype=kind, device="cuda") for _ in range(2)]
    return gen, table, caches


def test_batches_of_chunks_and_single_tokens():
    """Four sequences over four passes: each takes a chunk, one token, or none. Every operator against 64 bits, on
    what the one before it left; single tokens also through attend_pages."""
    from paper_2609_12299_amd import attend_pages, rotary_frequencies
    passes = [(40, 1, 0, 129), (1, 33, 2, 0), (70, 1, 1, 1), (1, 1, 1, 1)]
    gen, table, (k, v) = start(4, 160)
    lens = np.zeros(4, np.int64)
    f = rotary_frequencies(48)
    for i, new in enumerate(passes):
        log(f"[gpu] pass {i} {new}")
        T = sum(new)
        fused = torch.randn((T, H * G + 2 * H, D), generator=gen, device="cuda").bfloat16()
        offsets, starts = ints(np.cumsum([0, *new]).tolist()), ints(lens.tolist())
        lens += new
        q = rotate.check(dict(q=fused[:, :H * G], new_k=fused[:, H * G:-H], new_v=fused[:, -H:], k_cache=k, v_cache=v, table=table,
                              starts=starts, offsets=offsets, frequencies=f), what=f"pass {i}")
        a = dict(q=q, k_cache=k, v_cache=v, table=table, lens=ints(lens.tolist()), offsets=offsets)
        out = attend.check(a, window=50, sinks=3)["out"]
        if min(new) == max(new) == 1:
            b = attend_pages(q, k, v, table, a["lens"], window=50, sinks=3)["out"]
            # two results of the same formula, each off by half a step of a value and of a weight
            assert ((out.float() - b.float()).abs() <= 4 * 2.0 ** -8 * v.float().abs().max()).all()
        logits = out.reshape(T, -1)
        score.check(logits, torch.randint(0, logits.shape[1], (T,), generator=gen, device="cuda").int(), 7, f"pass {i}")


def test_a_pass_in_a_graph():
    """The three operators captured once; what they read changes between replays, and eager passes come between them."""
    from paper_2609_12299_amd import attend_chunks, rotary_frequencies, rotate_tokens, score_tokens
    log("[gpu] a pass in a graph")
    new, past = (20, 1, 100), (0, 900, 3000)
    gen, table, (k, v) = start(3, 3200)
    k.copy_(torch.randn(k.shape, generator=gen, device="cuda")), v.copy_(torch.randn(v.shape, generator=gen, device="cuda"))
    T = sum(new)
    fused = torch.randn((T, H * G + 2 * H, D), generator=gen, device="cuda").bfloat16()
    starts, lens = ints(past), ints([n + p for n, p in zip(new, past)])
    offsets, f = ints(np.cumsum([0, *new]).tolist()), rotary_frequencies(D)
    tokens = torch.randint(0, H * G * D, (T,), generator=gen, device="cuda").int()

    def one():
        q = rotate_tokens(fused[:, :H * G], fused[:, H * G:-H], fused[:, -H:], k, v, table, starts, f, offsets)["out"]
        out = attend_chunks(q, k, v, table, lens, offsets, lse=True)
        return [q, *out.values(), *score_tokens(out["out"].view(T, -1), tokens, top=3).values()]
    one()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):  # two of them, over the same pool of memory
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=graphs[0][0].pool() if graphs else None):
            got = one()
        graphs.append((g, got))
    for i in range(4):
        fused.mul_(-0.8), tokens.add_(1)
        starts.sub_(1 if i else 0), lens.sub_(1 if i else 0)
        starts.clamp_(min=0), lens.clamp_(min=1)
        want = one()
        g, got = graphs[i % 2]
        for x in got:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)), i


def dense_scores(m, tokens):
    """Log probabilities of tokens[1:] in a forward pass over the whole sequence, 64 bits."""
    x = m.embed.double()[tokens]
    n = len(tokens)
    mask = torch.full((n, n), float("-inf"), dtype=torch.float64, device=tokens.device).triu(1)
    if m.frequencies is not None:
        a = torch.arange(n, device=tokens.device)[:, None, None] * m.frequencies
        c, s = torch.cos(a), torch.sin(a)

    def turn(y):
        if m.frequencies is None:
            return y
        y0, y1 = y.chunk(2, 2)
        return torch.cat([y0 * c - y1 * s, y1 * c + y0 * s], 2)
    for i in range(m.layers):
        qkv = (x @ m.qkv[i].double()).view(n, -1, m.head_dim)
        q, k, v = qkv.split([m.heads, m.kv_heads, m.kv_heads], 1)
        q, k = turn(q), turn(k)
        k, v = (t.repeat_interleave(m.heads // m.kv_heads, 1) for t in (k, v))
        w = (q.transpose(0, 1) @ k.permute(1, 2, 0).contiguous()) * m.head_dim ** -0.5 + mask
        o = torch.softmax(w, 2) @ v.transpose(0, 1).contiguous()
        x = x + o.transpose(0, 1).reshape(n, -1) @ m.out[i].double()
    logp = torch.log_softmax(x @ m.logits.double(), 1)
    return logp[torch.arange(n - 1, device=tokens.device), tokens[1:]]


@pytest.mark.parametrize("chunk,rotary,page", [(1, True, 16), (7, False, 8), (7, True, 16), (64, True, 32), (1000, False, 16)])
def test_prompts_in_chunks(chunk, rotary, page):
    """A prompt's scores and a search from it, whatever the chunks, are those of a dense pass."""
    from decode_loop import Model, read, search
    log(f"[gpu] prompts in chunks {chunk} {rotary} {page}")
    m = Model(layers=2, vocab=257, rotary=rotary)
    gen = torch.Generator(device="cuda").manual_seed(5)
    prompts = torch.randint(3, m.vocab, (3, 90), generator=gen, device="cuda")
    got = read(m, prompts, chunk, top=2, page_size=page)
    assert got["logprobs"].shape == (3, 89) and got["top_tokens"].shape == (3, 89, 2)
    for g in range(3):
        want = dense_scores(m, prompts[g])
        # 16-bit activations and logits: each log probability is off by about 2^-8 of logits of a few
        # units, in either direction
        assert abs(got["logprobs"][g].double().sum().item() - want.sum().item()) < 0.05 * 89
    tokens, scores, finished, d = search(m, prompts, 3, 5, page_size=page, chunk=chunk)
    for g in range(3):
        for b in range(3):
            want = dense_scores(m, tokens[g, b])[-5:].sum().item()
            assert abs(scores[g, b].item() - want) < 0.05 * 5, (g, b)


def test_markers():
    """One properly nested pair after the other per wave, and the same answers with and without."""
    from paper_2609_12299_amd import (NUM_ALL_REGIONS, PROMPT_REGION_NAMES, ArgusError, MarkerBuffer, RegionAttribution,
                                      attend_chunks, rotary_frequencies, rotate_tokens, score_tokens, to_host)
    log("[gpu] prompt markers")
    a = attend.build("bf16", sizes=[(300, 9000), (1, 20000), (0, 40)], D=128, G=4, ps=64, junk=False)
    short = attend.build("fp16", sizes=[(30, 100)], D=64, G=4, ps=16)
    long = attend.build("bf16", sizes=[(6000, 300)], H=4, D=128, G=4, ps=64, junk=False)
    r = rotate.build()
    x, t = score.build("bf16", 3, 300001)
    y, u = score.build("fp32", 900, 701)
    z, w = score.build("fp16", 3, 20000)

    def all_of_them(markers):
        caches = r["k_cache"].clone(), r["v_cache"].clone()
        got = rotate_tokens(r["q"], r["new_k"], r["new_v"], *caches, r["table"], r["starts"], r["frequencies"], r["offsets"],
                            markers=markers)
        out = [*caches, *got.values()]
        for b in (a, short, long):
            out += attend_chunks(**b, lse=True, markers=markers).values()
        out += score_tokens(x, t, 5, markers=markers).values()
        out += score_tokens(z, w, 2, markers=markers).values()
        return out + list(score_tokens(y, u, markers=markers).values())

    plain = all_of_them(None)
    m = MarkerBuffer(1 << 20, ctx_base=100, region_base=5)
    marked = all_of_them(m)
    torch.cuda.synchronize()
    for p, q in zip(plain, marked):
        assert torch.equal(p.float().nan_to_num(), q.float().nan_to_num())
    assert 0 < m.used < 1 << 20
    res = to_host(RegionAttribution(5 + NUM_ALL_REGIONS, max_records=m.used).run(m.records()))
    c = res["counters"]
    assert int(c[0]) == m.used and int(c[1]) == m.used and int(c[9]) == m.used // 2  # all valid, all matched
    assert int(c[10]) == int(c[11]) == int(c[12]) == int(c[13]) == int(c[31]) == 0
    counts = [int(n[0]) for n in res["region_stats"][5:]]
    assert not any(counts[:NUM_ALL_REGIONS - len(PROMPT_REGION_NAMES)])
    assert all(counts[NUM_ALL_REGIONS - len(PROMPT_REGION_NAMES):]), counts
    # a buffer that cannot take a call's records: refused, nothing written, nothing counted
    small = MarkerBuffer(m.used)
    small.c.used = m.used - 3
    before = small.buffer.clone()
    for call in (lambda: attend_chunks(**a, markers=small), lambda: score_tokens(x, t, markers=small),
                 lambda: rotate_tokens(r["q"], None, None, None, None, None, r["starts"], r["frequencies"], r["offsets"], markers=small)):
        with pytest.raises(ArgusError, match="marker records"):
            call()
    assert small.used == m.used - 3 and torch.equal(small.buffer, before)


def test_contexts_of_a_block():
    from paper_2609_12299_amd import ALL_REGION_NAMES, MarkerBuffer, attend_chunks, score_tokens
    log("[gpu] contexts of a block")
    m = MarkerBuffer(1 << 18, ctx_base=40)

    def contexts(region):
        torch.cuda.synchronize()
        words = m.records().cpu().numpy().view(np.uint32).reshape(-1, 4)
        return set(words[words[:, 3] & 0xFFFF == ALL_REGION_NAMES.index(region), 2].tolist())
    score_tokens(*score.build("bf16", 3, 20000), markers=m)
    assert m.used == 3 * 16 * 2 and contexts("score.rows") == set(range(40, 88))
    m.clear()
    score_tokens(*score.build("bf16", 3, 2000), markers=m)
    assert m.used == 3 * 4 * 2 and contexts("score.rows") == set(range(40, 52))
    m.clear()
    attend_chunks(**attend.build(sizes=[(10, 20)], H=2, G=3), markers=m)  # a row tile, a place for one more, two heads
    assert contexts("chunk") == set(range(40, 40 + m.used // 2)) and m.used == 2 * 4 * 2
    m.clear()
    attend_chunks(**attend.build(sizes=[(10, 3000)], H=2, G=3, junk=False), markers=m)
    assert contexts("chunk.plan") == set(range(40, 56)) and min(contexts("chunk")) == 40  # (each launch from ctx_base on)
    m.clear()
    attend_chunks(**attend.build(sizes=[(1100, 0)], H=128, G=1, D=128, ps=16, junk=False), markers=m)
    assert m.used == (1100 // 256 + 1) * 128 * 8 * 2


def inputs(op):
    if op == "chunks":
        return attend.build("bf16", junk=False)
    if op == "rotate":
        return rotate.build()
    x, t = score.build("bf16", 30, 20011)
    return dict(logits=x, tokens=t)


def call(op, a, stream=None):
    import paper_2609_12299_amd as fw
    if op == "chunks":
        return fw.attend_chunks(**a, lse=True, stream=stream)
    if op == "rotate":
        k, v = a["k_cache"], a["v_cache"]
        return dict(fw.rotate_tokens(**a, stream=stream), k=k, v=v)
    return fw.score_tokens(**a, top=4, stream=stream)


@pytest.mark.parametrize("op", ["chunks", "rotate", "score"])
def test_inputs_given_up_after_the_call(op):
    """On a stream of its own: the memory of what a call was given is not handed on while it may still read it."""
    log(f"[gpu] streams {op}")
    want = call(op, inputs(op))
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    a = inputs(op)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)  # the call's kernels come after the fills below
    got = call(op, a, stream)
    like = [(x.shape, x.dtype) for x in a.values()]
    a.clear()
    junk = [torch.full(shape, 1, dtype=dt, device="cuda") for shape, dt in like for _ in range(2)]
    torch.cuda.synchronize()
    mine = np.ones(len(want["out"]), bool) if op == "rotate" else slice(None)
    assert len(junk) and all(torch.equal(got[n][mine] if n == "out" else got[n], want[n][mine] if n == "out" else want[n]) for n in want)


@pytest.mark.parametrize("op", ["chunks", "rotate", "score"])
def test_two_streams_at_once(op):
    """Calls that overlap, each with its own workspace."""
    log(f"[gpu] two streams {op}")
    a, want = inputs(op), call(op, inputs(op))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(6):
        got.append(call(op, a, streams[i % 2]))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(g[n], want[n]) for n in want)


def test_gradients_are_refused_and_writes_are_seen():
    import paper_2609_12299_amd as fw
    log("[gpu] gradients")
    a, r = inputs("chunks"), inputs("rotate")
    x, t = score.build("fp32", 2, 100)
    with pytest.raises(fw.ArgusError, match="requires gradients"):
        fw.attend_chunks(**{**a, "q": a["q"].contiguous().requires_grad_()})
    with pytest.raises(fw.ArgusError, match="requires gradients"):
        fw.rotate_tokens(**{**r, "new_k": r["new_k"].contiguous().requires_grad_()})
    with pytest.raises(fw.ArgusError, match="requires gradients"):
        fw.score_tokens(x.requires_grad_(), t)
    with torch.no_grad():
        fw.score_tokens(x, t)
    # what a call writes counts as changed in place
    w = torch.ones_like(r["k_cache"], requires_grad=True)
    y = (w * r["k_cache"]).sum()
    before = r["k_cache"]._version
    fw.rotate_tokens(**r)
    assert r["k_cache"]._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    out = torch.zeros_like(a["q"].contiguous())
    before = out._version
    fw.attend_chunks(**a, out=out)
    assert out._version > before


def test_no_heads():
    from paper_2609_12299_amd import attend_chunks, rotate_tokens
    log("[gpu] no heads")
    a, r = inputs("chunks"), inputs("rotate")
    room = torch.full((4096,), 7.0, dtype=torch.bfloat16, device="cuda")
    none = room.as_strided((len(a["q"]), 0, 64), (0, 64, 1))
    got = attend_chunks(**{**a, "q": none}, lse=True, out=none)
    assert got["out"].shape == none.shape and got["lse"].shape == (len(a["q"]), 0)
    want = r["k_cache"].clone(), r["v_cache"].clone()
    rotate_tokens(**{**r, "k_cache": want[0], "v_cache": want[1]})
    assert rotate_tokens(**{**r, "q": r["q"][:, :0]})["out"].shape == (len(r["q"]), 0, 64)
    assert torch.equal(r["k_cache"], want[0]) and torch.equal(r["v_cache"], want[1]) and (room == 7).all()


def test_example_runs():
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "decode_loop.py"), "--steps", "4", "--groups", "2",
                        "--prompt", "40", "--chunk", "16", "--rotary"], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "0 mismatched, 0 unclosed, 0 orphans" in r.stdout
    assert all(name in r.stdout for name in ("nats a token", "chunk", "rotate", "score.rows", "attend.tokens"))
