"""Calls that use a workspace: two at once on streams of their own, and inputs given up after the call."""
from __future__ import annotations

import pytest

import test_gpu_prompt_attend as attend
import test_gpu_prompt_score as score
from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def inputs(op, i):
    """Two inputs of one shape (so that each would fit the other's workspace), with other plans and answers."""
    if op == "chunks":  # the row tiles of both sequences are cut, in pieces of other lengths
        return attend.build("bf16", H=2, G=4, D=128, ps=64, sizes=[[(16, 20000), (5, 9000)], [(5, 9000), (16, 20000)]][i], seed=i, junk=False)
    if op == "chunks of 256 rows":
        return attend.build("bf16", H=64, G=1, D=128, ps=64, sizes=[[(2100, 0), (30, 15000)], [(30, 15000), (2100, 0)]][i], seed=i, junk=False)
    x, t = score.build("bf16", 3, 300001, seed=i)
    return dict(logits=x, tokens=t)


def call(op, a, stream=None):
    import paper_2609_12299_amd as fw
    if op == "score":
        return fw.score_tokens(**a, top=5, stream=stream)
    return fw.attend_chunks(**a, lse=True, stream=stream)


@pytest.fixture
def needs(monkeypatch):
    """The sizes of the workspaces that calls ask for."""
    from paper_2609_12299_amd import prompt
    seen, real = [], prompt._workspace

    def spy(need, ints):
        seen.append(need)
        return real(need, ints)
    monkeypatch.setattr(prompt, "_workspace", spy)
    return seen


OPS = ["chunks", "chunks of 256 rows", "score"]


@pytest.mark.parametrize("op", OPS)
def test_two_streams_at_once(op, needs):
    log(f"[gpu] two streams {op}")
    both = [inputs(op, i) for i in range(2)]
    want = [call(op, a) for a in both]
    assert not all(torch.equal(want[0][n], want[1][n]) for n in want[0])
    torch.cuda.synchronize()
    streams, gate = [torch.cuda.Stream() for _ in range(3)], torch.cuda.Event()
    with torch.cuda.stream(streams[2]):
        torch.cuda._sleep(40_000_000)
        gate.record()
    for s in streams[:2]:  # both begin once all calls are enqueued
        s.wait_event(gate)
    got = [(i % 2, call(op, both[i % 2], streams[i % 2])) for i in range(8)]
    torch.cuda.synchronize()
    assert len(needs) == 10 and min(needs) > 0
    for i, g in got:
        assert all(torch.equal(g[n], want[i][n]) for n in g)


@pytest.mark.parametrize("op", OPS)
def test_inputs_and_workspaces_given_up_after_the_call(op, needs):
    log(f"[gpu] given up {op}")
    want = call(op, inputs(op, 0))
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    a = inputs(op, 0)
    like = [(x.shape, x.dtype) for x in a.values()]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(40_000_000)  # the call's kernels come after the fills below
    got = call(op, a, stream)
    assert min(needs) > 0
    a.clear()
    junk = [torch.full(shape, 1, dtype=dt, device="cuda") for shape, dt in like for _ in range(2)]
    junk += [torch.full(((needs[-1] + 259) // 4,), -1, dtype=torch.int32, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert len(junk) and all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("op", OPS)
def test_two_graphs_of_one_pool(op, needs):
    """Captured calls whose workspaces lie in one pool, replayed in turns with eager calls between them."""
    log(f"[gpu] two graphs {op}")
    both = [inputs(op, i) for i in range(2)]
    want = [call(op, a) for a in both]
    torch.cuda.synchronize()
    graphs = []
    for a in both:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=graphs[0][0].pool() if graphs else None):
            got = call(op, a)
        graphs.append((g, got))
    assert min(needs) > 0
    for i in (0, 1, 1, 0, 0, 1):
        g, got = graphs[i]
        for x in got.values():
            x.zero_()
        g.replay()
        call(op, both[1 - i])
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[i][n]) for n in got)
