"""Decode-step operators on a stream of their own: the memory of what they were given is not handed on
while they may still read it."""
from __future__ import annotations

import pytest

from gpu_util import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def ints(*shape, below, seed):
    return torch.randint(0, below, shape, generator=torch.Generator().manual_seed(seed)).int().cuda()


def randoms(*shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).cuda()


S, P, N, H, D, PS = 8, 40, 400, 2, 64, 16


def table():
    return torch.randperm(N, generator=torch.Generator().manual_seed(1))[:S * P].reshape(S, P).int().cuda()


def inputs(op):
    if op == "attend":
        return dict(q=randoms(S, 8, D, seed=2).bfloat16(), k_cache=randoms(N, H, PS, D, seed=3).bfloat16(),
                    v_cache=randoms(N, H, PS, D, seed=4).bfloat16(), table=table(), lens=ints(S, below=P * PS, seed=5))
    if op == "append":
        return dict(new_k=randoms(S, H, D, seed=2).bfloat16(), new_v=randoms(S, H, D, seed=3).bfloat16(), table=table(),
                    starts=ints(S, below=P * PS, seed=5))
    if op == "step":
        return dict(table=table(), lens=ints(S, below=P * PS, seed=5), parents=ints(S, below=S, seed=6),
                    grow=ints(S, below=40, seed=7), held=ints(N, below=2, seed=8))
    if op == "compact":
        return dict(table=table(), refs=ints(N, below=2, seed=8))
    return dict(logits=randoms(S, 4, 5000, seed=2), scores=randoms(S, 4, seed=3),
                finished=ints(S, 4, below=5, seed=4) == 0)


def call(op, a, stream=None):
    import paper_2609_12299_amd as fw
    if op == "attend":
        return fw.attend_pages(**a, lse=True, stream=stream)
    if op == "append":
        k, v = (torch.zeros(N, H, PS, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        fw.append_tokens(a["new_k"], a["new_v"], k, v, a["table"], a["starts"], stream=stream)
        return dict(k=k, v=v)
    if op == "step":
        return fw.step_pages(**a, page_size=PS, stream=stream)
    if op == "compact":
        return fw.compact_pages(**a, stream=stream)
    return fw.select_beams(**a, k=4, eos=2, stream=stream)


@pytest.mark.parametrize("op", ["attend", "append", "step", "compact", "select"])
def test_inputs_given_up_after_the_call(op):
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
    assert len(junk) and all(torch.equal(got[n], want[n]) for n in want)
