"""Decode-step operators beside autograd: what requires gradients is refused, what is written in place is
known to be written."""
from __future__ import annotations

import pytest

from gpu_util import log
from test_gpu_decode_streams import D, H, N, PS, call, inputs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

FLOATS = [("attend", "q"), ("attend", "k_cache"), ("attend", "v_cache"), ("append", "new_k"), ("append", "new_v"),
          ("select", "logits"), ("select", "scores")]


@pytest.mark.parametrize("op,name", FLOATS)
def test_gradients_are_refused(op, name):
    from paper_2609_12299_amd import ArgusError
    log(f"[gpu] gradients {op} {name}")
    a = inputs(op)
    want = call(op, a)
    a[name].requires_grad_()
    with pytest.raises(ArgusError, match="no backward pass"):
        call(op, a)
    with torch.no_grad():
        got = call(op, a)
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) and not got[n].requires_grad for n in want)


def test_caches_and_results_that_require_gradients():
    from paper_2609_12299_amd import ArgusError, append_tokens, attend_pages, compact_pages, step_pages
    log("[gpu] gradients of caches")
    new, a, s, c = inputs("append"), inputs("attend"), inputs("step"), inputs("compact")
    k, v, pool = (torch.zeros(2, N, H, PS, D, dtype=torch.bfloat16, device="cuda", requires_grad=True) for _ in range(3))
    scale = torch.ones(H, device="cuda", requires_grad=True)
    out = torch.zeros_like(a["q"], requires_grad=True)
    for run in (lambda: append_tokens(new["new_k"], new["new_v"], k[0], v.detach()[0], new["table"], new["starts"]),
                lambda: append_tokens(new["new_k"], new["new_v"], k.detach()[0], v[0], new["table"], new["starts"]),
                lambda: attend_pages(**a, k_scale=scale), lambda: attend_pages(**a, v_scale=scale),
                lambda: attend_pages(**a, out=out), lambda: step_pages(**s, page_size=PS, caches=(pool,)),
                lambda: compact_pages(**c, caches=(pool,))):
        with pytest.raises(ArgusError, match="no backward pass"):
            run()


def test_tensors_written_in_place_are_marked():
    """A backward pass that has kept a cache finds that it was written on, as for torch's own operators."""
    from paper_2609_12299_amd import append_tokens, attend_pages, compact_pages, step_pages
    log("[gpu] versions")
    new, a, s, c = inputs("append"), inputs("attend"), inputs("step"), inputs("compact")
    k, v = (torch.zeros(2, N, H, PS, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.zeros_like(a["q"])
    for run, changed in ((lambda: append_tokens(new["new_k"], new["new_v"], k[0], v[0], new["table"], new["starts"]), (k, v)),
                         (lambda: append_tokens(new["new_k"], new["new_v"], k[0], v[0], new["table"], new["starts"],
                                                stream=torch.cuda.current_stream()), (k, v)),
                         (lambda: step_pages(**s, page_size=PS, caches=(k, v)), (k, v)),
                         (lambda: compact_pages(**c, caches=(k,)), (k,)), (lambda: attend_pages(**a, out=out), (out,))):
        before = [x._version for x in changed]
        run()
        assert all(x._version == b + 1 for x, b in zip(changed, before))
    weight = torch.ones(D, device="cuda", requires_grad=True)
    loss = (k[0].float() * weight).sum() + (v[0, 0, 0, 0] * weight.bfloat16()).sum()
    append_tokens(new["new_k"], new["new_v"], k[0], v[0], new["table"], new["starts"])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    torch.cuda.synchronize()


def test_inference_mode():
    from paper_2609_12299_amd import append_tokens
    log("[gpu] inference mode")
    with torch.inference_mode():
        new = inputs("append")
        k, v = (torch.zeros(N, H, PS, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        append_tokens(new["new_k"], new["new_v"], k, v, new["table"], new["starts"])
        torch.cuda.synchronize()
        assert k.any() and v.any()
