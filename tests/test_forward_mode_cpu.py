"""Forward-mode derivatives: the operators have none, so a tensor with a tangent is refused (results without one would pass for
constants). On the CPU, before any launch."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")


def calls():
    """(name of the tensor that gets a tangent, the call with it), one for each tensor of each operator."""
    import paper_2609_12299_amd as fw
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    c, f = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.ones(32, dtype=torch.float64)
    tab, three, two, one = torch.zeros(3, 2).int(), torch.zeros(3).int(), torch.tensor([0, 3]).int(), torch.zeros(1).int()
    scale, x, s = torch.ones(2), torch.zeros(3, 50), torch.zeros(1, 3)
    pool = torch.zeros(2, 3, 2, 16, 64, dtype=torch.bfloat16)
    pages = dict(q=q, k_cache=c, v_cache=c, table=tab, lens=three)
    append = dict(new_k=k, new_v=k, k_cache=c, v_cache=c, table=tab, starts=three)
    chunks = dict(q=q, k_cache=c, v_cache=c, table=tab[:1], lens=one, offsets=two)
    rotate = dict(q=q, new_k=k, new_v=k, k_cache=c, v_cache=c, table=tab[:1], starts=one, frequencies=f, offsets=two)
    floats = {"k_scale": scale, "v_scale": scale}
    for op, a, more in ((fw.attend_pages, pages, dict(floats, out=q)), (fw.append_tokens, append, floats),
                        (fw.attend_chunks, chunks, dict(floats, out=q)), (fw.rotate_tokens, rotate, dict(floats, out=q)),
                        (fw.score_tokens, dict(logits=x, tokens=three), {}),
                        (fw.select_beams, dict(logits=x[None], scores=s, k=2), {})):
        for name, t in {**a, **more}.items():
            if getattr(t, "is_floating_point", bool)():
                yield op, {**a, name: t}, name
    yield fw.step_pages, dict(table=tab, lens=three, parents=None, grow=None, page_size=16, caches=(pool,)), "caches"
    yield fw.compact_pages, dict(table=tab, refs=three, caches=(pool,)), "caches"


@pytest.fixture
def went_on(monkeypatch):
    """The wrappers take tensors on the CPU, and no call reaches the library (on a machine with a GPU it would read them)."""
    from paper_2609_12299_amd import decode, prompt
    prompt._t()
    seen = []
    for m, names in ((decode, ("attend", "append", "step", "compact", "select")), (prompt, ("attend", "rotate", "score"))):
        monkeypatch.setattr(m, "_elsewhere", lambda stream, dev: False)
        for name in names:
            monkeypatch.setattr(m, "_lib_" + name, lambda *args, op=f"{m.__name__}.{name}": seen.append(op) or 0)
    monkeypatch.setattr(decode, "_raw_stream", lambda index: 0)
    return seen


def test_tangents_are_refused(went_on):
    import torch.autograd.forward_ad as forward

    from paper_2609_12299_amd import ArgusError
    n = 0
    for op, a, name in calls():
        with forward.dual_level():
            def dual(x):
                return forward.make_dual(x.clone(), torch.ones_like(x))
            b = {**a, name: tuple(map(dual, a[name])) if name == "caches" else dual(a[name])}
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(ArgusError, match="tangent"):
                    op(**b)
        n += 1
    assert n == 6 + 6 + 6 + 9 + 1 + 2 + 2 and not went_on


def test_plain_tensors_within_a_level_pass(went_on):
    import torch.autograd.forward_ad as forward
    with forward.dual_level():
        for op, a, name in calls():
            op(**a)
    assert len(went_on) == 32 and len(set(went_on)) == 8
