"""What the operators of a prompt's pass are measured on: attention of chunks of new tokens over a
paged cache, rotary positions of queries and of keys on their way into the pages, and the scores of
given tokens (log probability, entropy, rank, best alternatives).

A case is one call of one operator.  `run` computes it either in plain torch, in 32 bits, or with
the library's kernels (`own`); `exact` gives the defined values in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

KINDS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32,
         "fp8": torch.float8_e4m3fn}
FP8_MAX = 448.0


# ------------------------------------------------------------------- cases
#
# new: new tokens of a sequence, past: tokens that it has in the cache already, each from the first
# number to the second, evenly over their logarithm.

def _attend(name, kind, seqs, new, past, kv_heads, group, dim, page, window=0, sinks=0):
    c = dict(op="attend", kind=kind, seqs=seqs, new_least=new[0], new_most=new[1], past_least=past[0],
             past_most=past[1], kv_heads=kv_heads, group=group, dim=dim, page=page, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _rotate(name, kind, source, seqs, new, past, heads, kv_heads, dim, rotated, page, interleaved, factor=1.0):
    c = dict(op="rotate", kind=kind, source=source, seqs=seqs, new_least=new[0], new_most=new[1],
             past_least=past[0], past_most=past[1], heads=heads, kv_heads=kv_heads, dim=dim, rotated=rotated,
             page=page, interleaved=interleaved, factor=factor)
    return dict(c, name=name) if name else c


def _score(name, kind, rows, vocab, top, masked=0):
    c = dict(op="score", kind=kind, rows=rows, vocab=vocab, top=top, masked=masked)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's short question, all of it new: launches count
        _attend("attend_short_prompt", "bf16", 1, (45, 45), (0, 0), 4, 8, 64, 16),
        # a serving batch in which answers under way (one new token) run beside prompts in chunks, with
        # a window over the last 4096 tokens and four first tokens that stay visible; an odd head size
        _attend("attend_mixed_window", "fp16", 40, (1, 700), (1, 9000), 8, 5, 96, 32, 4096, 4),
        # prompts taken in chunks of 512 over a cache held in 8 bits
        _attend("attend_chunks_fp8", "fp8", 16, (512, 512), (512, 15872), 8, 8, 128, 64),
        # a long prompt in one pass: the product of queries and keys is what it costs
        _attend("attend_long_prompt", "bf16", 1, (16384, 16384), (0, 0), 8, 8, 128, 64),
        # a few proposed tokens of long documents checked at once: the cache's length is what it costs
        _attend("attend_proposals", "bf16", 4, (6, 6), (131000, 131000), 8, 8, 128, 64),
        # the new token of every sequence of a decode step, far into their texts
        _rotate("rotate_step", "bf16", "bf16", 64, (1, 1), (100, 100000), 32, 8, 128, 128, 16, False),
        # prompts of all lengths into a cache of 8 bits; a part of the head turns, neighbours in pairs
        _rotate("rotate_prompts_fp8", "fp8", "bf16", 40, (1, 8192), (0, 512), 32, 8, 128, 64, 64, True),
        # a long prompt far into a context that was stretched: angles of positions beyond 10^6
        _rotate("rotate_far", "fp16", "fp16", 1, (65537, 65537), (1000000, 1000000), 24, 8, 96, 96, 32, False, 8.0),
        # one new token's score and five alternatives
        _score("score_one", "bf16", 1, 32000, 5),
        # the scores of a prompt's tokens over a large vocabulary of odd size, with alternatives
        _score("score_prompt", "bf16", 2048, 128003, 20),
        # scores alone, in 32 bits; a part of the vocabulary is not allowed (minus infinity)
        _score("score_masked", "fp32", 500, 65537, 0, 1000),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "rotate", "rotate", "score", "score"])
    if op == "attend":
        kind, kv_heads = rng.choice(["bf16", "fp16", "fp8"]), rng.choice([1, 2, 4, 8])
        group, dim = rng.choice([1, 2, 4, 5, 7, 8, 16]), rng.choice([64, 80, 96, 128, 256])
        seqs = _between(rng, 1, 64)
        past = rng.choice([0, _between(rng, 1, 131072)])
        past = min(past, (1 << 27) // (seqs * kv_heads * dim))
        new = _between(rng, 1, 8192)
        while seqs * kv_heads * group * new * (new + past) * dim > 1 << 39 or seqs * kv_heads * (new + past) * dim > 1 << 28:
            new = (new + 1) // 2
        window = rng.choice([0, 0, _between(rng, 16, 8192)])
        return _attend("", kind, seqs, (rng.choice([0, 1, new]), new), (rng.choice([0, past]), past), kv_heads, group,
                       dim, rng.choice([8, 16, 32, 64, 128]), window, rng.choice([0, 1, 4, 64]) if window else 0)
    if op == "rotate":
        kind = rng.choice(["bf16", "fp16", "fp8"])
        source = rng.choice(["bf16", "fp16"]) if kind == "fp8" else kind
        kv_heads, dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 256])
        heads = kv_heads * rng.choice([1, 2, 4, 7])
        seqs = _between(rng, 1, 96)
        new = min(rng.choice([1, _between(rng, 2, 65536)]), 240000000 // (seqs * (heads + 2 * kv_heads) * dim))
        past = rng.choice([0, _between(rng, 1, 1000000)])
        return _rotate("", kind, source, seqs, (rng.choice([0, 1, new]), new), (rng.choice([0, past]), past), heads,
                       kv_heads, dim, rng.choice([dim, dim, dim // 2, dim // 4 * 2]), rng.choice([8, 16, 32, 64, 128]),
                       rng.choice([False, True]), rng.choice([1.0, 4.0, 32.0]))
    kind = rng.choice(["bf16", "fp16", "fp32"])
    vocab = _between(rng, 1000, 200003)
    rows = _between(rng, 1, max(1, min(4096, (1 << (27 if kind == "fp32" else 28)) // vocab)))
    return _score("", kind, rows, vocab, rng.choice([0, 1, 5, 20, 64]), rng.choice([0, 0, vocab // 3]))


# ------------------------------------------------------------------ inputs

def _spread(n, lo, hi):
    """n numbers from the least to the most, evenly over their logarithm; the same for every seed."""
    if n == 1 or lo == hi:
        return [hi] * n
    a, b = math.log(lo + 1), math.log(hi + 1)
    return [int(round(math.exp(a + (b - a) * i / (n - 1)))) - 1 for i in range(n)]


def _sizes(case, seed):
    """(new, past) of each sequence.  Which past goes with which number of new tokens is the same for
    every seed (so is the work), the order of the sequences is not."""
    new = _spread(case["seqs"], case["new_least"], case["new_most"])
    past = _spread(case["seqs"], case["past_least"], case["past_most"])
    random.Random(1).shuffle(past)
    both = list(zip(new, past))
    random.Random(seed).shuffle(both)
    return [n for n, _ in both], [p for _, p in both]


def _random(shape, gen, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16 if dtype == KINDS["fp8"] else dtype).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(new):
    ends = [0]
    for n in new:
        ends.append(ends[-1] + n)
    return _ints(ends)


def _table(used, gen):
    """Page tables of sequences that share nothing: pages of a pool in random order, -1 where none is used."""
    count = int(used.sum())
    pages = count + count // 16 + 1
    table = torch.full(used.shape, -1, dtype=torch.int32, device="cuda")
    table[used] = torch.randperm(pages, generator=gen, device="cuda")[:count].int()
    return table, pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return dict({"attend": _prepare_attend, "rotate": _prepare_rotate, "score": _prepare_score}[case["op"]](case, seed, gen),
                op=case["op"])


def _prepare_attend(case, seed, gen):
    H, D, ps, window, sinks = case["kv_heads"], case["dim"], case["page"], case["window"], case["sinks"]
    new, past = _sizes(case, seed)
    lens = _ints([a + b for a, b in zip(new, past)])
    columns = max(1, -(-int(lens.max()) // ps))
    col = torch.arange(columns, device="cuda")
    used = col * ps < lens[:, None]
    if window:  # pages that no query sees any more have been given back
        used &= ((col + 1) * ps > _ints(past)[:, None] + 1 - window) | (col * ps < sinks)
    table, pages = _table(used, gen)
    kind = KINDS[case["kind"]]
    k, v = (_random((pages, H, ps, D), gen, kind) for _ in range(2))
    # what lies behind a sequence's end in its last page was never written: anything, NaN too
    some = torch.nonzero(lens % ps)[:, 0]
    last = table[some, (lens[some] // ps).long()].long()
    junk = torch.arange(ps, device="cuda") >= (lens[some] % ps)[:, None]
    for c in (k, v):
        tail = c[last].float()
        c[last] = tail.masked_fill_(junk[:, None, :, None], float("nan")).to(kind)
    # queries as a fused projection leaves them, keys and values of the same rows behind them
    heads = H * case["group"]
    fused = _random((max(sum(new), 1), heads + 2 * H, D), gen, torch.float16 if case["kind"] == "fp16" else torch.bfloat16)
    state = dict(q=fused[:sum(new), :heads], k=k, v=v, table=table, lens=lens, offsets=_offsets(new), most=max(new),
                 window=window, sinks=sinks, scale=D ** -0.5, k_scale=None, v_scale=None)
    if case["kind"] == "fp8":
        state.update({n: torch.rand(H, generator=gen, device="cuda") + 0.5 for n in ("k_scale", "v_scale")})
    return state


def _frequencies(rotated, factor):
    """Radians per token of each pair.  A context stretched by a factor: pairs that turn often over the
    first 8192 tokens stay, those that do not come round are slowed down by it, others in between."""
    i = torch.arange(rotated // 2, dtype=torch.float64, device="cuda")
    f = 10000.0 ** (-2 * i / rotated)
    turns = 8192 * f / (2 * math.pi)
    keep = ((turns - 1) / 31).clamp(0, 1) if factor != 1.0 else 1.0
    return f / factor * (1 - keep) + f * keep if factor != 1.0 else f


def _prepare_rotate(case, seed, gen):
    H, D, ps, heads = case["kv_heads"], case["dim"], case["page"], case["heads"]
    new, past = _sizes(case, seed)
    T = sum(new)
    fused = _random((max(T, 1), heads + 2 * H, D), gen, KINDS[case["source"]])[:T]
    # pages of the new tokens alone: those of the past are none of this call's business
    columns = max(1, -(-max(a + b for a, b in zip(new, past)) // ps))
    first, ends = _ints(past)[:, None], _ints([a + b for a, b in zip(new, past)])[:, None]
    col = torch.arange(columns, device="cuda")
    table, pages = _table(((col + 1) * ps > first) & (col * ps < ends), gen)
    most = sum(-(-n // ps) + 1 for n in new)
    kind = KINDS[case["kind"]]
    k, v = (torch.zeros((max(pages, most), H, ps, D), dtype=kind, device="cuda") for _ in range(2))
    state = dict(q=fused[:, :heads], new_k=fused[:, heads:heads + H], new_v=fused[:, heads + H:], k=k, v=v, table=table,
                 starts=_ints(past), offsets=_offsets(new), single=case["new_least"] == case["new_most"] == 1,
                 frequencies=_frequencies(case["rotated"], case["factor"]), interleaved=case["interleaved"],
                 amplitude=1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0, k_scale=None, v_scale=None)
    if case["kind"] == "fp8":
        state.update({n: torch.rand(H, generator=gen, device="cuda") * 0.05 + 0.01 for n in ("k_scale", "v_scale")})
    return state


def _prepare_score(case, seed, gen):
    """Logits as a product leaves them, tokens as such a model would choose them; some of the vocabulary
    may not be chosen."""
    R, V = case["rows"], case["vocab"]
    logits = (torch.randn((R, V), generator=gen, device="cuda") * 2.5).to(KINDS[case["kind"]])
    if case["masked"]:
        logits[:, torch.randperm(V, generator=gen, device="cuda")[:case["masked"]]] = -math.inf
    noise = torch.empty((R, V), device="cuda").exponential_(generator=gen)
    tokens = (logits.float() - torch.log(noise)).argmax(1).int()
    return dict(logits=logits, tokens=tokens, top=case["top"])


# ------------------------------------------------------------- plain forms

def _plain_attend(s):
    q, k, v, table, lens = s["q"], s["k"], s["v"], s["table"], s["lens"].long()
    rows, heads, D = q.shape
    H, ps = k.shape[1], k.shape[2]
    S, G, dev = len(lens), heads // H, q.device
    first = s["offsets"].long()
    n = first[1:] - first[:-1]
    at = torch.arange(table.shape[1] * ps, device=dev)
    page = table.clamp(min=0).long()
    there = (at < lens[:, None]) & (table >= 0).repeat_interleave(ps, 1)

    def tokens_of(c, scale):  # [S, H, tokens, D] in 32 bits, nothing where there is none
        x = c[page].transpose(1, 2).reshape(S, H, -1, D).float()
        x = x if scale is None else x * scale[:, None, None]
        return x.masked_fill_(~there[:, None, :, None], 0.0)

    kt = tokens_of(k, s["k_scale"]).transpose(2, 3).contiguous()
    vt = tokens_of(v, s["v_scale"])
    out = torch.empty((rows + 1, heads, D), device=dev)
    lse = torch.empty((rows + 1, heads), device=dev)
    # as many queries of every sequence at a time as leave room for their scores
    step = max(1, min(s["most"], (1 << 31) // max(1, S * heads * len(at))))
    for i0 in range(0, s["most"], step):
        i = torch.arange(i0, min(i0 + step, s["most"]), device=dev)
        real = i < n[:, None]
        row = torch.where(real, first[:-1, None] + i, rows)
        pos = (lens - n)[:, None] + i
        seen = there[:, None] & (at <= pos[..., None])
        if s["window"]:
            seen &= (at > pos[..., None] - s["window"]) | (at < s["sinks"])
        qi = q[row.clamp(max=max(rows - 1, 0))].float().reshape(S, len(i), H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, -1, D)
        score = ((qi.contiguous() @ kt) * s["scale"]).reshape(S, H, G, len(i), -1)
        score.masked_fill_(~seen[:, None, None], -math.inf)
        top = score.amax(-1, keepdim=True)
        p = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
        total = p.sum(-1, keepdim=True)
        o = (p.reshape(S, H, -1, len(at)) @ vt).reshape(S, H, G, len(i), D) / torch.where(total == 0, 1.0, total)
        out[row] = o.permute(0, 3, 1, 2, 4).reshape(S, len(i), heads, D)
        lse[row] = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(S, len(i), heads)
        del score, p
    return dict(out=out[:rows].to(q.dtype), lse=lse[:rows])


def _sequence_and_position(s):
    row = torch.arange(s["q"].shape[0], device=s["table"].device)
    seq = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    return seq, s["starts"].long()[seq] + row - s["offsets"].long()[seq]


def _plain_rotate(s):
    seq, pos = _sequence_and_position(s)
    R = 2 * len(s["frequencies"])
    angle = pos[:, None].double() * s["frequencies"]  # far positions need the 64 bits
    c, d = ((f(angle) * s["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    part = (slice(0, R, 2), slice(1, R, 2)) if s["interleaved"] else (slice(0, R // 2), slice(R // 2, R))

    def turned(x):
        x = x.float()
        y = x.clone()
        y[..., part[0]] = x[..., part[0]] * c - x[..., part[1]] * d
        y[..., part[1]] = x[..., part[1]] * c + x[..., part[0]] * d
        return y

    ps = s["k"].shape[2]
    page, place = s["table"][seq, pos // ps].long(), pos % ps

    def write(cache, x, scale):
        if scale is not None:
            x = (x / scale[:, None]).clamp(-FP8_MAX, FP8_MAX)
        byte = torch.uint8 if cache.dtype == KINDS["fp8"] else cache.dtype
        cache.view(byte)[page, :, place] = x.to(cache.dtype).view(byte)
        return cache

    return dict(out=turned(s["q"]).to(s["q"].dtype), k=write(s["k"], turned(s["new_k"]), s["k_scale"]),
                v=write(s["v"], s["new_v"].float(), s["v_scale"]))


def _plain_score(s):
    x, token, K = s["logits"].float(), s["tokens"].long()[:, None], s["top"]
    d = x - x.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    log = torch.log(total)
    entropy = log[:, 0] - (e * d).masked_fill_(e == 0, 0.0).sum(1) / total[:, 0]
    mine = x.gather(1, token)
    at = torch.arange(x.shape[1], device=x.device)
    rank = ((x > mine) | ((x == mine) & (at < token))).sum(1)
    out = dict(logprobs=(d.gather(1, token) - log)[:, 0], entropy=entropy, ranks=rank.int())
    if K:
        best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :K]
        out.update(top_logprobs=d.gather(1, best) - log, top_tokens=best.int())
    return out


# --------------------------------------------------------------------- run

def run(state):
    s = state
    if not own:
        return {"attend": _plain_attend, "rotate": _plain_rotate, "score": _plain_score}[s["op"]](s)
    import paper_2609_12299_amd as fw
    if s["op"] == "attend":
        return fw.attend_chunks(s["q"], s["k"], s["v"], s["table"], s["lens"], s["offsets"], scale=s["scale"],
                                window=s["window"], sinks=s["sinks"], k_scale=s["k_scale"], v_scale=s["v_scale"], lse=True)
    if s["op"] == "rotate":
        out = fw.rotate_tokens(s["q"], s["new_k"], s["new_v"], s["k"], s["v"], s["table"], s["starts"], s["frequencies"],
                               offsets=None if s["single"] else s["offsets"], interleaved=s["interleaved"],
                               amplitude=s["amplitude"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return dict(out, k=s["k"], v=s["v"])
    return fw.score_tokens(s["logits"], s["tokens"], top=s["top"])


# -------------------------------------------------------------------- work

def _width(kind):
    return {"fp8": 1, "fp32": 4}.get(kind, 2)


def work(case):
    """Inputs read once and outputs written once; of a cache what the call has to look at."""
    if case["op"] == "score":
        R = case["rows"]
        return {"bytes": R * (case["vocab"] * _width(case["kind"]) + 16 + 8 * case["top"]), "flops": 0}
    new, past = _sizes(case, 0)
    T, D = sum(new), case["dim"]
    if case["op"] == "rotate":
        kv = 2 * T * case["kv_heads"] * D
        b = T * (4 * case["heads"] * D + 4) + kv * (2 + _width(case["kind"])) + 12 * case["seqs"] + 4 * case["rotated"]
        return {"bytes": b, "flops": 0}
    w, sinks = case["window"], case["sinks"]
    heads, read, pairs = case["kv_heads"] * case["group"], 0, 0
    for n, p in zip(new, past):
        if not n:
            continue
        lo = max(0, p + 1 - w) if w else 0  # of the first query
        read += p + n - lo + min(sinks, lo)
        full = n * p + n * (n + 1) // 2
        if w:  # the m-th position sees min(m + 1, window) tokens, and those of the first that lie before them
            far = max(0, p + n - max(p, w))  # queries whose window leaves tokens out
            if far:
                first = max(p, w)  # the first of them
                left = far * (first + 1 - w) + far * (far - 1) // 2
                back = sum(min(sinks, m + 1 - w) for m in range(first, first + far))
                full += back - left
        pairs += full
    b = 2 * read * case["kv_heads"] * D * _width(case["kind"]) + 4 * (read // case["page"] + 2 * case["seqs"])
    return {"bytes": b + T * heads * (4 * D + 4), "flops": 4 * pairs * heads * D}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "score":
        x = s["logits"].double()
        lse = torch.logsumexp(x, 1, keepdim=True)
        p = torch.softmax(x, 1)
        out = dict(logprobs=(x.gather(1, s["tokens"].long()[:, None]) - lse)[:, 0], ranks=None,
                   entropy=-torch.special.xlogy(p, p).sum(1))
        if case["top"]:
            out.update(top_logprobs=torch.topk(x, case["top"], 1).values - lse, top_tokens=None)
        return out
    if case["op"] == "rotate":
        seq, pos = _sequence_and_position(s)
        R, ps = case["rotated"], case["page"]
        turn = torch.polar(torch.full((), s["amplitude"], dtype=torch.float64, device="cuda").expand(len(pos), R // 2),
                           pos[:, None].double() * s["frequencies"])[:, None]

        def turned(x):
            x = x.double()
            z = x[..., :R].reshape(*x.shape[:2], R // 2, 2) if case["interleaved"] else x[..., :R].reshape(*x.shape[:2], 2, R // 2).transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            z = z if case["interleaved"] else z.transpose(2, 3)
            return torch.cat([z.reshape(*x.shape[:2], R), x[..., R:]], 2)

        out = dict(out=turned(s["q"]))
        page = s["table"][seq, pos // ps].long()
        for name, x in (("k", turned(s["new_k"])), ("v", s["new_v"].double())):
            c = s[name].double()
            if case["kind"] == "fp8":
                x = (x / s[name + "_scale"].double()[:, None]).clamp(-FP8_MAX, FP8_MAX)
            c[page, :, pos % ps] = x
            out[name] = c
        return out
    rows, heads, D = s["q"].shape
    H, G, ps = case["kv_heads"], case["group"], case["page"]
    out = torch.zeros((rows, heads, D), dtype=torch.float64, device="cuda")
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device="cuda")
    ends = s["offsets"].tolist()
    for i, length in enumerate(s["lens"].tolist()):
        a, b = ends[i], ends[i + 1]
        for r0 in range(a, b, 1024):
            r1 = min(r0 + 1024, b)
            pos = torch.arange(r0, r1, device="cuda") - b + length
            j = torch.arange(int(pos[-1]) + 1, device="cuda")
            if case["window"]:  # what none of these queries sees may not even have a page
                j = j[(j > int(pos[0]) - case["window"]) | (j < case["sinks"])]
            hidden = j > pos[:, None]
            if case["window"]:
                hidden |= (j <= pos[:, None] - case["window"]) & (j >= case["sinks"])
            page = s["table"][i, j // ps].long()
            for h in range(H):
                k, v = (c[page, h, j % ps].double() for c in (s["k"], s["v"]))
                if s["k_scale"] is not None:
                    k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
                for g in range(h * G, (h + 1) * G):
                    score = (s["q"][r0:r1, g].double() @ k.T * s["scale"]).masked_fill_(hidden, -math.inf)
                    lse[r0:r1, g] = torch.logsumexp(score, 1)
                    out[r0:r1, g] = torch.softmax(score, 1) @ v
    return dict(out=out, lse=lse)
