"""What the decode-step operators are measured on: attention of one new token over a paged cache,
the writing of new tokens into its pages, the move of its page tables from one step to the next
(fork, copy on write, growth, release), its compaction, and beam search's selection.

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

def _attend(name, kind, seqs, shortest, longest, kv_heads, group, dim, page, window=0, sinks=0):
    c = dict(op="attend", kind=kind, seqs=seqs, shortest=shortest, longest=longest,
             kv_heads=kv_heads, group=group, dim=dim, page=page, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _append(name, kind, source, seqs, shortest, longest, kv_heads, dim, page):
    c = dict(op="append", kind=kind, source=source, seqs=seqs, shortest=shortest, longest=longest,
             kv_heads=kv_heads, dim=dim, page=page)
    return dict(c, name=name) if name else c


def _step(name, groups, beams, columns, pages, layers, kv_heads, dim, page, window=0, sinks=0):
    c = dict(op="step", groups=groups, beams=beams, columns=columns, pages=pages, layers=layers,
             kv_heads=kv_heads, dim=dim, page=page, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _compact(name, seqs, columns, pages, layers, kv_heads, dim, page):
    c = dict(op="compact", seqs=seqs, columns=columns, pages=pages, layers=layers,
             kv_heads=kv_heads, dim=dim, page=page)
    return dict(c, name=name) if name else c


def _select(name, kind, groups, beams, vocab, k):
    c = dict(op="select", kind=kind, groups=groups, beams=beams, vocab=vocab, k=k)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's decode step early in an answer: a single short sequence, where launches count
        _attend("attend_one_short", "bf16", 1, 177, 177, 4, 8, 64, 16),
        # a serving batch of very different lengths, with a window over the last 4096 tokens and
        # four first tokens that stay visible; a head size that is no power of two
        _attend("attend_window_ragged", "fp16", 96, 1, 30011, 8, 4, 96, 32, 4096, 4),
        # a serving batch over a cache held in 8 bits, an empty slot among the sequences
        _attend("attend_fp8_batch", "fp8", 48, 0, 32768, 8, 8, 128, 64),
        # few long documents: the length is what there is to split
        _attend("attend_long", "bf16", 4, 262143, 262143, 8, 8, 128, 64),
        # the new token of every sequence of a decode step
        _append("append_step", "bf16", "bf16", 64, 1, 1, 8, 128, 16),
        # prompts of all lengths written after their prefill, into a cache of 8 bits
        _append("append_prompts_fp8", "fp8", "bf16", 40, 1, 16384, 8, 128, 64),
        # beam search for a few requests: four beams each, reordered every step
        _step("step_beams_few", 4, 4, 64, 1024, 22, 4, 64, 16),
        # a large serving batch in beam search with a sliding window; requests end and start
        _step("step_beams_batch", 64, 8, 256, 16384, 8, 4, 64, 16, 2048, 64),
        # a small pool tidied between requests
        _compact("compact_small", 8, 64, 640, 2, 4, 64, 16),
        # a pool after hours of serving: half of its pages free, all over it
        _compact("compact_pool", 192, 256, 16384, 8, 4, 64, 16),
        # beam search of one request
        _select("select_one", "bf16", 1, 4, 32000, 4),
        # a batch of beam searches over a large vocabulary of odd size
        _select("select_batch", "bf16", 96, 8, 128003, 8),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "step", "compact", "select", "select"])
    if op == "attend":
        kind = rng.choice(["bf16", "fp16", "fp8"])
        seqs, kv_heads = _between(rng, 1, 128), rng.choice([1, 2, 4, 8, 16])
        dim, page = rng.choice([64, 80, 96, 128, 256]), rng.choice([8, 16, 32, 64, 128])
        most = max(64, min(262143, (1 << 29) // (seqs * kv_heads * dim)))
        longest = _between(rng, 40, most)
        shortest = rng.choice([0, 1, longest, longest])
        window = rng.choice([0, 0, _between(rng, 16, 8192)])
        group = rng.choice([1, 2, 4, 7, 8, 16, 24])
        return _attend("", kind, seqs, shortest, longest, kv_heads, group, dim, page, window,
                       rng.choice([0, 1, 4, 64]) if window else 0)
    if op == "append":
        kind = rng.choice(["bf16", "fp16", "fp8"])
        source = rng.choice(["bf16", "fp16"]) if kind == "fp8" else kind
        longest = rng.choice([1, _between(rng, 2, 8192)])
        return _append("", kind, source, _between(rng, 1, 96 if longest < 4096 else 40),
                       rng.choice([0, 1, longest]), longest, rng.choice([1, 2, 4, 8]),
                       rng.choice([64, 80, 96, 128, 256]) // (2 if longest >= 4096 else 1) // 16 * 16,
                       rng.choice([8, 16, 32, 64, 128]))
    if op == "step":
        beams, columns = rng.choice([1, 2, 4, 5, 8]), _between(rng, 16, 256)
        groups = _between(rng, 1, max(1, min(64, 512 // beams)))
        pages = groups * columns + groups * beams * 24 + 32
        window = rng.choice([0, _between(rng, 64, 2048)])
        return _step("", groups, beams, columns, pages, rng.choice([1, 2, 5, 8]), 4,
                     rng.choice([64, 96, 128]) if pages < 8192 else 64, rng.choice([8, 16]),
                     window, 64 if window else 0)
    if op == "compact":
        seqs, columns = _between(rng, 1, 192), _between(rng, 16, 256)
        pages = min(16384, max(64, int(seqs * columns * rng.uniform(0.3, 0.6))))
        return _compact("", seqs, columns, pages, rng.choice([1, 2, 5, 8]), 4, rng.choice([64, 96]),
                        rng.choice([8, 16]))
    kind = rng.choice(["bf16", "fp16", "fp32"])
    beams, vocab = rng.choice([1, 2, 4, 5, 8, 16]), _between(rng, 1000, 200003)
    groups = _between(rng, 1, max(1, min(96, (24 << 20) // (beams * vocab))))
    return _select("", kind, groups, beams, vocab, rng.choice([1, beams, min(2 * beams, 32)]))


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """Lengths from the shortest to the longest, evenly over their logarithm; the same for every
    seed but for their order."""
    n, lo, hi = case["seqs"], case["shortest"], case["longest"]
    if n == 1 or lo == hi:
        return [hi] * n
    a, b = math.log(lo + 1), math.log(hi + 1)
    return [int(round(math.exp(a + (b - a) * i / (n - 1)))) - 1 for i in range(n)]


def _shuffled_lengths(case, seed):
    out = _lengths(case)
    random.Random(seed).shuffle(out)
    return out


def _random(shape, gen, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16 if dtype == KINDS["fp8"] else dtype).to(dtype)


def _pool(case):
    """Shape of one of the two caches: layers, pages, heads, tokens of a page, head size."""
    return case["layers"], case["pages"], case["kv_heads"], case["page"], case["dim"]


def _tables(lens, page, columns, gen, held=None, pages=None):
    """Page tables of sequences that share nothing: pages of a pool in random order; entries of
    pages that are not held, and those beyond a sequence, are -1."""
    n = torch.tensor([-(-x // page) for x in lens], device="cuda")
    col = torch.arange(columns, device="cuda")
    used = col < n[:, None]
    if held is not None:
        used &= held(col, torch.tensor(lens, device="cuda")[:, None])
    count = int(used.sum())
    pages = pages or count + count // 16 + 1
    table = torch.full((len(lens), columns), -1, dtype=torch.int32, device="cuda")
    table[used] = torch.randperm(pages, generator=gen, device="cuda")[:count].int()
    return table, pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return dict({"attend": _prepare_attend, "append": _prepare_append, "step": _prepare_step,
                 "compact": _prepare_compact, "select": _prepare_select}[case["op"]](case, seed, gen),
                op=case["op"])


def _prepare_attend(case, seed, gen):
    S, H, D, ps = case["seqs"], case["kv_heads"], case["dim"], case["page"]
    window, sinks = case["window"], case["sinks"]
    lens = _shuffled_lengths(case, seed)
    columns = max(1, -(-case["longest"] // ps))
    held = None
    if window:  # pages that no query sees any more have been given back
        held = lambda col, n: ((col + 1) * ps > n - window) | (col * ps < sinks)  # noqa: E731
    table, pages = _tables(lens, ps, columns, gen, held)
    kind = KINDS[case["kind"]]
    k, v = (_random((pages, H, ps, D), gen, kind) for _ in range(2))
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # what lies behind a sequence's end in its last page was never written: anything, NaN too
    some = torch.nonzero(lens % ps)[:, 0]
    last = table[some, (lens[some] // ps).long()].long()
    junk = torch.arange(ps, device="cuda") >= (lens[some] % ps)[:, None]
    for c in (k, v):
        tail = c[last].float()
        c[last] = tail.masked_fill_(junk[:, None, :, None], float("nan")).to(kind)
    q = _random((S, H * case["group"], D), gen, torch.float16 if case["kind"] == "fp16" else torch.bfloat16)
    state = dict(q=q, k=k, v=v, table=table, lens=lens, window=window, sinks=sinks,
                 scale=D ** -0.5, k_scale=None, v_scale=None)
    if case["kind"] == "fp8":
        state.update({n: torch.rand(H, generator=gen, device="cuda") + 0.5 for n in ("k_scale", "v_scale")})
    return state


def _prepare_append(case, seed, gen):
    S, H, D, ps = case["seqs"], case["kv_heads"], case["dim"], case["page"]
    rows = _shuffled_lengths(case, seed)
    rnd = random.Random(seed + 1)
    starts = [rnd.randrange(512) for _ in rows]
    columns = -(-(max(case["longest"], 1) + 512) // ps)
    most = sum(-(-(x + 512) // ps) for x in rows)  # the same for every seed
    table, pages = _tables([a + b for a, b in zip(starts, rows)], ps, columns, gen, pages=most)
    T = sum(rows)
    source = KINDS[case["source"]]
    # one buffer holds a token's keys and values, as a fused projection leaves them
    fused = _random((max(T, 1), 2, H, D), gen, source)[:T]
    kind = KINDS[case["kind"]]
    k, v = (torch.zeros((pages, H, ps, D), dtype=kind, device="cuda") for _ in range(2))
    ends = torch.tensor([0] + rows, device="cuda").cumsum(0).int()
    state = dict(new_k=fused[:, 0], new_v=fused[:, 1], k=k, v=v, table=table, offsets=ends,
                 starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                 single=case["shortest"] == case["longest"] == 1, k_scale=None, v_scale=None)
    if case["kind"] == "fp8":
        state.update({n: torch.rand(H, generator=gen, device="cuda") * 0.05 + 0.01 for n in ("k_scale", "v_scale")})
    return state


def _prepare_step(case, seed, gen):
    """Groups of beams that share the pages of their prompt; a beam's own tokens lie in pages of
    its own.  One group in eight ends and makes room for a new request."""
    G, W, P, ps, pages = case["groups"], case["beams"], case["columns"], case["page"], case["pages"]
    S = G * W
    ints = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=gen, device="cuda")  # noqa: E731
    lens = ints(ps, (P - 1) * ps, G).repeat_interleave(W)
    shared = torch.clamp(lens // ps - ints(0, 17, G).repeat_interleave(W), min=0)
    n = -(-lens // ps)
    col = torch.arange(P, device="cuda")
    row = torch.arange(S, device="cuda")
    owner = torch.where(col < shared[:, None], (row // W * W)[:, None], row[:, None])
    used = (col < n[:, None]) & (owner == row[:, None])
    # fewer pages than the longest tables could take: the last groups wait outside
    order = torch.cumsum(used.reshape(-1).int(), 0).reshape(S, P) - 1
    waiting = (order.reshape(G, -1).amax(1) >= pages * 7 // 8).repeat_interleave(W)
    perm = torch.randperm(pages, generator=gen, device="cuda").int()
    ids = torch.where(used, perm[order.clamp(0, pages - 1)], -1)
    table = ids[owner, col.expand(S, P)]
    table = torch.where((col < n[:, None]) & ~waiting[:, None], table, -1)
    lens = torch.where(waiting, 0, lens)
    parents = (row // W * W).int() + ints(0, W, S).int()
    ended = (ints(0, 8, G) == 0).repeat_interleave(W) | waiting
    parents = torch.where(ended, -1, parents)
    prompt = ints(1, max(2, min(256, P * ps // 2)), G).repeat_interleave(W)
    grow = torch.where(ended, torch.where(row % W == 0, prompt, 0), 1)
    held = (ints(0, 64, pages) == 0).int()  # a prefix cache holds pages too
    caches = [_random(_pool(case), gen, torch.bfloat16) for _ in range(2)]
    return dict(table=table.int().contiguous(), lens=lens.int(), parents=parents, grow=grow.int(),
                held=held, caches=caches, page=ps, window=case["window"], sinks=case["sinks"])


def _prepare_compact(case, seed, gen):
    S, P, pages = case["seqs"], case["columns"], case["pages"]
    live = pages // 2
    perm = torch.randperm(pages, generator=gen, device="cuda").int()[:live]
    n = torch.randint(0, P + 1, (S,), generator=gen, device="cuda")
    used = torch.arange(P, device="cuda") < n[:, None]
    pick = torch.randint(0, live, (S, P), generator=gen, device="cuda")
    table = torch.where(used, perm[pick], -1).contiguous()
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    refs.index_add_(0, table[used].long(), torch.ones_like(table[used]))
    refs[perm[: live // 8].long()] += 1  # held elsewhere too
    caches = [_random(_pool(case), gen, torch.bfloat16) for _ in range(2)]
    return dict(table=table, refs=refs, caches=caches)


def _prepare_select(case, seed, gen):
    """Logits as a product in 16 bits leaves them (a coarse grid, so equal values are common).  The
    beams' scores are such that candidates of two beams lie at least 1/(32 beams) apart: which comes
    first does not hang on the last bit of a logarithm."""
    N, W, V = case["groups"], case["beams"], case["vocab"]
    logits = torch.randn((N, W, V), generator=gen, device="cuda") * 2.5
    logits = (logits * 32).round().clamp(-480, 480) / 32
    lse = torch.logsumexp(logits.double(), 2)
    behind = torch.randint(0, 96, (N, W), generator=gen, device="cuda") / 32
    beam = torch.arange(W, device="cuda")
    scores = (lse - 14.0 - behind + beam / (32.0 * W)).float()
    finished = torch.rand((N, W), generator=gen, device="cuda") < 0.1
    # a beam that has ended stands for itself, with a score between two steps of the grid
    ended = (-2.0 - behind + (beam + 0.5) / (32.0 * W)).float()
    return dict(logits=logits.to(KINDS[case["kind"]]), scores=torch.where(finished, ended, scores),
                finished=finished, k=case["k"], eos=2)


# ------------------------------------------------------------- plain forms

def _plain_attend(s):
    q, k, v, table, lens = s["q"], s["k"], s["v"], s["table"], s["lens"].long()
    S, Hq, D = q.shape
    pages, H, ps, _ = k.shape
    at = torch.arange(table.shape[1] * ps, device=q.device)
    seen = (at < lens[:, None]) & (table >= 0).repeat_interleave(ps, 1)
    if s["window"]:
        seen &= (at >= lens[:, None] - s["window"]) | (at < s["sinks"])
    page = table.clamp(min=0).long()

    def rows(c, scale):  # [S, H, tokens, D] in 32 bits, nothing where nothing is seen
        x = c[page].transpose(1, 2).reshape(S, H, -1, D).float()
        x = x if scale is None else x * scale[:, None, None]
        return x.masked_fill_(~seen[:, None, :, None], 0.0)

    qt = q.float().reshape(S, H, Hq // H, D).transpose(2, 3).contiguous()
    score = (rows(k, s["k_scale"]) @ qt).transpose(2, 3) * s["scale"]  # [S, H, G, tokens]
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(3, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(3, keepdim=True)
    out = (p.contiguous() @ rows(v, s["v_scale"])) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total))[..., 0]
    return dict(out=out.reshape(S, Hq, D).to(q.dtype), lse=lse.reshape(S, Hq))


def _places(s):
    """Sequence, page and place in its page of every new token, and whether the page is held."""
    ps = s["k"].shape[2]
    row = torch.arange(s["new_k"].shape[0], device=s["table"].device)
    seq = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    pos = s["starts"].long()[seq] + row - s["offsets"].long()[seq]
    return s["table"][seq, pos // ps].long(), pos % ps


def _plain_append(s):
    page, place = _places(s)

    def write(c, x, scale):
        x = x.float()
        if scale is not None:
            x = (x / scale[:, None]).clamp(-FP8_MAX, FP8_MAX)
        byte = torch.uint8 if c.dtype == KINDS["fp8"] else c.dtype
        c.view(byte)[page, :, place] = x.to(c.dtype).view(byte)
        return c

    return dict(k=write(s["k"], s["new_k"], s["k_scale"]), v=write(s["v"], s["new_v"], s["v_scale"]))


def _plain_step(s):
    table, ps, held = s["table"].long(), s["page"], s["held"].long()
    dev, (S_in, P), N = table.device, table.shape, len(held)
    parent = s["parents"].long()
    S = len(parent)
    bad = (parent < -1) | (parent >= S_in)
    kept = (parent >= 0) & ~bad
    src = torch.where(kept, parent, 0)
    old = torch.where(kept, s["lens"].long()[src].clamp(0, P * ps), 0)
    want = old + s["grow"].long().clamp(min=0)
    new = want.clamp(max=P * ps)
    n_old, n_new = -(-old // ps), -(-new // ps)
    col, row = torch.arange(P, device=dev), torch.arange(S, device=dev)
    entry = torch.where(kept[:, None] & (col < n_old[:, None]), table[src], -1)
    entry = torch.where((entry >= 0) & (entry < N), entry, -1)
    if s["window"]:  # no later query sees these
        first = old + (new > old).long() - s["window"]
        gone = ((col + 1) * ps <= first[:, None]) & (col * ps >= s["sinks"])
        entry = torch.where(gone, -1, entry)
    flat = torch.where(entry >= 0, entry, N).reshape(-1)
    refs = torch.bincount(flat, minlength=N + 1)[:N] + held
    # a page that ends inside: of those who have it last, the longest (then the first) may write on
    last = entry.gather(1, (old // ps).clamp(max=P - 1)[:, None])[:, 0]
    ends = (old % ps > 0) & (last >= 0)
    at = torch.where(ends, last, N)
    key = torch.where(ends, old * S + (S - 1 - row), -1)
    best = torch.full((N + 1,), -1, device=dev).scatter_reduce_(0, at, key, "amax")
    count = torch.bincount(at, minlength=N + 1)
    alone = (held[at.clamp(max=N - 1)] == 0) & (count[at] == refs[at.clamp(max=N - 1)]) & (best[at] == key)
    copy = ends & (new > old) & ~alone
    need = copy.long() + n_new - n_old
    base = torch.cumsum(need, 0) - need
    free = torch.sort((refs > 0).int(), stable=True).indices
    n_free = (refs == 0).sum()

    def fresh(rank):
        return torch.where(rank < n_free, free[rank.clamp(max=N - 1)], -1)

    grown = fresh(base[:, None] + copy[:, None] + col - n_old[:, None])
    out = torch.where((col >= n_old[:, None]) & (col < n_new[:, None]), grown, entry)
    dst = torch.where(copy, fresh(base), -1)
    out = torch.where(copy[:, None] & (col == (old // ps)[:, None]), dst[:, None], out)
    refs = refs - torch.bincount(torch.where(copy, last, N), minlength=N + 1)[:N]
    total = need.sum()
    at = torch.arange(N, device=dev)
    refs = refs.scatter_add(0, free, ((at < total) & (at < n_free)).long())
    done = copy & (dst >= 0)
    for_copy = torch.nonzero(done)[:, 0]
    k, v = s["caches"]
    k[:, dst[for_copy]] = k[:, last[for_copy]]
    v[:, dst[for_copy]] = v[:, last[for_copy]]
    zero = torch.zeros((), dtype=torch.long, device=dev)
    counters = torch.stack([total, (total - n_free).clamp(min=0), done.sum(), (refs > 0).sum(),
                            bad.sum(), (want > new).sum(), zero, zero])
    return dict(table=out.int(), lens=new.int(), refs=refs.int(), counters=counters.int(), k=k, v=v)


def _plain_compact(s):
    table, refs = s["table"].long(), s["refs"]
    N, dev = len(refs), table.device
    live = refs > 0
    n = live.sum()
    at = torch.arange(N, device=dev)
    hole, mover = ~live & (at < n), live & (at >= n)
    rank = torch.where(at < n, torch.cumsum(hole.int(), 0), torch.cumsum(mover.int(), 0)) - 1
    holes = torch.sort((~hole).int(), stable=True).indices
    to = torch.where(mover, holes[rank.clamp(min=0)], at)
    to = torch.where(live, to, -1)
    known = (table >= 0) & (table < N)
    out = torch.where(known, to[table.clamp(0, N - 1)], -1)
    counts = torch.zeros(N + 1, dtype=torch.int32, device=dev).scatter_(0, torch.where(live, to, N), refs)
    counts[N] = 0
    src = torch.nonzero(mover)[:, 0]
    k, v = s["caches"]
    k[:, to[src]] = k[:, src]
    v[:, to[src]] = v[:, src]
    zero = torch.zeros((), dtype=torch.long, device=dev)
    counters = torch.stack([n, mover.sum(), zero, zero, zero, zero, zero, zero])
    return dict(table=out.int(), refs=counts[:N], map=to.int(), counters=counters.int(), k=k, v=v)


def _plain_select(s):
    x, score, finished, K = s["logits"].float(), s["scores"], s["finished"], s["k"]
    N, W, V = x.shape
    top = x.amax(2, keepdim=True)
    lse = (top + torch.log(torch.exp(x - top).sum(2, keepdim=True)))
    L = min(K, V)
    best = torch.sort(x, dim=2, descending=True, stable=True)
    token, logit = best.indices[..., :L], best.values[..., :L]
    cand = score[..., None] + (logit - lse)
    # a beam that has ended stands for itself alone
    stay = torch.full_like(cand, -math.inf)
    stay[..., 0] = score
    cand = torch.where(finished[..., None], stay, cand)
    token = torch.where(finished[..., None], s["eos"], token)
    cand = torch.where(torch.isnan(cand), -math.inf, cand).reshape(N, -1)
    got = torch.sort(cand, dim=1, descending=True, stable=True)
    value, at = got.values[:, :K], got.indices[:, :K]
    fine = value > -math.inf
    row = torch.arange(N, device=x.device)[:, None] * W + at // L
    token = torch.where(fine, token.reshape(N, -1).gather(1, at), -1)
    row = torch.where(fine, row, -1)
    ended = fine & (finished.reshape(-1)[row.clamp(min=0)] | (token == s["eos"]))
    return dict(scores=value, parents=row.int(), tokens=token.int(), finished=ended)


# --------------------------------------------------------------------- run

def run(state):
    s = state
    if not own:
        return {"attend": _plain_attend, "append": _plain_append, "step": _plain_step,
                "compact": _plain_compact, "select": _plain_select}[s["op"]](s)
    import paper_2609_12299_amd as fw
    if s["op"] == "attend":
        return fw.attend_pages(s["q"], s["k"], s["v"], s["table"], s["lens"], scale=s["scale"],
                               window=s["window"], sinks=s["sinks"], k_scale=s["k_scale"],
                               v_scale=s["v_scale"], lse=True)
    if s["op"] == "append":
        fw.append_tokens(s["new_k"], s["new_v"], s["k"], s["v"], s["table"], s["starts"],
                         offsets=None if s["single"] else s["offsets"], k_scale=s["k_scale"],
                         v_scale=s["v_scale"])
        return dict(k=s["k"], v=s["v"])
    if s["op"] == "step":
        out = fw.step_pages(s["table"], s["lens"], s["parents"], s["grow"], s["page"], held=s["held"],
                            caches=s["caches"], window=s["window"], sinks=s["sinks"])
    elif s["op"] == "compact":
        out = fw.compact_pages(s["table"], s["refs"], caches=s["caches"])
    else:
        return fw.select_beams(s["logits"], s["scores"], s["k"], finished=s["finished"], eos=s["eos"])
    out = {k: v for k, v in out.items() if not k.startswith("_")}
    return dict(out, k=s["caches"][0], v=s["caches"][1])


# -------------------------------------------------------------------- work

def _width(kind):
    return {"fp8": 1, "fp32": 4}.get(kind, 2)


def work(case):
    """Inputs read once and outputs written once; of a page table what the call has to look at."""
    op = case["op"]
    if op == "attend":
        lens, w = _lengths(case), case["window"]
        seen = sum(n if not w or n <= w else w + min(case["sinks"], n - w) for n in lens)
        heads = case["kv_heads"] * case["group"]
        b = 2 * seen * case["kv_heads"] * case["dim"] * _width(case["kind"])
        b += 4 * (seen // case["page"] + case["seqs"]) + case["seqs"] * heads * (4 * case["dim"] + 4)
        return {"bytes": b, "flops": 4 * seen * heads * case["dim"]}
    if op == "append":
        values = 2 * sum(_lengths(case)) * case["kv_heads"] * case["dim"]
        return {"bytes": values * (_width(case["source"]) + _width(case["kind"])) + 8 * case["seqs"],
                "flops": 0}
    layers = case.get("layers", 0)
    page = 4 * layers * case.get("kv_heads", 0) * case.get("page", 0) * case.get("dim", 0)  # keys and values
    if op == "step":
        # of W beams that take a random one of W parents each, (1 - 1/W)^W of the parents are left
        # out: the others' last pages are each written on by one beam and copied by the rest
        S, W = case["groups"] * case["beams"], case["beams"]
        copies = S * (1 - 1 / 8) * (1 - 1 / case["page"]) * (1 - 1 / W) ** W if W > 1 else 0
        tables = 4 * S * (2 * case["columns"] + 4) + 8 * case["pages"]
        return {"bytes": tables + int(copies) * 2 * page, "flops": 0}
    if op == "compact":
        N = case["pages"]
        return {"bytes": 8 * case["seqs"] * case["columns"] + 12 * N + N // 4 * 2 * page, "flops": 0}
    rows = case["groups"] * case["beams"]
    return {"bytes": rows * (case["vocab"] * _width(case["kind"]) + 5) + case["groups"] * case["k"] * 13,
            "flops": 0}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    if case["op"] in ("step", "compact"):
        return None  # whole numbers, and pages copied bit for bit
    s = prepare(case, seed)
    if case["op"] == "append":
        if case["kind"] != "fp8":
            return None  # copied bit for bit
        page, place = _places(s)
        out = {}
        for name in ("k", "v"):
            c = s[name].double()
            x = s["new_" + name].double() / s[name + "_scale"].double()[:, None]
            c[page, :, place] = x.clamp(-FP8_MAX, FP8_MAX)
            out[name] = c
        return out
    if case["op"] == "select":
        plain = _plain_select(s)  # which candidates: whole numbers; their scores from here on in 64 bits
        row, token = plain["parents"].long(), plain["tokens"].long()
        lse = torch.logsumexp(s["logits"].double(), 2).reshape(-1)
        at = row.clamp(min=0)
        base = s["scores"].double().reshape(-1)[at]
        own_score = base + s["logits"].reshape(-1, case["vocab"])[at, token.clamp(min=0)].double() - lse[at]
        score = torch.where(s["finished"].reshape(-1)[at], base, own_score)
        return dict(scores=torch.where(row >= 0, score, -math.inf), parents=None, tokens=None, finished=None)
    S, Hq, D = s["q"].shape
    H, ps = case["kv_heads"], case["page"]
    out = torch.zeros((S, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((S, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["lens"].tolist()):
        j = torch.arange(n, device="cuda")
        if case["window"]:
            j = j[(j >= n - case["window"]) | (j < case["sinks"])]
        if not len(j):
            continue
        page = s["table"][i, j // ps].long()
        for h in range(H):
            k, v = (c[page, h, j % ps].double() for c in (s["k"], s["v"]))
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            g = slice(h * case["group"], (h + 1) * case["group"])
            score = s["q"][i, g].double() @ k.T * s["scale"]
            lse[i, g] = torch.logsumexp(score, 1)
            out[i, g] = torch.exp(score - lse[i, g][:, None]) @ v
    return dict(out=out, lse=lse)
