"""Beam search over a paged cache, and where its time goes.

A small transformer with random weights answers a few prompts with beam search.
Every step is made of this library's operators: page tables move on with the
beams that were selected (step_pages), the new token's keys and values go into
their pages (append_tokens), attention reads them (attend_pages), and the next
beams are selected (select_beams).  With --chunk the prompts are taken so many tokens
at a time (attend_chunks) and scored first (score_tokens); with --rotary queries and keys
have rotary positions (rotate_tokens).  The operators write marker records of their
own regions; region attribution of those records says how long each took, on which
waves.

    python examples/decode_loop.py [--steps 32] [--groups 8] [--beams 4] [--marked 8] [--chunk 64] [--rotary]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2609_12299_amd import (ALL_REGION_NAMES, NUM_ALL_REGIONS, MarkerBuffer, RegionAttribution,  # noqa: E402
                                  append_tokens, attend_chunks, attend_pages, compact_pages, rotary_frequencies,
                                  rotate_tokens, score_tokens, select_beams, step_pages)


class Model:
    """Random weights: `layers` of attention with grouped heads and a residual, tied embeddings; with
    `rotary` the positions are rotary, else there are none."""

    def __init__(self, layers=4, vocab=4099, heads=8, kv_heads=2, head_dim=64, seed=0, device="cuda", rotary=False):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.layers, self.vocab, self.heads, self.kv_heads, self.head_dim = layers, vocab, heads, kv_heads, head_dim
        self.frequencies = rotary_frequencies(head_dim, device=device) if rotary else None
        width = heads * head_dim

        def weight(*shape):
            w = torch.randn(shape, generator=gen, device=device) * shape[-2] ** -0.5
            return w.to(torch.bfloat16)
        self.embed = torch.randn((vocab, width), generator=gen, device=device).to(torch.bfloat16)
        self.qkv = [weight(width, (heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.out = [weight(width, width) for _ in range(layers)]
        self.logits = weight(width, vocab)


class Decoder:
    """Sequences of a batch in beam search: page tables, caches, scores."""

    def __init__(self, model: Model, groups: int, beams: int, page_size=16, columns=16, pages=None, device="cuda"):
        self.m, self.G, self.W, self.ps = model, groups, beams, page_size
        S = groups * beams
        pages = pages or S * columns + S
        shape = (model.layers, pages, model.kv_heads, page_size, model.head_dim)
        self.caches = tuple(torch.zeros(shape, dtype=torch.bfloat16, device=device) for _ in range(2))
        self.table = torch.full((S, columns), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(S, dtype=torch.int32, device=device)
        self.parents = torch.arange(S, dtype=torch.int32, device=device)
        self.one = torch.ones(S, dtype=torch.int32, device=device)
        # one beam of each group is alive at first
        self.scores = torch.full((groups, beams), float("-inf"), device=device)
        self.scores[:, 0] = 0.0
        self.finished = torch.zeros((groups, beams), dtype=torch.bool, device=device)
        self.refs = None

    def forward(self, tokens, markers=None):
        """The logits after one more token of every sequence."""
        m = self.m
        moved = step_pages(self.table, self.lens, self.parents, self.one, self.ps, caches=self.caches, markers=markers)
        starts = moved["lens"] - 1
        self.table, self.lens, self.refs = moved["table"], moved["lens"], moved["refs"]
        x = m.embed[tokens.long()]
        for layer in range(m.layers):
            qkv = (x @ m.qkv[layer]).view(x.shape[0], -1, m.head_dim)
            q, k, v = qkv.split([m.heads, m.kv_heads, m.kv_heads], 1)
            k_cache, v_cache = self.caches[0][layer], self.caches[1][layer]
            q = self.place(q, k, v, k_cache, v_cache, starts, None, markers)
            a = attend_pages(q, k_cache, v_cache, self.table, self.lens, markers=markers)["out"]
            x = x + a.view(x.shape[0], -1) @ m.out[layer]
        return x @ m.logits

    def place(self, q, k, v, k_cache, v_cache, starts, offsets, markers):
        """New keys and values into their pages; the queries, turned where positions are rotary."""
        m = self.m
        if m.frequencies is None:
            append_tokens(k, v, k_cache, v_cache, self.table, starts, offsets, markers=markers)
            return q
        return rotate_tokens(q, k, v, k_cache, v_cache, self.table, starts, m.frequencies, offsets, markers=markers)["out"]

    def take(self, tokens, markers=None):
        """The logits [sequences, n, vocab] of n more tokens of every sequence, in one pass."""
        m, (S, n) = self.m, tokens.shape
        moved = step_pages(self.table, self.lens, self.parents, self.one * n, self.ps, caches=self.caches, markers=markers)
        starts = moved["lens"] - n
        self.table, self.lens, self.refs = moved["table"], moved["lens"], moved["refs"]
        offsets = torch.arange(0, S * n + 1, n, dtype=torch.int32, device=tokens.device)
        x = m.embed[tokens.reshape(-1).long()]
        for layer in range(m.layers):
            qkv = (x @ m.qkv[layer]).view(x.shape[0], -1, m.head_dim)
            q, k, v = qkv.split([m.heads, m.kv_heads, m.kv_heads], 1)
            k_cache, v_cache = self.caches[0][layer], self.caches[1][layer]
            q = self.place(q, k, v, k_cache, v_cache, starts, offsets, markers)
            a = attend_chunks(q, k_cache, v_cache, self.table, self.lens, offsets, markers=markers)["out"]
            x = x + a.view(x.shape[0], -1) @ m.out[layer]
        return (x @ m.logits).view(S, n, -1)

    def stay(self):
        self.parents = torch.arange(len(self.lens), dtype=torch.int32, device=self.lens.device)

    def select(self, logits, eos=-1, markers=None):
        """The next beams, and the token that each goes on with."""
        best = select_beams(logits.view(self.G, self.W, -1), self.scores, self.W, finished=self.finished, eos=eos,
                            markers=markers)
        self.scores, self.finished = best["scores"], best["finished"]
        self.parents = best["parents"].view(-1)
        return best["tokens"].view(-1)

    def compact(self, markers=None):
        """The pages in use to the front of the pool."""
        moved = compact_pages(self.table, self.refs, caches=self.caches, markers=markers)
        self.table, self.refs = moved["table"], moved["refs"]
        return moved["counters"]


def read(model: Model, prompts, chunk: int, top=0, markers=None, page_size=16):
    """What the model makes of prompts [groups, length], taken `chunk` tokens at a time: log probabilities, entropies
    and ranks [groups, length - 1] of their tokens behind the first, and the `top` alternatives to each."""
    G, L = prompts.shape
    d = Decoder(model, G, 1, page_size, -(-L // page_size))
    parts = []
    for i in range(0, L - 1, chunk):
        d.stay()
        n = min(chunk, L - 1 - i)
        logits = d.take(prompts[:, i:i + n], markers)
        chosen = prompts[:, i + 1:i + n + 1].reshape(-1).int()
        got = score_tokens(logits.view(G * n, -1), chosen, top=top, markers=markers)
        parts.append({name: x.view(G, n, *x.shape[1:]) for name, x in got.items()})
    return {name: torch.cat([p[name] for p in parts], 1) for name in parts[0]} if parts else {}


def search(model: Model, prompts, beams: int, steps: int, eos: int = -1, markers=None, marked: int = 0,
           page_size=16, chunk=0):
    """Beam search from prompts [groups, length], the last `marked` steps with markers; returns (tokens
    [groups, beams, length + steps], scores [groups, beams], finished, decoder).  The prompts are taken token by
    token, or `chunk` at a time."""
    G, L = prompts.shape
    columns = -(-(L + steps) // page_size)
    d = Decoder(model, G, beams, page_size, columns)
    rows = prompts.repeat_interleave(beams, 0)
    for i in range(0, L, chunk or 1):
        d.stay()
        logits = d.take(rows[:, i:i + chunk])[:, -1].contiguous() if chunk else d.forward(rows[:, i])
    history = rows.clone()
    for i in range(steps):
        mk = markers if i >= steps - marked else None
        tokens = d.select(logits, eos, mk)
        # a beam without a candidate goes on from itself, with a score of -inf: nothing selects it again
        alive = d.parents >= 0
        d.parents = torch.where(alive, d.parents, torch.arange(len(d.parents), device=d.parents.device).int())
        tokens = torch.where(alive, tokens, 0)
        history = torch.cat([history[d.parents.long()], tokens[:, None].to(history.dtype)], 1)
        if i + 1 < steps:
            logits = d.forward(tokens, mk)
    return history.view(G, beams, -1), d.scores, d.finished, d


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--groups", type=int, default=8)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=100)
    ap.add_argument("--marked", type=int, default=8, help="steps at the end that write markers")
    ap.add_argument("--chunk", type=int, default=0, help="tokens of a prompt taken at a time (0: one, and no scores of them)")
    ap.add_argument("--rotary", action="store_true", help="rotary positions")
    args = ap.parse_args()
    model = Model(rotary=args.rotary)
    gen = torch.Generator(device="cuda").manual_seed(1)
    prompts = torch.randint(3, model.vocab, (args.groups, args.prompt), generator=gen, device="cuda")
    markers = MarkerBuffer(1 << 22)
    if args.chunk:
        seen = read(model, prompts, args.chunk, markers=markers)
        if seen:
            print(f"prompts of {args.prompt} tokens, {args.chunk} at a time: {seen['logprobs'].mean().item():.3f} nats a token, "
                  f"entropy {seen['entropy'].mean().item():.3f}, median rank {int(seen['ranks'].median())}")
    tokens, scores, finished, d = search(model, prompts, args.beams, args.steps, eos=2, markers=markers, marked=args.marked,
                                         chunk=args.chunk)
    live, moved = d.compact(markers).tolist()[:2]
    records = markers.records()
    report = RegionAttribution(NUM_ALL_REGIONS, max_records=len(records), instances=False, instance_excl=False)
    stats = report.run(records)
    torch.cuda.synchronize()
    rows = stats["region_stats"].cpu().numpy()
    counters = stats["counters"].cpu().numpy()
    print(f"{args.groups} prompts, {args.beams} beams, {args.steps} steps ({min(args.marked, args.steps)} marked): best scores "
          + ", ".join(f"{x:.2f}" for x in scores[:, 0].tolist()))
    print(f"{live} pages in use, {moved} moved to the front; {len(records)} marker records, "
          f"{int(counters[10])} mismatched, {int(counters[11])} unclosed, {int(counters[12])} orphans")
    print(f"{'region':16s} {'instances':>10s} {'mean us':>10s} {'least us':>10s} {'most us':>10s}")
    for r, name in enumerate(ALL_REGION_NAMES):
        n = int(rows[r][0])
        if n:
            print(f"{name:16s} {n:10d} {int(rows[r][1]) / n / 100:10.2f} {int(rows[r][3]) / 100:10.2f} {int(rows[r][4]) / 100:10.2f}")


if __name__ == "__main__":
    main()
