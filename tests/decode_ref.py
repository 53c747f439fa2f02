"""The decode-step operators from their definitions, on the CPU: numbers in 64 bits, tables one
sequence after the other in plain Python."""
from __future__ import annotations

import math

import numpy as np
import torch

EPS = 2.0 ** -24  # half a step of 32 bits
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half a step of a result: 8 and 11 significant bits


def attend(q, k, v, table, lens, scale, window=0, sinks=0, k_scale=None, v_scale=None):
    """(out, lse, and how far each may be off in 32 bits).  q [S, heads, D], k and v [pages, H, ps, D]."""
    S, heads, D = q.shape
    N, H, ps, _ = k.shape
    G = heads // H
    P = table.shape[1]
    out, lse = np.zeros((S, heads, D)), np.full((S, heads), -np.inf)
    tol_o, tol_l = np.zeros((S, heads, D)), np.zeros((S, heads))
    kinds = ROUND[q.dtype]
    q64 = q.double().cpu().numpy()
    tab, n_tok = table.cpu().numpy(), lens.cpu().numpy()
    for s in range(S):
        n = min(max(int(n_tok[s]), 0), P * ps)
        at = [j for j in range(n) if (not window or j >= n - window or j < sinks) and 0 <= tab[s, j // ps] < N]
        if not at:
            continue
        pages, places = torch.tensor([int(tab[s, j // ps]) for j in at]), torch.tensor([j % ps for j in at])
        kk = k[pages.to(k.device), :, places.to(k.device)].double().cpu().numpy()  # [tokens, H, D]
        vv = v[pages.to(v.device), :, places.to(v.device)].double().cpu().numpy()
        for h in range(heads):
            kh, vh = kk[:, h // G], vv[:, h // G]
            if k_scale is not None:
                kh, vh = kh * float(k_scale[h // G]), vh * float(v_scale[h // G])
            with np.errstate(all="ignore"):
                x = kh @ q64[s, h] * scale
                top = x.max()
                p = np.exp(x - top)
                o = (p[:, None] * vh).sum(0) / p.sum() if top > -np.inf else np.zeros(D)
                out[s, h] = o
                lse[s, h] = top + math.log(p.sum()) if top > -np.inf else -np.inf
                # a score's error: its products and their sum (the products of 16-bit numbers are exact), then
                # scale, k_scale and log2 e; a weight's: of its exponent, the exponential, and its two parts (2^-16)
                dx = ((D + 2) * EPS * (np.abs(kh) @ np.abs(q64[s, h])) * abs(scale) + 6 * EPS * np.abs(x) + 4 * EPS * abs(top)).max()
                rel = 2 * dx + 2.0 ** -16 + 2 * (len(at) + 16) * EPS
                mean = (p[:, None] * np.abs(vh)).sum(0) / p.sum()
                tol_o[s, h] = kinds * 1.01 * np.abs(o) + rel * mean + 2.0 ** -25
                tol_l[s, h] = dx + (len(at) + 16) * EPS + 4 * EPS * abs(lse[s, h])
    return out, lse, tol_o, tol_l


def step(table, lens, parents, grow, ps, N, held=None, window=0, sinks=0):
    """Tables, lens, refs, counters and the copies [(source, destination)] as the definition has them."""
    S0, P = table.shape
    S = S0 if parents is None else len(parents)
    rows, news, olds = [], [], []
    bad = cut = 0
    for s in range(S):
        par = s if parents is None else int(parents[s])
        if par < -1 or par >= S0:
            bad += 1
            par = -1
        L = min(max(int(lens[par]), 0), P * ps) if par >= 0 else 0
        g = max(int(grow[s]), 0) if grow is not None else 0
        if L + g > P * ps:
            cut += 1
        M = min(L + g, P * ps)
        row = [int(x) if 0 <= x < N else -1 for x in table[par][:-(-L // ps)]] if par >= 0 else []
        if window:
            first = L - window + (1 if M > L else 0)
            row = [-1 if (c + 1) * ps <= first and c * ps >= sinks else x for c, x in enumerate(row)]
        rows.append(row)
        olds.append(L)
        news.append(M)
    hold = [max(int(x), 0) for x in held] if held is not None else [0] * N
    refs = list(hold)
    for r in rows:
        for x in r:
            if x >= 0:
                refs[x] += 1
    free = [p for p in range(N) if refs[p] == 0]
    have, needed, copied, took, copies = len(free), 0, 0, 0, []

    def fresh():
        nonlocal needed, took
        needed += 1
        if took == have:
            return -1
        took += 1
        return free[took - 1]

    first_refs, first_rows = list(refs), [list(r) for r in rows]
    for s in range(S):
        L, M, row = olds[s], news[s], rows[s]
        if L % ps and M > L and row[-1] >= 0:
            page = row[-1]
            last = [o for o in range(S) if olds[o] % ps and first_rows[o] and first_rows[o][-1] == page]
            alone = (hold[page] == 0 and first_refs[page] == len(last)
                     and min(last, key=lambda o: (-olds[o], o)) == s)
            if not alone:
                row[-1] = fresh()
                refs[page] -= 1
                if row[-1] >= 0:
                    refs[row[-1]] += 1
                    copied += 1
                    copies.append((page, row[-1]))
        for _ in range(-(-M // ps) - -(-L // ps)):
            row.append(fresh())
            if row[-1] >= 0:
                refs[row[-1]] += 1
    out = np.full((S, P), -1, np.int32)
    for s, r in enumerate(rows):
        out[s, :len(r)] = r
    counters = [needed, needed - took, copied, sum(r > 0 for r in refs), bad, cut, 0, 0]
    return out, np.array(news, np.int32), np.array(refs, np.int32), np.array(counters, np.int32), copies


def compact(table, refs):
    N = len(refs)
    n = int((refs > 0).sum())
    holes = [p for p in range(n) if refs[p] <= 0]
    movers = [p for p in range(n, N) if refs[p] > 0]
    to = {p: p for p in range(n) if refs[p] > 0}
    to.update(zip(movers, holes))
    new = np.zeros(N, np.int32)
    for p, x in to.items():
        new[x] = refs[p]
    tab = np.array([[to.get(int(e), -1) for e in r] for r in table], np.int32).reshape(table.shape)
    m = np.array([to.get(p, -1) for p in range(N)], np.int32)
    return tab, new, m, np.array([n, len(movers), 0, 0, 0, 0, 0, 0], np.int32), list(zip(movers, holes))


def select(logits, scores, k, finished=None, eos=-1):
    """scores (64 bits), parents, tokens, finished.  logits [G, W, V], torch, any type."""
    G, W, V = logits.shape
    x = logits.double().cpu().numpy()
    sc = np.full((G, k), -np.inf)
    par, tok = np.full((G, k), -1, np.int32), np.full((G, k), -1, np.int32)
    fin = np.zeros((G, k), bool)
    for g in range(G):
        cands = []
        for w in range(W):
            base = float(scores[g, w])
            if finished is not None and finished[g, w]:
                if base > -np.inf:
                    cands.append((-base, w, 0.0, int(eos)))
                continue
            row = x[g, w]
            with np.errstate(all="ignore"):
                top = row.max()
                # (in this order: at 10^30 top + log has no place for the logarithm, in 64 bits either)
                val = base + ((row - top) - np.log(np.exp(row - top).sum()))
            ok = np.nonzero(val > -np.inf)[0]
            best = ok[np.lexsort((ok, -row[ok]))][:k]
            cands += [(-val[t], w, -row[t], int(t)) for t in best]
        cands.sort()
        for r, (v, w, _, t) in enumerate(cands[:k]):
            sc[g, r], par[g, r], tok[g, r] = -v, g * W + w, t
            fin[g, r] = bool(finished is not None and finished[g, w]) or (t == eos and eos >= 0)
    return sc, par, tok, fin
