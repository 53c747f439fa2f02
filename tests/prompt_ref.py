"""The operators of a prompt's pass from their definitions, on the CPU in 64 bits, and how far a result
in 32 bits may be from them."""
from __future__ import annotations

import numpy as np
import torch

from decode_ref import EPS, ROUND


def attend(q, k, v, table, lens, offsets, scale, window=0, sinks=0, k_scale=None, v_scale=None):
    """(out, lse, tolerances of both, whether a row is a sequence's).  q [rows, heads, D], k and v [pages, H, ps, D]."""
    R, heads, D = q.shape
    N, H, ps, _ = k.shape
    G, P, S = heads // H, table.shape[1], table.shape[0]
    out, lse = np.zeros((R, heads, D)), np.full((R, heads), -np.inf)
    tol_o, tol_l = np.zeros((R, heads, D)), np.zeros((R, heads))
    real = np.zeros(R, bool)
    half = ROUND[q.dtype]
    q64, tab = q.double().cpu().numpy(), table.cpu().numpy()
    ends, n_tok = offsets.cpu().numpy(), lens.cpu().numpy()
    for s in range(S):
        a, b = int(ends[s]), int(ends[s + 1])
        n = min(max(int(n_tok[s]), 0), P * ps)
        real[a:b] = True
        if a == b or n == 0:
            continue
        pos = np.arange(a, b) - b + n
        at = np.array([j for j in range(n) if 0 <= tab[s, j // ps] < N], dtype=np.int64)
        if not len(at):
            continue
        seen = at <= pos[:, None]
        if window:
            seen &= (at > pos[:, None] - window) | (at < sinks)
        some = seen.any(0)
        at, seen = at[some], seen[:, some]
        if not len(at):
            continue
        pages, places = torch.from_numpy(tab[s, at // ps].astype(np.int64)), torch.from_numpy(at % ps)
        kk = k[pages.to(k.device), :, places.to(k.device)].double().cpu().numpy()  # [tokens, H, D]
        vv = v[pages.to(v.device), :, places.to(v.device)].double().cpu().numpy()
        for h in range(heads):
            kh, vh = kk[:, h // G], vv[:, h // G]
            if k_scale is not None:
                kh, vh = kh * float(k_scale[h // G]), vh * float(v_scale[h // G])
            with np.errstate(all="ignore"):
                x = q64[a:b, h] @ kh.T * scale
                x[~seen] = -np.inf
                top = x.max(1, keepdims=True)
                fine = top[:, 0] > -np.inf
                safe = np.where(fine[:, None], top, 0.0)
                p = np.exp(x - safe)
                total = p.sum(1, keepdims=True)
                div = np.where(fine[:, None], total, 1.0)
                odd = ~np.isfinite(vh).all()
                if odd:  # (what is not seen has no part, whatever it is)
                    o = np.stack([(p[i, seen[i]][:, None] * vh[seen[i]]).sum(0) for i in range(b - a)]) / div
                else:
                    o = p @ vh / div
                out[a:b, h] = np.where(fine[:, None], o, 0.0)
                lse[a:b, h] = np.where(fine, safe[:, 0] + np.log(div[:, 0]), -np.inf)
                # a score's error: its products and their sum (the products of 16-bit numbers are exact), then
                # scale, k_scale and log2 e; a weight's: of its exponent, the exponential, and its rounding to 16
                # bits (in fp16 to 2^-32 of the largest at least)
                size = np.where(seen, np.abs(q64[a:b, h]) @ np.abs(kh).T * abs(scale), 0.0)
                big = np.where(seen & np.isfinite(x), np.abs(x), 0.0)
                dx = ((D + 2) * EPS * size + 6 * EPS * big + 4 * EPS * np.abs(safe)).max(1, keepdims=True)
                rel = 2 * dx + half + 2 * (len(at) + 16) * EPS
                # (a value that is not finite is the same in both, or the row is odd and looked at by itself)
                vf = np.where(np.isfinite(vh), np.abs(vh), 0.0)
                mean = p @ vf / div
                tol_o[a:b, h] = half * 1.01 * np.abs(np.where(np.isfinite(o), o, 0.0)) + rel * mean + 2.0 ** -25 \
                    + len(at) * 2.0 ** -32 * vf.max()
                tol_l[a:b, h] = dx[:, 0] + (len(at) + 16) * EPS + 4 * EPS * np.abs(np.where(fine, lse[a:b, h], 0.0))
    return out, lse, tol_o, tol_l, real


def positions(starts, offsets, rows):
    """(sequence or -1, position) of each row."""
    starts = starts.cpu().numpy().astype(np.int64)
    if offsets is None:
        return np.arange(rows), starts[:rows]
    ends = offsets.cpu().numpy().astype(np.int64)
    seq, pos = np.full(rows, -1), np.zeros(rows, np.int64)
    for s in range(len(starts)):
        for r in range(ends[s], ends[s + 1]):
            seq[r], pos[r] = s, starts[s] + r - ends[s]
    return seq, pos


def turn(x, pos, frequencies, interleaved, amplitude):
    """(turned rows in 64 bits, how far 32 bits may be off before the last rounding).  x [rows, heads, D]."""
    x = x.double().cpu().numpy()
    f = frequencies.cpu().numpy()
    n = len(f)
    a = pos[:, None] * f  # 64 bits: off by 2^-53 of an angle of up to 2^31
    c, s = np.cos(a)[:, None] * amplitude, np.sin(a)[:, None] * amplitude
    i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    y, tol = x.copy(), np.zeros_like(x)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    # the part of a turn behind the point is rounded to 2^-26, its cosine and sine to two steps: 2.5e-7; the
    # products and their sum add three halves of one
    tol[..., i] = tol[..., j] = (np.abs(x[..., i]) + np.abs(x[..., j])) * abs(amplitude) * 2.0 ** -21
    return y, tol


def score(logits, tokens, top):
    """dict of logprobs, entropy, ranks, top_logprobs, top_tokens, and tolerances."""
    x = logits.double().cpu().numpy()
    R, V = x.shape
    tok = tokens.cpu().numpy()
    out = dict(logprobs=np.full(R, np.nan), entropy=np.full(R, np.nan), ranks=np.full(R, -1, np.int32),
               top_logprobs=np.full((R, top), np.nan), top_tokens=np.full((R, top), -1, np.int32))
    tol = dict(logprobs=np.zeros(R), entropy=np.zeros(R), top_logprobs=np.zeros((R, top)))
    for r in range(R):
        row = x[r]
        m = row.max()
        if np.isnan(row).any() or not np.isfinite(m):
            continue
        d = row - m
        e = np.exp(d)
        S = e.sum()
        fine = e > 0
        T = (e[fine] * d[fine]).sum()
        log = np.log(S)
        out["entropy"][r] = log - T / S
        # weights: of d, its product with log2 e, the exponential; sums: an addition for each 256th of the
        # row and 64 more of steps, lanes, waves and parts, as many moves of up to four roundings
        adds = V / 256 + 64
        each = np.where(fine, 2 * np.abs(np.where(fine, d, 0.0)) + 4, 0.0) * EPS
        rel = (e * each).sum() / S + 4 * adds * EPS
        relT = (e[fine] * np.abs(d[fine]) * each[fine]).sum() / S + 5 * adds * EPS * abs(T) / S
        tol["entropy"][r] = rel + 4 * EPS * log + relT + abs(T) / S * (rel + 4 * EPS) + 2 * EPS * abs(out["entropy"][r])
        order = np.lexsort((np.arange(V), -row))
        order = order[np.isfinite(row[order])]
        lp = lambda t: (row[t] - m) - log  # noqa: E731
        tl = lambda t: rel + EPS * (np.abs(row[t] - m) + 4 * log + 2 * np.abs(lp(t)))  # noqa: E731
        t = int(tok[r])
        if 0 <= t < V:
            out["logprobs"][r], out["ranks"][r] = lp(t), (row > row[t]).sum() + (row[:t] == row[t]).sum()
            tol["logprobs"][r] = tl(t) if np.isfinite(row[t]) else 0.0
        else:
            out["logprobs"][r] = -np.inf
        k = min(top, len(order))
        out["top_tokens"][r, :k], out["top_logprobs"][r, :k], out["top_logprobs"][r, k:] = order[:k], lp(order[:k]), -np.inf
        tol["top_logprobs"][r, :k] = tl(order[:k])
    return out, tol
