"""CPU oracle of what a server runs around the 8-bit paged cache (numpy, fp64 and Python integers).

TEST INFRASTRUCTURE ONLY, like the rest of this package.  It states include/lookat_serve.h plainly: one row, one head, one
candidate at a time.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np


# ---- rotary positions
def rope_frequencies(r, base, scaling="none", factor=1.0, original_len=0.0, low=1.0, high=32.0):
    """(radians per position of each pair, factor on cosines and sines)"""
    if scaling == "base":
        base = base * factor ** (r / (r - 2))
    f = [base ** (-2 * i / r) for i in range(r // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling in ("bands", "ramp"):
        if scaling == "bands":
            keep = [(original_len * x / (2 * math.pi) - low) / (high - low) for x in f]
        else:
            at = lambda u: r * math.log(original_len / (2 * math.pi * u)) / (2 * math.log(base))  # noqa: E731
            i0, i1 = max(math.floor(at(high)), 0), min(math.ceil(at(low)), r - 1)
            keep = [1 - (i - i0) / max(i1 - i0, 0.001) for i in range(r // 2)]
        keep = [min(max(c, 0.0), 1.0) for c in keep]
        f = [x * (c + (1 - c) / factor) for x, c in zip(f, keep)]
    return f, 0.1 * math.log(factor) + 1 if scaling == "ramp" else 1.0


def rope(x, positions, turns, amplitude, interleaved):
    """x [T][H][d]; turns: whole numbers, fractions of 2^64 per position.  fp64."""
    x = np.asarray(x).astype(np.float64)
    y = x.copy()
    c = len(turns)
    for t, p in enumerate(positions):
        for i, f in enumerate(turns):
            at = (int(p) * int(f)) % (1 << 64)
            angle = 2 * math.pi * float(Fraction(at if at < 1 << 63 else at - (1 << 64), 1 << 64))
            cos, sin = amplitude * math.cos(angle), amplitude * math.sin(angle)
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + c)
            y[t, :, a] = x[t, :, a] * cos - x[t, :, b] * sin
            y[t, :, b] = x[t, :, b] * cos + x[t, :, a] * sin
    return y


# ---- attention of packed prompts
def attend_packed(q, k, v, starts, scale):
    """(out, sum of weight * |value|, largest sum |q k| scale) per query, fp64; zeros for tokens of no row."""
    q, k, v = (np.asarray(x).astype(np.float64) for x in (q, k, v))
    T, H, _ = q.shape
    g = H // k.shape[1]
    out, mag, reach = np.zeros((T, H, v.shape[2])), np.zeros((T, H, v.shape[2])), np.zeros((T, H))
    for lo, hi in zip(starts[:-1], starts[1:]):
        for h in range(H):
            for t in range(lo, hi):
                kk, vv = k[lo:t + 1, h // g], v[lo:t + 1, h // g]
                s = kk @ q[t, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h], mag[t, h] = w @ vv, w @ np.abs(vv)
                reach[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * scale
    return out, mag, reach


# ---- beam search
def beam_select(scores, lengths, finished, tokens, logits, eos, penalty):
    """The new (scores fp64, lengths, finished, tokens, next_ids, parents, gap): gap is the least distance between the ranks of
    neighbours among the chosen and the first that was not (infinite where there is none)."""
    G, W = scores.shape
    V = logits.shape[1]
    out_s, out_l, out_f = np.full((G, W), -math.inf), lengths.copy(), finished.copy()
    out_t = None if tokens is None else tokens.copy()
    ids, parents = np.full((G, W), max(eos, 0)), np.arange(G * W).reshape(G, W).copy()
    gap = math.inf
    for gr in range(G):
        cands = []
        for w in range(W):
            s = float(scores[gr, w])
            if not math.isfinite(s):
                continue
            if finished[gr, w]:
                cands.append((s / max(int(lengths[gr, w]), 1) ** penalty, w * V + max(eos, 0), s))
                continue
            x = logits[gr * W + w].astype(np.float64)
            top = x.max()
            if not math.isfinite(top):
                continue
            score = s + ((x - top) - math.log(math.fsum(np.exp(x - top))))
            rank = score / max(int(lengths[gr, w]) + 1, 1) ** penalty
            best = np.argsort(-rank, kind="stable")[:W + 1]
            cands += [(rank[c], w * V + int(c), score[c]) for c in best if score[c] > -math.inf]
        cands.sort(key=lambda c: (-c[0], c[1]))
        for a, b in zip(cands[:W], cands[1:W + 1]):
            if a[0] != b[0]:
                gap = min(gap, a[0] - b[0])
        for place, (_, at, score) in enumerate(cands[:W]):
            w, c = at // V, at % V
            was, done = int(lengths[gr, w]), bool(finished[gr, w])
            out_s[gr, place], parents[gr, place], ids[gr, place] = score, gr * W + w, c
            out_l[gr, place] = was + (not done)
            out_f[gr, place] = done or c == eos
            if out_t is not None:
                out_t[gr, place] = tokens[gr, w]
                if not done and 0 <= was < out_t.shape[2]:
                    out_t[gr, place, was] = c
        for place in range(len(cands[:W]), W):
            out_f[gr, place] = bool(finished[gr, place])
    return out_s, out_l, out_f.astype(np.int32), out_t, ids.reshape(-1), parents.reshape(-1), gap
