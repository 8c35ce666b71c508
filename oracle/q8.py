"""CPU oracle of the 8-bit paged cache (numpy, fp64 and Python integers).

TEST INFRASTRUCTURE ONLY, like the rest of this package.  It states include/lookat_q8.h plainly: one block, one row, one
page at a time, in the order the text gives.
"""
from __future__ import annotations

import math

import numpy as np

R = {"int8": 127.0, "e4m3": 448.0}


def e4m3_values():
    """The value of each of the 256 bytes (0x7f and 0xff are NaN)."""
    out = np.zeros(256)
    for byte in range(256):
        e, f = (byte >> 3) & 15, byte & 7
        x = f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        out[byte] = math.nan if e == 15 and f == 7 else (-x if byte & 0x80 else x)
    return out


_E4M3 = e4m3_values()


def values_of(raw, fmt):
    """The numbers held by an array of bytes."""
    return raw.view(np.int8).astype(np.float64) if fmt == "int8" else _E4M3[raw]


def bytes_of(x, fmt):
    """The bytes of the 8-bit numbers nearest to x, ties to even."""
    x = np.asarray(x, dtype=np.float64)
    if fmt == "int8":
        return np.clip(np.rint(x), -127, 127).astype(np.int8).view(np.uint8)
    grid = _E4M3[:127]                                          # 0 .. 448 ascending
    mag = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(grid, mag), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - mag, mag - grid[lo]
    pick = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return (pick | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def finite(x):
    """fp16 input as the append takes it."""
    return np.nan_to_num(np.asarray(x).astype(np.float64), nan=0.0, posinf=65504.0, neginf=-65504.0)


def append(raw, amax, x, tables, seq_lens, n_new, fmt):
    """In place: raw uint8 [n_pages][H][page][d], amax [n_pages][H]; x fp16 [B][H][n][d]."""
    n_pages, H, P, d = raw.shape
    x = finite(x)
    cap = tables.shape[1] * P
    for b in range(len(seq_lens)):
        count = min(max(int(n_new[b]), 0), x.shape[2])
        first = int(seq_lens[b]) - count
        by_block = {}
        for i in range(count):
            t = first + i
            if 0 <= t < min(max(int(seq_lens[b]), 0), cap):
                by_block.setdefault(t // P, []).append((t % P, i))
        for blk, items in by_block.items():
            p = int(tables[b][blk])
            if not 0 <= p < n_pages:
                continue
            at, src = [o for o, _ in items], [i for _, i in items]
            for h in range(H):
                new = x[b, h, src]
                was = max(float(amax[p, h]), 0.0) if at[0] > 0 else 0.0
                now = max(was, float(np.abs(new).max()))
                if at[0] > 0 and now > was > 0:
                    kept = values_of(raw[p, h, : at[0]], fmt)
                    raw[p, h, : at[0]] = bytes_of(kept * was / now, fmt)
                raw[p, h, at] = bytes_of(R[fmt] * new / now, fmt) if now > 0 else 0
                amax[p, h] = now


def attend(k_raw, k_amax, v_raw, v_amax, q, tables, seq_lens, fmt, scale):
    """(out [B][H_q][L_q][d_v], mag: sum_t alpha_t |v_t| of the same shape, reach: the largest sum_d |q_d k_d| * scale that a
    query meets, [B][H_q][L_q]) in fp64."""
    q = np.asarray(q).astype(np.float64)
    B, Hq, Lq, _ = q.shape
    n_pages, H, P, d_v = v_raw.shape
    g = Hq // H
    out, mag, reach = np.zeros((B, Hq, Lq, d_v)), np.zeros((B, Hq, Lq, d_v)), np.zeros((B, Hq, Lq))
    for b in range(B):
        n = min(max(int(seq_lens[b]), 0), tables.shape[1] * P)
        tok = [(int(tables[b][t // P]), t % P, t) for t in range(n)]
        tok = [x for x in tok if 0 <= x[0] < n_pages]
        if not tok:
            continue
        p, o, pos = (np.array(x) for x in zip(*tok))
        for h in range(H):
            k = values_of(k_raw[p, h, o], fmt) * (k_amax[p, h].astype(np.float64) / R[fmt])[:, None]
            v = values_of(v_raw[p, h, o], fmt) * (v_amax[p, h].astype(np.float64) / R[fmt])[:, None]
            for r in range(h * g, h * g + g):
                for i in range(Lq):
                    see = pos <= n - Lq + i
                    if not see.any():
                        continue
                    s = k[see] @ q[b, r, i] * scale
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    out[b, r, i] = w @ v[see]
                    mag[b, r, i] = w @ np.abs(v[see])
                    reach[b, r, i] = (np.abs(k[see]) @ np.abs(q[b, r, i])).max() * scale
    return out, mag, reach


# ---- pages: a state is a dict of lists: tables (rows of page ids), seq_lens, refs, free (the stack) ----
def extend(st, n_new, page, max_pages):
    """(copies [(src, dst)], ok); the state is changed in place only if ok."""
    tables, lens, refs, free = [list(r) for r in st["tables"]], list(st["seq_lens"]), list(st["refs"]), list(st["free"])
    copies = []
    for b, n in enumerate(n_new):
        n = max(int(n), 0)
        L = lens[b]
        if not 0 <= L <= max_pages * page or L + n > max_pages * page:
            return [], False
        have, need = -(-L // page), -(-(L + n) // page)
        if n and L % page:
            last = tables[b][have - 1]
            if not 0 <= last < len(refs):
                return [], False
            if refs[last] > 1:
                if not free:
                    return [], False
                p = free.pop()
                refs[last] -= 1
                refs[p] = 1
                tables[b][have - 1] = p
                copies.append((last, p))
        for i in range(have, need):
            if not free:
                return [], False
            p = free.pop()
            refs[p] = 1
            tables[b][i] = p
        lens[b] = L + n
    st.update(tables=tables, seq_lens=lens, refs=refs, free=free)
    return copies, True


def fork(st, parents, page):
    tables, lens, refs = st["tables"], st["seq_lens"], st["refs"]
    blocks = [-(-n // page) for n in lens]
    new_tables, new_lens = [list(r) for r in tables], []
    for b, p in enumerate(parents):
        if 0 <= p < len(tables):
            new_tables[b][: blocks[p]] = tables[p][: blocks[p]]
            new_lens.append(lens[p])
        else:
            new_lens.append(0)
    before = list(refs)
    for b in range(len(tables)):
        for p in tables[b][: blocks[b]]:
            refs[p] -= 1
    for b, n in enumerate(new_lens):
        for p in new_tables[b][: -(-n // page)]:
            refs[p] += 1
    st["free"] += [p for p in range(len(refs)) if before[p] > 0 and refs[p] == 0]
    st.update(tables=new_tables, seq_lens=new_lens)


def compact(st, page):
    """remap: page -> its new id, -1 for pages that nobody holds."""
    refs = st["refs"]
    n = len(refs)
    live = [p for p in range(n) if refs[p] > 0]
    gaps = [p for p in range(len(live)) if refs[p] <= 0]
    remap = [p if refs[p] > 0 else -1 for p in range(n)]
    for src, dst in zip([p for p in live if p >= len(live)], gaps):
        remap[src] = dst
    st["tables"] = [[remap[p] if i < -(-m // page) else p for i, p in enumerate(row)] for row, m in zip(st["tables"], st["seq_lens"])]
    st["refs"] = [0] * n
    for p in live:
        st["refs"][remap[p]] = refs[p]
    # pages that nobody holds keep refs as they are (0)
    st["free"] = list(range(n - 1, len(live) - 1, -1))
    return remap


# ---- how far fp32 attention may be off ----
def attend_rms_tolerance(reach, d_k, L):
    """Bound of ||got - out|| / ||out|| for fp32 results over values that do not depend on the scores.

    A relative error e_t of the weights alpha_t changes the result by sum_t alpha_t e_t (v_t - out).  Values of independent
    signs add up as alpha_t v_t do in out itself, so the norm of that is at most the largest |e_t| of out's norm, twice that
    with the share in the denominator.  |e_t|: a score is d_k / 16 products of 16 dims that are added one after another,
    each addition off by at most 2^-23 of sum |q k| <= reach, then a few roundings of the scaled score, its block's exponent
    (a few units) and its distance to the maximum; the exponential and the weight's two fp16 numbers are good to 2^-22 each.
    Sums: chains of up to 64 additions in the tensor pipe, which cuts off (2^-23 each), and roundings of independent sign in
    the fp32 sums over the tokens (2^-24 times the root of their number)."""
    e = (d_k / 16 + 6) * 2.0 ** -23 * (float(np.max(reach)) + 4) + 2 * 2.0 ** -22
    return 2 * e + 64 * 2.0 ** -23 + math.sqrt(L) * 2.0 ** -24
