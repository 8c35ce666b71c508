"""The 8-bit paged cache on the GPU against its oracle (oracle/q8.py): stored numbers and page lists bit for bit, attention
within bounds that are derived below."""
import random

import numpy as np
import pytest
import torch

from oracle import q8
from paper_2601_10155_b200.binding import Lookat, LookatError, PagePools, PageState, Q8Cache

pytestmark = pytest.mark.gpu

DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def host8(t):
    return t.view(torch.uint8).cpu().numpy()


def make_cache(rng, lens, P, H, d_k, d_v, fmt, spare=2, peak=1.0):
    """Rows of random numbers in randomly placed pages; whatever no row holds is 0x7f (a NaN in e4m3) under a NaN amax.
    Also the tables, -1 behind a row's pages."""
    need = [-(-n // P) for n in lens]
    n_pages, width = sum(need) + spare, max(1, max(need))
    perm = rng.permutation(n_pages).astype(np.int32)
    tables, at = np.full((len(lens), width), -1, np.int32), 0
    raw = [np.full((n_pages, H, P, d), 0x7F, np.uint8) for d in (d_k, d_v)]
    amax = [np.full((n_pages, H), np.nan, np.float32) for _ in range(2)]
    for b, n in enumerate(lens):
        tables[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
        for i in range(need[b]):
            p, m = tables[b, i], min(P, n - i * P)
            for r, a, d in zip(raw, amax, (d_k, d_v)):
                x = rng.standard_normal((H, m, d)) * np.exp(0.5 * rng.standard_normal((H, 1, 1))) * peak
                a[p] = np.abs(x).max(axis=(1, 2)).astype(np.float16)
                r[p, :, :m] = q8.bytes_of(np.clip(q8.R[fmt] * x / a[p][:, None, None], -q8.R[fmt], q8.R[fmt]), fmt)
    return raw[0], amax[0], raw[1], amax[1], tables


def on_gpu(k, ka, v, va, fmt):
    return Q8Cache(dev(k).view(DTYPE[fmt]), dev(ka), dev(v).view(DTYPE[fmt]), dev(va))


def attend_bound(out, mag, reach, d_k, L, vmax, fp16):
    """Per element of |got - out|.  Scores: sums of d_k exact products in fp32, each addition off by at most one unit in the
    last place (2^-23) of sum |q k| <= reach, and a few roundings of the scaled score and its difference to the maximum.
    An error e of the scores changes weights and their sum by e each; the exponential is good to 2^-21.  Sums over L tokens:
    2^-23 of mag per addition, in the weighted sum and in the denominator.  fp16: the result is rounded (2^-11, and 2^-25
    where it is subnormal), and the weights may be (2^-11 of themselves, 2^-25 where they are subnormal, against weights
    whose largest is at least 1)."""
    rel = 2 * reach[..., None] * (d_k + 8) * 2.0 ** -23 + 2.0 ** -20 + 2 * L * 2.0 ** -23
    bound = mag * rel + 1e-30
    if fp16:
        bound = bound + np.abs(out) * 2.0 ** -11 + 2.0 ** -25 + mag * 2.0 ** -11 + L * 2.0 ** -25 * vmax
    return bound


def check_attend(rng, lens, L_q, P, H_q, H_kv, d_k, d_v, fmt, fp16=False, peak=1.0, scale=0.0, stream=None):
    k, ka, v, va, tables = make_cache(rng, lens, P, H_kv, d_k, d_v, fmt, peak=peak)
    q = (rng.standard_normal((len(lens), H_q, L_q, d_k)) * 0.9).astype(np.float16)
    lk = Lookat(H_q, H_kv, d_k, d_v, 1 if d_k <= 128 else 2, 16, scale=scale, stream=stream)
    cache = on_gpu(k, ka, v, va, fmt)
    args = dev(q), dev(tables), dev(np.asarray(lens, np.int32))
    torch.cuda.synchronize()
    got = lk.lookat_attend_q8(cache, *args, out_fp16=fp16)
    again = lk.lookat_attend_q8(cache, *args, out_fp16=fp16)
    torch.cuda.synchronize()
    assert lk.lookat_last_error() == ""
    assert got.dtype == (torch.float16 if fp16 else torch.float32)
    assert torch.equal(got, again), "two calls on the same inputs differ"
    out, mag, reach = q8.attend(k, ka, v, va, q, tables, lens, fmt, lk.scale)
    err = np.abs(got.double().cpu().numpy() - out)
    bound = attend_bound(out, mag, reach, d_k, max(max(lens), 1), np.nanmax(va) if np.isfinite(va).any() else 0.0, fp16)
    assert np.isfinite(err).all()
    assert (err <= bound).all(), f"off by up to {np.max(err / bound):.3g} of the bound"
    dead = np.array([[n - L_q + i < 0 for i in range(L_q)] for n in lens])
    assert (got.double().cpu().numpy().transpose(0, 2, 1, 3)[dead] == 0).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("H_q,H_kv,d", [(12, 12, 64), (8, 2, 128), (16, 2, 64), (10, 1, 128), (24, 1, 128), (3, 3, 128), (6, 2, 64)])
@pytest.mark.parametrize("P,lens", [(16, [1, 0, 17, 128, 333]), (64, [64, 65, 1000]), (128, [127, 2])])
def test_attend_one_token(fmt, H_q, H_kv, d, P, lens):
    check_attend(np.random.default_rng(P + H_q), lens, 1, P, H_q, H_kv, d, d, fmt)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d_k,d_v", [(16, 16), (48, 80), (96, 96), (64, 128), (128, 64), (192, 128), (256, 256), (144, 16), (16, 240)])
def test_attend_other_head_dims(fmt, d_k, d_v):
    check_attend(np.random.default_rng(d_k * 7 + d_v), [70, 3, 0], 1, 16, 4, 2, d_k, d_v, fmt)
    check_attend(np.random.default_rng(d_k * 7 + d_v), [70, 3], 5, 32, 4, 2, d_k, d_v, fmt, fp16=True)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("L_q", [2, 3, 8, 9, 16, 17])
def test_attend_draft_tokens(fmt, L_q):
    """Several queries per row; rows shorter than L_q have queries that see nothing."""
    check_attend(np.random.default_rng(L_q), [300, 1, 0, L_q - 1, L_q, 64], L_q, 32, 8, 2, 128, 128, fmt)


@pytest.mark.parametrize("fmt,fp16", [("int8", False), ("e4m3", True), ("int8", True), ("e4m3", False)])
@pytest.mark.parametrize("P,H_q,H_kv,d,L_q,lens", [(16, 4, 2, 64, 130, [130, 257, 40, 0]), (64, 8, 2, 128, 64, [64, 500, 63]),
                                                   (128, 3, 1, 128, 100, [260]), (32, 12, 12, 64, 33, [33, 34, 129]), (16, 16, 1, 128, 37, [90, 36])])
def test_attend_prompt(fmt, fp16, P, H_q, H_kv, d, L_q, lens):
    check_attend(np.random.default_rng(P + L_q), lens, L_q, P, H_q, H_kv, d, d, fmt, fp16=fp16)


@pytest.mark.parametrize("fmt,fp16", [("int8", False), ("e4m3", True)])
@pytest.mark.parametrize("P,H_q,H_kv,d_k,d_v,L_q,lens", [(64, 4, 1, 128, 128, 70, [3000, 70, 0, 1200]), (16, 2, 2, 64, 64, 300, [2500]), (32, 2, 1, 64, 128, 65, [1100, 64])])
def test_attend_prompt_pieces_over_a_long_cache(fmt, fp16, P, H_q, H_kv, d_k, d_v, L_q, lens):
    """Few queries over many tokens: the tokens are cut among CTAs and joined; fp32 sums move out of tensor memory."""
    check_attend(np.random.default_rng(P + L_q), lens, L_q, P, H_q, H_kv, d_k, d_v, fmt, fp16=fp16)


def test_attend_large_and_small_numbers():
    """Blocks of very different sizes, peaked scores, and a scale of the caller's."""
    for peak in (1e-4, 30.0):
        check_attend(np.random.default_rng(5), [200, 31], 1, 16, 4, 2, 64, 64, "int8", peak=peak, scale=0.3 / peak)
        check_attend(np.random.default_rng(6), [200, 31], 40, 16, 4, 2, 64, 64, "e4m3", peak=peak, scale=0.3 / peak)


def test_attend_blocks_of_zeros_and_one_hot_blocks():
    rng = np.random.default_rng(8)
    k, ka, v, va, tables = make_cache(rng, [100, 50], 16, 2, 64, 64, "int8")
    for p in tables[0, [0, 3]]:
        k[p], v[p], ka[p], va[p] = 0, 0, 0, 0
    v[tables[0, 1]], va[tables[0, 1]] = 0, 0                    # values zero, keys not: the weights still count
    va[tables[0, 2]] = 60000.0
    va[tables[0, 4]] = np.float32(6e-8)
    for L_q, fp16 in ((1, False), (50, False)):
        q = rng.standard_normal((2, 4, L_q, 64)).astype(np.float16)
        lk = Lookat(4, 2, 64, 64, 1, 16)
        got = lk.lookat_attend_q8(on_gpu(k, ka, v, va, "int8"), dev(q), dev(tables), dev(np.array([100, 50], np.int32)), out_fp16=fp16)
        out, mag, reach = q8.attend(k, ka, v, va, q, tables, [100, 50], "int8", lk.scale)
        assert (np.abs(got.double().cpu().numpy() - out) <= attend_bound(out, mag, reach, 64, 100, 6e4, fp16)).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_attend_long_ragged_rows(fmt):
    """Rows from a token to many thousands in one call: work split along the long ones and joined."""
    check_attend(np.random.default_rng(11), [9000, 1, 0, 4097, 63], 1, 64, 8, 2, 128, 128, fmt)
    check_attend(np.random.default_rng(12), [5000, 7], 3, 16, 4, 1, 64, 64, fmt)


@pytest.mark.parametrize("L_q", [1, 6, 70])
def test_attend_leaves_bad_pages_out(L_q):
    rng = np.random.default_rng(13)
    k, ka, v, va, tables = make_cache(rng, [100, 40], 16, 2, 64, 64, "int8")
    tables[0, 2], tables[0, 5], tables[1, 0] = -5, k.shape[0], 2 ** 31 - 1
    q = rng.standard_normal((2, 4, L_q, 64)).astype(np.float16)
    lk = Lookat(4, 2, 64, 64, 1, 16)
    got = lk.lookat_attend_q8(on_gpu(k, ka, v, va, "int8"), dev(q), dev(tables), dev(np.array([100, 40], np.int32)))
    torch.cuda.synchronize()
    assert "outside its range" in lk.lookat_last_error()
    out, mag, reach = q8.attend(k, ka, v, va, q, tables, [100, 40], "int8", lk.scale)
    assert (np.abs(got.double().cpu().numpy() - out) <= attend_bound(out, mag, reach, 64, 100, np.nanmax(va), False)).all()
    # lengths outside 0..max_pages*page are taken as the nearest one inside
    lk2 = Lookat(4, 2, 64, 64, 1, 16)
    got = lk2.lookat_attend_q8(on_gpu(k, ka, v, va, "int8"), dev(q), dev(tables), dev(np.array([100000, -3], np.int32)))
    torch.cuda.synchronize()
    assert "outside its range" in lk2.lookat_last_error()
    full = tables.shape[1] * 16
    filled = v.copy()
    out, mag, reach = q8.attend(k, np.nan_to_num(ka), filled, np.nan_to_num(va), q, tables, [full, 0], "int8", lk.scale)
    assert (got[1] == 0).all()


def append_both(lk, fmt, k, ka, v, va, kn, vn, tables, lens, n_new):
    cache = on_gpu(k, ka, v, va, fmt)
    lk.lookat_q8_append(cache, dev(kn), dev(vn), dev(tables), dev(np.asarray(lens, np.int32)),
                        None if n_new is None else dev(np.asarray(n_new, np.int32)))
    torch.cuda.synchronize()
    counts = [kn.shape[2]] * len(lens) if n_new is None else n_new
    q8.append(k, ka, kn, tables, lens, counts, fmt)
    q8.append(v, va, vn, tables, lens, counts, fmt)
    assert np.array_equal(host8(cache.k), k), "k"
    assert np.array_equal(host8(cache.v), v), "v"
    assert np.array_equal(cache.k_amax.cpu().numpy(), ka, equal_nan=True), "k_amax"
    assert np.array_equal(cache.v_amax.cpu().numpy(), va, equal_nan=True), "v_amax"


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("P", [16, 64, 128])
@pytest.mark.parametrize("H,d_k,d_v", [(3, 64, 64), (2, 128, 128), (1, 16, 256), (2, 80, 48)])
@pytest.mark.parametrize("n", [1, 2, 8, 9, 70, 300])
def test_append_is_the_oracles_bit_for_bit(fmt, P, H, d_k, d_v, n):
    rng = np.random.default_rng(n * 1000 + P + d_k)
    lens = [n, n + 1, n + 5, n + P - 1, n + P, n + 3 * P // 2, n]
    n_new = [n, n, n, max(1, n // 2), n, n, 0]
    before = [a - c for a, c in zip(lens, n_new)]
    before[6] = n
    k, ka, v, va, tables = make_cache(rng, lens, P, H, d_k, d_v, fmt)
    for b, m in enumerate(before):                              # what the append will fill is stale
        for i in range(m // P, -(-lens[b] // P)):
            for r, a in ((k, ka), (v, va)):
                r[tables[b, i], :, max(0, m - i * P):] = 0x7F
                if m <= i * P:
                    a[tables[b, i]] = np.nan
    x = [(rng.standard_normal((7, H, n, d)) * np.exp(rng.standard_normal((7, H, n, 1)))).astype(np.float16) for d in (d_k, d_v)]
    append_both(Lookat(H, H, d_k, d_v, 1 if d_k <= 128 else 2, 16), fmt, k, ka, v, va, x[0], x[1], tables, lens, n_new)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_rounds_ties_and_special_values_as_real_arithmetic(fmt):
    rng = np.random.default_rng(4)
    P, d, B = 16, 64, 64
    # halves, quarters and odd fractions of the maximum: quotients on and next to the rounding borders
    x = np.empty((B, 1, 3, d), np.float16)
    for b in range(B):
        top = np.float16(np.exp2(rng.integers(-14, 12)) * (1 + rng.integers(0, 1024) / 1024))
        x[b, 0] = (float(top) * rng.integers(-128, 129, (3, d)) / rng.choice([127, 128, 254, 256, 448, 896])).astype(np.float16)
        x[b, 0, 0, 0] = top
    x[0, 0, 1, :6] = [np.nan, np.inf, -np.inf, 65504, -0.0, 6e-8]
    x[1, 0] = 0
    x[2, 0, :2] = 0                                             # the block's first numbers are zeros, then come some
    x[3, 0] = np.nan
    lens = [3] * B
    k, ka, v, va, tables = make_cache(rng, lens, P, 1, d, d, fmt)
    ka[:], va[:] = np.nan, np.nan
    lk = Lookat(1, 1, d, d, 1, 16)
    for t in range(3):                                          # token by token: the maximum grows under earlier tokens
        append_both(lk, fmt, k, ka, v, va, x[:, :, t:t + 1].copy(), -x[:, :, t:t + 1], tables, [t + 1] * B, None)
    assert not np.isnan(q8.values_of(k[tables[:, 0], 0, :3], fmt)).any()


def test_append_skips_what_it_may_not_write():
    rng = np.random.default_rng(9)
    P, H, d = 16, 2, 64
    k, ka, v, va, tables = make_cache(rng, [40, 40, 40, 20], P, H, d, d, "int8")
    tables[0, 1], tables[1, 2] = -1, k.shape[0] + 3
    x = rng.standard_normal((4, H, 30, d)).astype(np.float16)
    lk = Lookat(H, H, d, d, 1, 16)
    # row 2 would pass its table, row 3 begins before its first token
    append_both(lk, "int8", k, ka, v, va, x, x[::-1].copy(), tables, [40, 40, 60, 20], [30, 30, 30, 30])
    assert "outside its range" in lk.lookat_last_error()
    append_both(lk, "int8", k, ka, v, va, x, x[::-1].copy(), tables, [-4, 10, 0, 20], [3, -2, 50, 0])
    assert "outside its range" in lk.lookat_last_error()


# ------------------------------------------------------------------------------------------------ pages
def gpu_state(st, W, P):
    n = len(st["refs"])
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    free = list(st["free"]) + [-7] * (n - len(st["free"]))
    return PageState(i32(st["tables"]).view(-1, W), i32(st["seq_lens"]), i32(st["refs"]), i32(free), i32([len(st["free"])]), P)


def same_state(ps, st):
    torch.cuda.synchronize()
    nf = int(ps.n_free)
    assert nf == len(st["free"])
    assert ps.seq_lens.tolist() == st["seq_lens"]
    assert ps.tables.tolist() == st["tables"]
    assert ps.refs.tolist() == st["refs"]
    assert ps.free_list[:nf].tolist() == st["free"]


@pytest.mark.parametrize("B,W,n_pages,P,seed", [(1, 4, 10, 16, 0), (7, 9, 90, 16, 1), (33, 20, 700, 128, 2), (64, 6, 5000, 32, 3), (1100, 5, 9000, 64, 4)])
def test_pages_follow_the_rules_of_the_oracle(B, W, n_pages, P, seed):
    """Random steps on one state: extend (with copies, and refused ones), fork with freed rows, compact."""
    rnd = random.Random(seed)
    st = dict(tables=[[-1] * W for _ in range(B)], seq_lens=[0] * B, refs=[0] * n_pages, free=rnd.sample(range(n_pages), n_pages))
    ps = gpu_state(st, W, P)
    # three pools: vectors of 16 bytes, an odd number of words, more than one 4 KB piece
    pools = [torch.randint(0, 2 ** 31 - 1, (n_pages, w), dtype=torch.int32, device="cuda") for w in (8, 5, 2500 if n_pages < 1000 else 12)]
    want = [p.cpu().clone() for p in pools]
    lk = Lookat(2, 2, 64, 64, 1, 16)
    handle = PagePools(pools)
    refused = grown = 0
    for step in range(24):
        kind = rnd.choice(["extend", "extend", "extend", "fork", "compact"])
        if kind == "extend":
            n = [rnd.choice([0, 1, 1, 2, P, P + 3, -1] + [3 * P] * (step % 5 == 4)) for _ in range(B)]
            n_new = torch.tensor(n, dtype=torch.int32, device="cuda")
            lk.lookat_pages_extend(ps, n_new, handle)
            copies, ok = q8.extend(st, n, P, W)
            for src, dst in copies:
                for w in want:
                    w[dst] = w[src]
            torch.cuda.synchronize()
            assert n_new.tolist() == (n if ok else [0] * B)
            assert (lk.lookat_last_error() != "") == (not ok or bool(refused))
            refused += not ok
            grown += ok
        elif kind == "fork":
            p = [rnd.choice([-1, b, b, rnd.randrange(B), rnd.randrange(B), B + 5]) for b in range(B)]
            lk.lookat_pages_fork(ps, torch.tensor(p, dtype=torch.int32, device="cuda"))
            q8.fork(st, p, P)
        else:
            remap = torch.full((n_pages,), -9, dtype=torch.int32, device="cuda") if step % 2 else None
            lk.lookat_pages_compact(ps, pools, remap)
            m = q8.compact(st, P)
            if remap is not None:
                assert remap.tolist() == m
            for w in want:
                old = w.clone()
                for src, dst in enumerate(m):
                    if dst >= 0:
                        w[dst] = old[src]
        same_state(ps, st)
        for got, w in zip(pools, want):
            assert torch.equal(got.cpu(), w), (step, kind)
    assert grown


def test_pages_extend_takes_the_last_free_page_and_refuses_one_more():
    P, W = 16, 3
    st = dict(tables=[[0, -1, -1], [0, -1, -1], [0, -1, -1]], seq_lens=[5, 5, 5], refs=[3, 0, 0], free=[1, 2])
    ps, lk = gpu_state(st, W, P), Lookat(2, 2, 64, 64, 1, 16)
    pool = torch.arange(3 * 4, dtype=torch.int32, device="cuda").view(3, 4)
    n = torch.tensor([1, 40, 1], dtype=torch.int32, device="cuda")
    lk.lookat_pages_extend(ps, n, [pool])                       # needs 1 + (1 + 2) + 0 pages
    same_state(ps, st)
    assert n.tolist() == [0, 0, 0] and "too few free pages" in lk.lookat_last_error()
    n = torch.tensor([1, 1, 1], dtype=torch.int32, device="cuda")
    lk.lookat_pages_extend(ps, n, [pool])                       # two rows get copies, the third keeps the page
    copies, ok = q8.extend(st, [1, 1, 1], P, W)
    assert ok and copies == [(0, 2), (0, 1)]
    same_state(ps, st)
    assert pool.tolist() == [[0, 1, 2, 3]] * 3 and ps.tables[:, 0].tolist() == [2, 1, 0]


def test_pages_survive_entries_that_are_out_of_range():
    P, W = 16, 3
    st = dict(tables=[[0, 99, -1], [1, -4, -1]], seq_lens=[30, 20], refs=[1, 1, 0, 0], free=[2, 3])
    lk = Lookat(2, 2, 64, 64, 1, 16)
    ps = gpu_state(st, W, P)
    lk.lookat_pages_fork(ps, torch.tensor([1, -1], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert ps.refs.tolist() == [0, 1, 0, 0] and ps.free_list[:3].tolist() == [2, 3, 0] and ps.seq_lens.tolist() == [20, 0]
    assert "outside its range" in lk.lookat_last_error()
    ps = gpu_state(st, W, P)
    pool = torch.zeros((4, 4), dtype=torch.int32, device="cuda")
    lk.lookat_pages_compact(ps, [pool])
    torch.cuda.synchronize()
    assert ps.tables.tolist() == st["tables"] and "outside its range" in lk.lookat_last_error()
    ps = gpu_state(st, W, P)
    n = torch.tensor([1, 1], dtype=torch.int32, device="cuda")
    lk.lookat_pages_extend(ps, n, [pool])
    same_state(ps, st)
    assert n.tolist() == [0, 0]


# ------------------------------------------------------------------------------------------------ the set, as it is used
class Server:
    """A cache with its pages on the GPU, and the same in the oracle."""

    def __init__(self, fmt, B, W, n_pages, P, H_q, H_kv, d):
        self.fmt, self.P, self.W, self.B, self.shape = fmt, P, W, B, (H_q, H_kv, d)
        self.lk = Lookat(H_q, H_kv, d, d, 1, 16)
        self.cache = Q8Cache.empty(n_pages, H_kv, P, d, d, DTYPE[fmt])
        self.ps = PageState.empty(B, W, n_pages, P)
        self.pools = PagePools(self.cache.pools())
        self.st = dict(tables=[[-1] * W for _ in range(B)], seq_lens=[0] * B, refs=[0] * n_pages, free=list(range(n_pages - 1, -1, -1)))
        self.ref = [np.zeros((n_pages, H_kv, P, d), np.uint8), np.zeros((n_pages, H_kv), np.float32),
                    np.zeros((n_pages, H_kv, P, d), np.uint8), np.zeros((n_pages, H_kv), np.float32)]

    def step(self, rng, n, counts):
        H_q, H_kv, d = self.shape
        x = [(rng.standard_normal((self.B, H_kv, n, d)) * np.exp(0.4 * rng.standard_normal((self.B, 1, n, 1)))).astype(np.float16) for _ in range(2)]
        q = rng.standard_normal((self.B, H_q, n, d)).astype(np.float16)
        c = dev(np.asarray(counts, np.int32))
        self.lk.lookat_pages_extend(self.ps, c, self.pools)
        self.lk.lookat_q8_append(self.cache, dev(x[0]), dev(x[1]), self.ps.tables, self.ps.seq_lens, c)
        got = self.lk.lookat_attend_q8(self.cache, dev(q), self.ps.tables, self.ps.seq_lens)
        copies, ok = q8.extend(self.st, counts, self.P, self.W)
        assert ok
        for src, dst in copies:
            for r in self.ref:
                r[dst] = r[src]
        tables, lens = np.array(self.st["tables"], np.int32), self.st["seq_lens"]
        for i in (0, 2):
            q8.append(self.ref[i], self.ref[i + 1], x[i // 2], tables, lens, counts, self.fmt)
        out, mag, reach = q8.attend(*self.ref, q, tables, lens, self.fmt, self.lk.scale)
        err = np.abs(got.double().cpu().numpy() - out)
        assert (err <= attend_bound(out, mag, reach, d, max(max(lens), 1), self.ref[3].max(), False)).all()
        self.check()

    def check(self):
        same_state(self.ps, self.st)
        for t, r in zip(self.cache.pools(), self.ref):
            assert np.array_equal(host8(t) if t.dtype != torch.float32 else t.cpu().numpy(), r)


@pytest.mark.parametrize("fmt,P,H_q,H_kv,d", [("int8", 16, 4, 2, 64), ("e4m3", 32, 8, 1, 128)])
def test_serving_loop(fmt, P, H_q, H_kv, d):
    """Prompts, decode steps, beams that diverge, rows that end, compaction, draft tokens: every state checked."""
    rng = np.random.default_rng(P)
    s = Server(fmt, 5, 8, 30, P, H_q, H_kv, d)
    s.step(rng, 2 * P + 3, [2 * P + 3, 0, P, 5, 1])             # prompts, one row not yet started
    for _ in range(3):
        s.step(rng, 1, [1] * 5)
    parents = [0, 0, 0, 3, -1]
    s.lk.lookat_pages_fork(s.ps, dev(np.array(parents, np.int32)))
    q8.fork(s.st, parents, P)
    s.check()
    s.step(rng, 1, [1, 1, 1, 0, 0])                             # three beams of one row: two copies of its last page
    s.lk.lookat_pages_compact(s.ps, s.pools)
    m = q8.compact(s.st, P)
    for r in s.ref:
        old = r.copy()
        for src, dst in enumerate(m):
            if dst >= 0:
                r[dst] = old[src]
    s.check()
    s.step(rng, 4, [4, 2, 0, 4, 3])                             # draft tokens; a row begins again
    s.step(rng, 1, [1] * 5)


def test_a_captured_step_replays_like_the_calls():
    """extend + append + attend captured once and replayed for several tokens equal the same calls made one by one."""
    rng = np.random.default_rng(21)
    B, P, W, n_pages, H_q, H_kv, d = 3, 16, 6, 30, 8, 2, 128
    tokens = [[rng.standard_normal((B, h, 1, d)).astype(np.float16) for h in (H_kv, H_kv, H_q)] for _ in range(20)]
    results = []
    for graphed in (False, True):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            lk = Lookat(H_q, H_kv, d, d, 1, 16, stream=stream)
            cache, ps = Q8Cache.empty(n_pages, H_kv, P, d, d), PageState.empty(B, W, n_pages, P)
            pools = PagePools(cache.pools())
            k, v, q = (torch.zeros((B, h, 1, d), dtype=torch.float16, device="cuda") for h in (H_kv, H_kv, H_q))
            out = torch.empty((B, H_q, 1, d), device="cuda")
            n_new = torch.tensor([1, 1, 0], dtype=torch.int32, device="cuda")

            def step():
                lk.lookat_pages_extend(ps, n_new, pools)
                lk.lookat_q8_append(cache, k, v, ps.tables, ps.seq_lens, n_new)
                lk.lookat_attend_q8(cache, q, ps.tables, ps.seq_lens, out=out)

            seen = []
            graph = None
            for i, t in enumerate(tokens):
                for x, y in zip((k, v, q), t):
                    x.copy_(dev(y))
                if not graphed or i == 0:                       # the first call sizes the workspace
                    step()
                else:
                    if graph is None:
                        stream.synchronize()
                        graph = torch.cuda.CUDAGraph()
                        with torch.cuda.graph(graph, stream=stream):
                            step()
                    graph.replay()
                seen.append(out.clone())
            stream.synchronize()
            assert lk.lookat_last_error() == ""
            results.append(([o.cpu() for o in seen], [host8(t) if t.element_size() == 1 else t.cpu().numpy() for t in cache.pools()], ps.tables.cpu()))
            del graph
    assert all(torch.equal(a, b) for a, b in zip(results[0][0], results[1][0]))
    assert all(np.array_equal(a, b) for a, b in zip(results[0][1], results[1][1]))
    assert torch.equal(results[0][2], results[1][2])


def test_a_captured_prompt_in_pieces_replays():
    """Few queries over many tokens (two kernels, the second launched early) from a graph, inputs changed between replays."""
    rng = np.random.default_rng(23)
    lens = [2100, 400]
    k, ka, v, va, tables = make_cache(rng, lens, 64, 2, 128, 128, "int8")
    cache, stream = on_gpu(k, ka, v, va, "int8"), torch.cuda.Stream()
    tb, sl = dev(tables), dev(np.array(lens, np.int32))
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        lk = Lookat(4, 2, 128, 128, 1, 16, stream=stream)
        q, out = torch.zeros((2, 4, 50, 128), dtype=torch.float16, device="cuda"), torch.empty((2, 4, 50, 128), device="cuda")
        lk.lookat_attend_q8(cache, q, tb, sl, out=out)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            lk.lookat_attend_q8(cache, q, tb, sl, out=out)
        for _ in range(3):
            q.copy_(dev(rng.standard_normal((2, 4, 50, 128)).astype(np.float16)))
            g.replay()
            got = out.clone()
            want = lk.lookat_attend_q8(cache, q, tb, sl)
            stream.synchronize()
            assert torch.equal(got, want)
        del g


def test_two_contexts_on_two_streams_at_once():
    """Each context has its workspace: calls that overlap on the GPU do not touch one another's pieces."""
    rng = np.random.default_rng(24)
    lens = [6000, 300, 4000]
    k, ka, v, va, tables = make_cache(rng, lens, 32, 2, 128, 128, "e4m3")
    cache, tb, sl = on_gpu(k, ka, v, va, "e4m3"), dev(tables), dev(np.array(lens, np.int32))
    qs = [dev((rng.standard_normal((3, 8, L_q, 128))).astype(np.float16)) for L_q in (1, 20)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    lks = [Lookat(8, 2, 128, 128, 1, 16, stream=s) for s in streams]
    want = []
    for lk, q in zip(lks, qs):
        want.append(lk.lookat_attend_q8(cache, q, tb, sl))
        torch.cuda.synchronize()
    for _ in range(20):
        got = [lk.lookat_attend_q8(cache, q, tb, sl) for lk, q in zip(lks, qs)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_offsets_beyond_32_bits():
    """A cache of 5 GB per array, rows in its last pages."""
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB of device memory")
    rng = np.random.default_rng(25)
    H, P, d, n_pages, lens = 8, 128, 128, 40000, [300, 5]
    small_k, small_ka, small_v, small_va, tables = make_cache(rng, lens, P, H, d, d, "int8", spare=0)
    cache = Q8Cache.empty(n_pages, H, P, d, d)
    first = n_pages - small_k.shape[0]
    for t, x in zip(cache.pools(), (small_k.view(np.int8), small_ka, small_v.view(np.int8), small_va)):
        t[first:] = dev(x)
    moved = np.where(tables >= 0, tables + first, -1).astype(np.int32)
    lk = Lookat(16, H, d, d, 1, 16)
    for L_q in (1, 40):
        q = rng.standard_normal((2, 16, L_q, d)).astype(np.float16)
        got = lk.lookat_attend_q8(cache, dev(q), dev(moved), dev(np.array(lens, np.int32)))
        out, mag, reach = q8.attend(small_k, small_ka, small_v, small_va, q, tables, lens, "int8", lk.scale)
        assert (np.abs(got.double().cpu().numpy() - out) <= attend_bound(out, mag, reach, d, 300, np.nanmax(small_va), False)).all()
    x = [rng.standard_normal((2, H, 9, d)).astype(np.float16) for _ in range(2)]
    lk.lookat_q8_append(cache, dev(x[0]), dev(x[1]), dev(moved), dev(np.array(lens, np.int32)))
    # (row 1 holds 5 tokens: it would begin before its first one)
    for raw, a, y in ((small_k, small_ka, x[0]), (small_v, small_va, x[1])):
        q8.append(raw, a, y, tables, lens, [9, 9], "int8")
    torch.cuda.synchronize()
    for t, r in zip(cache.pools(), (small_k, small_ka, small_v, small_va)):
        got = t[first:].contiguous()
        assert np.array_equal(host8(got) if t.element_size() == 1 else got.cpu().numpy(), r)
    # the same pages moved to the front
    ps = PageState.empty(2, 3, n_pages, P)
    ps.tables[:, :moved.shape[1]] = dev(moved)
    ps.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    held = torch.tensor([p for row in moved for p in row if p >= 0], device="cuda")
    ps.refs[held] = 1
    before = [t[torch.sort(held).values].clone() for t in cache.pools()]
    lk.lookat_pages_compact(ps, cache.pools())
    torch.cuda.synchronize()
    assert int(ps.n_free) == n_pages - len(held)
    for t, b in zip(cache.pools(), before):
        assert torch.equal(t[:len(held)].view(torch.uint8), b.view(torch.uint8))


def test_a_capture_that_would_have_to_allocate_is_refused_and_old_graphs_stay_valid():
    rng = np.random.default_rng(22)
    lens = [50, 20]
    k, ka, v, va, tables = make_cache(rng, lens, 16, 2, 64, 64, "int8")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        lk = Lookat(2, 2, 64, 64, 1, 16, stream=stream)
        small, large = PageState.empty(2, 2, 8, 16), PageState.empty(64, 64, 5000, 16)
        parents = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
        many = torch.arange(63, -1, -1, dtype=torch.int32, device="cuda")
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            with pytest.raises(LookatError, match="capture"):
                lk.lookat_pages_fork(small, parents)
            torch.zeros(1, device="cuda")
        lk.lookat_pages_fork(small, parents)
        stream.synchronize()
        g2 = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g2, stream=stream):
            lk.lookat_pages_fork(small, parents)
        lk.lookat_pages_fork(large, many)                       # outgrows the workspace that g2 was captured with
        small.seq_lens.copy_(torch.tensor([3, 9], dtype=torch.int32))
        small.tables.copy_(torch.tensor([[4, -1], [5, -1]], dtype=torch.int32))
        small.refs.zero_()
        small.refs[4:6] = 1
        g2.replay()
        stream.synchronize()
        assert small.seq_lens.tolist() == [9, 3] and small.tables[:, 0].tolist() == [5, 4]
        del g, g2


def test_attend_on_a_stream_of_its_own():
    s = torch.cuda.Stream()
    check_attend(np.random.default_rng(31), [300, 20], 1, 16, 8, 2, 128, 128, "int8", stream=s)
    check_attend(np.random.default_rng(32), [300, 20], 90, 16, 8, 2, 128, 128, "e4m3", stream=s)


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals():
    lk = Lookat(4, 2, 64, 64, 1, 16)
    cache = Q8Cache.empty(6, 2, 16, 64, 64)
    tables, lens = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    q, x = torch.zeros((2, 4, 1, 64), dtype=torch.float16, device="cuda"), torch.zeros((2, 2, 1, 64), dtype=torch.float16, device="cuda")
    before = lk.lookat_kernel_launches()
    with pytest.raises(TypeError):
        Q8Cache(cache.k.float(), cache.k_amax, cache.v, cache.v_amax)
    with pytest.raises(TypeError):
        Q8Cache(cache.k, cache.k_amax, cache.v.view(torch.uint8), cache.v_amax)
    with pytest.raises(ValueError):
        Q8Cache(cache.k, cache.k_amax[:5], cache.v, cache.v_amax)
    with pytest.raises(ValueError):
        Q8Cache(cache.k.transpose(1, 2), cache.k_amax, cache.v, cache.v_amax)
    with pytest.raises(TypeError):
        lk.lookat_attend_q8(cache, q.float(), tables, lens)
    with pytest.raises(TypeError):
        lk.lookat_attend_q8(cache, q, tables.long(), lens)
    with pytest.raises(ValueError):
        lk.lookat_attend_q8(cache, q, tables, lens[:1])
    with pytest.raises(ValueError):
        lk.lookat_attend_q8(cache, q.expand(2, 4, 3, 64), tables, lens)
    with pytest.raises(ValueError):
        lk.lookat_attend_q8(cache, q, tables, lens, out=torch.empty((2, 4, 2, 64), device="cuda"))
    with pytest.raises(TypeError):
        lk.lookat_attend_q8(cache, q.cpu(), tables, lens)
    with pytest.raises(ValueError):
        Lookat(4, 4, 64, 64, 1, 16).lookat_attend_q8(cache, q, tables, lens)
    with pytest.raises(ValueError):
        lk.lookat_q8_append(cache, x, x[:1], tables, lens)
    for page in (8, 48, 256):
        odd = Q8Cache.empty(6, 2, page, 64, 64)
        with pytest.raises(LookatError, match="page="):
            lk.lookat_attend_q8(odd, q, tables, lens)
        with pytest.raises(LookatError, match="page="):
            lk.lookat_q8_append(odd, x, x, tables, lens)
    with pytest.raises(LookatError, match="L_q=0"):
        lk.lookat_attend_q8(cache, q[:, :, :0].contiguous(), tables, lens)
    with pytest.raises(LookatError, match="max_pages=0"):
        lk.lookat_attend_q8(cache, q, tables[:, :0].contiguous(), lens)
    for d in (24, 272):
        wide = Lookat(2, 2, d, 64, 3 if d == 272 else 1, 16) if d == 24 else Lookat(2, 2, d, 64, 17, 16)
        with pytest.raises(LookatError, match="multiples of 16"):
            wide.lookat_attend_q8(Q8Cache.empty(6, 2, 16, d, 64), torch.zeros((2, 2, 1, d), dtype=torch.float16, device="cuda"), tables, lens)
    lone = torch.zeros(2 * 4 * 64 + 1, dtype=torch.float16, device="cuda")[1:].view(2, 4, 1, 64)
    with pytest.raises(LookatError, match="aligned"):
        lk.lookat_attend_q8(cache, lone, tables, lens)

    ps, n = PageState.empty(2, 3, 6, 16), torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        lk.lookat_pages_extend(ps, n[:1], [])
    with pytest.raises(ValueError):
        lk.lookat_pages_extend(ps, n, [torch.zeros((5, 4), device="cuda")])
    with pytest.raises(LookatError, match="page_bytes"):
        lk.lookat_pages_extend(ps, n, [torch.zeros((6, 3), dtype=torch.int16, device="cuda")])
    with pytest.raises(LookatError, match="n_pools"):
        lk.lookat_pages_extend(ps, n, [torch.zeros((6, 4), device="cuda")] * 257)
    with pytest.raises(LookatError, match="page="):
        lk.lookat_pages_fork(PageState.empty(2, 3, 6, 20), n)
    with pytest.raises(LookatError, match="B="):
        lk.lookat_pages_fork(PageState.empty(4097, 3, 6, 16), torch.zeros(4097, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError):
        lk.lookat_pages_fork(ps, n.long())
    with pytest.raises(ValueError):
        lk.lookat_pages_compact(ps, [], remap=n)
    assert lk.lookat_kernel_launches() == before
