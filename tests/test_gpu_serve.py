"""Rotary positions, attention of packed prompts, packed appends and beam selection on the GPU against their oracle
(oracle/serve.py), within bounds that are derived below."""
import math
import sys
import threading

import numpy as np
import pytest
import torch

from oracle import q8, serve
from paper_2601_10155_b200.binding import BeamState, Lookat, LookatError, PageState, Q8Cache, RopeTable

pytestmark = pytest.mark.gpu

DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts_of(lens, first=0):
    return np.concatenate([[first], first + np.cumsum(lens)]).astype(np.int32)


def finding(lk):
    torch.cuda.synchronize()
    return lk.lookat_last_error()


# ------------------------------------------------------------------------------------------------ rotary positions
def rope_bound(x, amplitude):
    """Angles are good to 2^-22, sine and cosine to 2^-22 on top, the factor and two products and a sum round 2^-24 each, and
    the result to fp16 (2^-11, 2^-25 where it is subnormal)."""
    x = np.abs(np.asarray(x).astype(np.float64)).max(axis=-1, keepdims=True) * amplitude
    return 2 * x * (2 * 2.0 ** -22 + 4 * 2.0 ** -24) + 2 * x * 2.0 ** -11 + 2.0 ** -25


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,H_kv,d,r,scaling", [(12, 12, 64, 64, "none"), (32, 8, 128, 128, "ramp"), (4, 2, 64, 32, "linear"), (5, 1, 48, 20, "base"), (3, 3, 16, 2, "none"),
                                                (6, 3, 128, 24, "bands"), (2, 2, 256, 256, "none"), (1, 1, 8, 8, "none"), (2, 1, 512, 512, "none"), (2, 2, 320, 36, "none"), (1, 1, 16, 14, "none"), (2, 1, 48, 48, "none"), (4, 2, 24, 16, "none"),
                                                (6, 2, 112, 96, "linear")])
@pytest.mark.parametrize("T", [1, 3, 70])
def test_rope(H, H_kv, d, r, scaling, interleaved, T):
    rng = np.random.default_rng(T + d)
    kw = dict(none={}, linear=dict(factor=4.0), base=dict(factor=8.0), bands=dict(factor=8.0, original_len=8192, low=1.0, high=4.0),
              ramp=dict(factor=16.0, original_len=4096))[scaling]
    tb = RopeTable(r, 10000.0, scaling, **kw)
    x = torch.from_numpy(rng.standard_normal((T, H + 2 * H_kv, d)).astype(np.float16)).cuda()
    q, k = x[:, :H], x[:, H:H + H_kv]
    pos = rng.integers(-5, 1 << 20, T)
    pos[0] = 2 ** 31 - 1
    lk = Lookat(H, H_kv, d, d, 1 if d <= 128 else 4, 16)
    q0, k0 = q.cpu().numpy(), k.cpu().numpy()
    got_q, got_k = lk.lookat_rope(q, k, i32(pos), tb, interleaved=interleaved)
    assert finding(lk) == "" and np.array_equal(q.cpu().numpy(), q0), "inputs change"
    for got, y in ((got_q, q0), (got_k, k0)):
        want = serve.rope(y, pos, tb.host, tb.amplitude, interleaved)
        err = np.abs(got.double().cpu().numpy() - want)
        assert (err <= rope_bound(y, tb.amplitude)).all(), float((err / rope_bound(y, tb.amplitude)).max())
        assert np.array_equal(got[..., r:].cpu().numpy(), y[..., r:])
    # in place, within the wider rows; [heads][tokens][d] as well; each alone
    heads_first = torch.empty((H, T, d), dtype=torch.float16, device="cuda").transpose(0, 1)
    assert lk.lookat_rope(q, None, i32(pos), tb, interleaved=interleaved, q_out=heads_first)[1] is None
    rest = x[:, H + H_kv:].clone()
    lk.lookat_rope(q, k, i32(pos), tb, interleaved=interleaved, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert torch.equal(q, got_q) and torch.equal(k, got_k) and torch.equal(heads_first, got_q) and torch.equal(rest, x[:, H + H_kv:])


def test_rope_of_many_tokens_is_that_of_few():
    """The heads that a thread takes depend on the number of tokens; the results do not."""
    lk, tb = Lookat(32, 8, 128, 128, 4, 16), RopeTable(128, 500000.0)
    x = torch.randn(9000, 40, 128, device="cuda").half()
    pos = torch.arange(9000, dtype=torch.int32, device="cuda")
    q, k = lk.lookat_rope(x[:, :32], x[:, 32:], pos, tb)
    for lo in (0, 4500, 8990):
        a, b = lk.lookat_rope(x[lo:lo + 10, :32], x[lo:lo + 10, 32:], pos[lo:lo + 10], tb)
        torch.cuda.synchronize()
        assert torch.equal(a, q[lo:lo + 10]) and torch.equal(b, k[lo:lo + 10])
    e, _ = lk.lookat_rope(x[:0, :32], None, pos[:0], tb)
    assert e.shape == (0, 32, 128)


def test_rope_from_two_threads_on_one_context():
    """Each call has its own rows, whatever another thread calls meanwhile."""
    lk, tb = Lookat(4, 2, 64, 64, 1, 16), RopeTable(64)
    pos = torch.arange(16, dtype=torch.int32, device="cuda")
    x = torch.randn(2, 16, 4, 64, device="cuda").half()
    want = [lk.lookat_rope(x[i], None, pos, tb)[0] for i in range(2)]
    out = torch.zeros(2, 400, 16, 4, 64, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()

    def run(i):
        for j in range(400):
            lk.lookat_rope(x[i], None, pos, tb, q_out=out[i, j])

    threads, interval = [threading.Thread(target=run, args=(i,)) for i in range(2)], sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(interval)
    assert finding(lk) == ""
    for i in range(2):
        assert (out[i] == want[i]).all()


def test_rope_refuses():
    lk, tb = Lookat(4, 2, 64, 64, 1, 16), RopeTable(64)
    x = torch.zeros(3, 4, 64, dtype=torch.float16, device="cuda")
    pos = i32([0, 1, 2])
    with pytest.raises(LookatError, match="both NULL"):
        lk._check(lk._lib.lookat_rope(lk._h, None, None, 3, pos.data_ptr(), tb.turns.data_ptr(), 64, 0, 1.0, None, None))
    with pytest.raises(LookatError, match="rotary_dim"):
        lk.lookat_rope(x, None, pos, RopeTable(128))
    with pytest.raises(LookatError, match="token_stride"):
        lk.lookat_rope(torch.zeros(3 * 300, dtype=torch.float16, device="cuda").as_strided((3, 4, 64), (257, 64, 1)), None, pos, tb)
    with pytest.raises(LookatError, match="16-byte aligned"):
        lk.lookat_rope(torch.zeros(3 * 256 + 8, dtype=torch.float16, device="cuda")[1:769].view(3, 4, 64), None, pos, tb)
    with pytest.raises(LookatError, match="neither within heads"):
        lk.lookat_rope(x, None, pos, tb, q_out=torch.zeros(600, dtype=torch.float16, device="cuda").as_strided((3, 4, 64), (128, 64, 1)))
    with pytest.raises(LookatError, match="amplitude"):
        tb.amplitude = math.nan
        lk.lookat_rope(x, None, pos, tb)
    for bad in (x.float(), x.cpu(), x[:, :3], x[..., ::2]):
        with pytest.raises((TypeError, ValueError)):
            lk.lookat_rope(bad, None, pos, RopeTable(64))


# ------------------------------------------------------------------------------------------------ attention of packed prompts
def attend_reference(q, k, v, starts, scale):
    """(out, sum of weight * |value|, largest sum |q k| scale) in fp64 on the GPU, one head of one row at a time."""
    T, H, _ = q.shape
    g = H // k.shape[1]
    out, mag, reach = (torch.zeros((T, H, v.shape[2]), dtype=torch.float64, device="cuda") for _ in range(3))
    for lo, hi in zip(starts[:-1], starts[1:]):
        for h in range(H if hi > lo else 0):
            a, b, c = q[lo:hi, h].double(), k[lo:hi, h // g].double(), v[lo:hi, h // g].double()
            later = torch.ones((hi - lo, hi - lo), dtype=torch.bool, device="cuda").triu_(1)
            w = torch.softmax((a @ b.T * scale).masked_fill(later, -math.inf), dim=1)
            out[lo:hi, h], mag[lo:hi, h] = w @ c, w @ c.abs()
            reach[lo:hi, h] = (a.abs() @ b.abs().T * scale).masked_fill(later, 0).amax(dim=1, keepdim=True)
    return out, mag, reach


def attend_bound(out, mag, reach, d_k, L, vmax):
    """Per element.  Scores: sums of d_k exact products in fp32, each addition off by at most 2^-23 of sum |q k| <= reach, and a
    few roundings of the scaled score and its difference to the maximum; an error e of the scores changes weights and their
    sum by e each; the exponential is good to 2^-20.  Sums over L tokens: 2^-23 of mag per addition, in the weighted sum and
    in the denominator.  The weights are rounded to fp16: 2^-11 of themselves, 2^-25 where they are subnormal, against a
    largest one of 2^7 or more.  The result is rounded: 2^-11, or 2^-25 where it is subnormal."""
    rel = 2 * reach * (d_k + 8) * 2.0 ** -23 + 2.0 ** -19 + 2 * L * 2.0 ** -23 + 2.0 ** -11
    return mag * rel + out.abs() * 2.0 ** -11 + 2.0 ** -25 + L * 2.0 ** -32 * vmax


def packed_inputs(rng, lens, H, H_kv, d_k, d_v, layout="fused", peak=1.0, first=3, behind=4):
    """Random queries, keys and values, with NaN and infinities in the tokens that no row holds."""
    T = first + sum(lens) + behind
    parts = [(rng.standard_normal((T, h, d)) * s).astype(np.float16) for h, d, s in ((H, d_k, peak), (H_kv, d_k, 1.0), (H_kv, d_v, 1.0))]
    for x in parts:
        x[:first], x[T - behind:] = np.inf, np.nan
    t = [torch.from_numpy(x).cuda() for x in parts]
    if layout == "fused" and d_k == d_v:
        t = list(torch.cat(t, dim=1).split([H, H_kv, H_kv], dim=1))
    elif layout == "heads":
        t = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in t]
    return t, starts_of(lens, first)


def check_attend(rng, lens, H, H_kv, d_k, d_v, layout="fused", peak=1.0, scale=0.0, inputs=None):
    (q, k, v), starts = packed_inputs(rng, lens, H, H_kv, d_k, d_v, layout, peak) if inputs is None else inputs
    lk = Lookat(H, H_kv, d_k, d_v, 1 if d_k <= 128 else 2, 16, scale=scale)
    T = q.shape[0]
    out = torch.full((T, H, d_v), 7.0, dtype=torch.float16, device="cuda")
    if layout == "heads":
        out = out.transpose(0, 1).contiguous().transpose(0, 1)
    lk.lookat_attend_packed(q, k, v, i32(starts), out=out)
    again = lk.lookat_attend_packed(q, k, v, i32(starts))
    assert finding(lk) == ""
    a, b = int(starts[0]), int(starts[-1])
    assert torch.equal(out[a:b], again[a:b]), "two calls on the same inputs differ"
    assert (out[:a] == 7).all() and (out[b:] == 7).all(), "tokens of no row are written"
    want, mag, reach = attend_reference(q, k, v, starts, lk.scale)
    bound = attend_bound(want, mag, reach, d_k, max(lens), float(v[a:b].abs().max()) if b > a else 0.0)
    err = (out.double() - want).abs()[a:b]
    assert bool((err <= bound[a:b]).all()), f"off by up to {float((err / bound[a:b]).max()):.3g} of the bound"


RAGGED = [[1], [17, 0, 128, 129], [300, 1, 1, 64, 255, 256, 257, 0], [40, 1000, 3]]


@pytest.mark.parametrize("layout", ["fused", "heads", "dense"])
@pytest.mark.parametrize("H,H_kv,d_k,d_v", [(12, 12, 64, 64), (8, 2, 128, 128), (6, 2, 64, 128), (3, 1, 128, 64), (16, 1, 128, 128), (10, 2, 64, 64), (1, 1, 64, 64),
                                            (4, 2, 16, 16), (2, 1, 96, 80), (2, 2, 256, 256), (3, 3, 48, 144), (4, 4, 192, 64), (2, 1, 128, 240)])
@pytest.mark.parametrize("lens", RAGGED)
def test_attend_packed(lens, H, H_kv, d_k, d_v, layout):
    check_attend(np.random.default_rng(sum(lens) + d_k), lens, H, H_kv, d_k, d_v, layout)


@pytest.mark.parametrize("H,H_kv,d", [(3, 1, 64), (32, 8, 128), (2, 2, 32)])
def test_attend_packed_long_and_many_rows(H, H_kv, d):
    """Few rows and many, whose tiles are found in different ways; more tiles than a CTA lists; rows short enough for the other form,
    some of them among long ones."""
    rng = np.random.default_rng(d)
    check_attend(rng, [5000, 2, 700], H, H_kv, d, d)
    check_attend(rng, [int(n) for n in rng.integers(0, 9, 400)], H, H_kv, d, d)
    check_attend(rng, [int(n) for n in rng.integers(0, 200, 65)], H, H_kv, d, d)
    check_attend(rng, [0] * 70 + [900] + [1] * 30 + [400, 0], H, H_kv, d, d)


def test_attend_packed_more_items_than_a_cta_lists():
    rng = np.random.default_rng(1)
    (q, k, v), starts = packed_inputs(rng, [150] * 400, 64, 64, 64, 64, first=0, behind=0)      # 400 * 64 items on at most 148 SMs
    lk = Lookat(64, 64, 64, 64, 1, 16)
    out = lk.lookat_attend_packed(q, k, v, i32(starts))
    assert finding(lk) == ""
    for b in (0, 7, 199, 399):
        lo, hi = int(starts[b]), int(starts[b + 1])
        want, mag, reach = attend_reference(q[lo:hi], k[lo:hi], v[lo:hi], [0, 150], lk.scale)
        assert bool(((out[lo:hi].double() - want).abs() <= attend_bound(want, mag, reach, 64, 150, float(v.abs().max()))).all())


@pytest.mark.parametrize("layout", ["fused", "heads"])
@pytest.mark.parametrize("H,H_kv", [(64, 1), (128, 1), (32, 1), (96, 2), (256, 2)])
def test_attend_packed_large_groups(H, H_kv, layout):
    """Groups of 32 to 128 query heads: a tile is a few tokens, or one; a warp's lines are part of a token's."""
    check_attend(np.random.default_rng(H), [40, 1, 9], H, H_kv, 64, 64, layout)
    check_attend(np.random.default_rng(H), [70, 200], H, H_kv, 128, 128, layout)


def test_attend_packed_windows_and_an_output_among_other_things():
    """Keys whose vectors overlap each other (heads 8 elements apart), and results into the middle of wider rows."""
    T, H, d = 300, 4, 64
    buf = torch.randn(T * 128 + 64, device="cuda").half()
    k = buf.as_strided((T, H, d), (128, 8, 1))
    q, v = torch.randn(T, H, d, device="cuda").half(), torch.randn(T, H, d, device="cuda").half()
    wide = torch.full((T, 3 * H, d), 7.0, dtype=torch.float16, device="cuda")
    out = wide[:, H:2 * H]
    lk = Lookat(H, H, d, d, 1, 16)
    lk.lookat_attend_packed(q, k, v, i32([0, 120, T]), out=out)
    want = lk.lookat_attend_packed(q, k.contiguous(), v, i32([0, 120, T]))
    assert finding(lk) == "" and torch.equal(out, want)
    assert (wide[:, :H] == 7).all() and (wide[:, 2 * H:] == 7).all()


def test_attend_packed_of_the_plain_oracle():
    """A small case against the oracle that is written one query at a time."""
    (q, k, v), starts = packed_inputs(np.random.default_rng(2), [9, 0, 33], 4, 2, 64, 64)
    lk = Lookat(4, 2, 64, 64, 1, 16)
    out = lk.lookat_attend_packed(q, k, v, i32(starts))
    want, mag, reach = (torch.from_numpy(x) for x in serve.attend_packed(q.cpu().numpy(), k.cpu().numpy(), v.cpu().numpy(), starts, lk.scale))
    a, b = starts[0], starts[-1]
    assert bool(((out.cpu().double() - want).abs() <= attend_bound(want, mag, reach[..., None], 64, 33, 5.0))[a:b].all())


@pytest.mark.parametrize("d", [64, 128, 32])
def test_attend_packed_peaked_scores_that_rise_and_fall(d):
    """The running exponent moves at every block, or never after the first; a scale of the caller's."""
    rng = np.random.default_rng(d)
    check_attend(rng, [600, 130], 4, 2, d, d, peak=20.0)
    check_attend(rng, [300], 4, 2, d, d, peak=1e-3, scale=5.0)
    for sign in (1.0, -1.0):
        (q, k, v), starts = packed_inputs(rng, [700], 2, 1, d, d, "dense")
        ramp = torch.linspace(-1, 1, q.shape[0], device="cuda") * sign * 8
        q[:, :, 0], k[:, :, 0] = 6.0, ramp[:, None].half()      # scores climb (or fall) by a steady amount per token
        check_attend(rng, [700], 2, 1, d, d, "dense", inputs=((q, k, v), starts))


def test_attend_packed_keys_that_are_not_seen_may_be_anything():
    """A NaN or an infinity among a row's keys or values: other rows are as ever, and so are queries before the key."""
    for d in (64, 128, 32):
        (q, k, v), starts = packed_inputs(np.random.default_rng(d), [200, 150, 90], 4, 2, d, d)
        lk = Lookat(4, 2, d, d, 1, 16)
        clean = lk.lookat_attend_packed(q, k, v, i32(starts))
        v[starts[1] + 1, 1], v[starts[1] + 100, 0, 3], v[starts[1] + 149] = math.inf, math.nan, math.inf
        k[starts[2] + 60] = math.nan
        got = lk.lookat_attend_packed(q, k, v, i32(starts))
        torch.cuda.synchronize()
        lo, hi = int(starts[1]), int(starts[2])
        a = int(starts[0])
        assert torch.equal(got[a:lo], clean[a:lo]) and torch.equal(got[hi:hi + 60], clean[hi:hi + 60])
        assert torch.isnan(got[hi + 60:hi + 90]).all()


def test_attend_packed_rows_out_of_range_are_empty():
    for d in (64, 32):
        (q, k, v), _ = packed_inputs(np.random.default_rng(d), [300], 2, 1, d, d, first=0, behind=0)
        lk = Lookat(2, 1, d, d, 1, 16)
        good = [0, 100, 300]
        clean = lk.lookat_attend_packed(q, k, v, i32(good))
        for starts, rows in (([0, 100, 301], [(0, 100)]), ([-1, 100, 300], [(100, 300)]), ([0, 100, 90], [(0, 100)]), ([0, 100, -2 ** 31], [(0, 100)])):
            out, lk = torch.full_like(clean, 7.0), Lookat(2, 1, d, d, 1, 16)
            lk.lookat_attend_packed(q, k, v, i32(starts), out=out)
            assert "out of range or order" in finding(lk)
            held = torch.zeros(300, dtype=torch.bool, device="cuda")
            for a, b in rows:
                held[a:b] = True
                assert torch.equal(out[a:b], clean[a:b])
            assert (out[~held] == 7).all()


def test_attend_packed_offsets_beyond_32_bits():
    for d in (64, 32):
        T, ts = 150, 1 << 24
        buf = torch.empty(T * ts, dtype=torch.float16, device="cuda")
        at = lambda h, off: buf.as_strided((T, h, d), (ts, d, 1), off)  # noqa: E731
        q, k, v, out = at(4, 0), at(2, 1024), at(2, 2048), at(4, 4096)
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda"))
        lk = Lookat(4, 2, d, d, 1, 16)
        lk.lookat_attend_packed(q, k, v, i32([0, 140, T]), out=out)
        want = lk.lookat_attend_packed(q.contiguous(), k.contiguous(), v.contiguous(), i32([0, 140, T]))
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        tb = RopeTable(d)
        pos = torch.arange(T, dtype=torch.int32, device="cuda")
        want = lk.lookat_rope(q, k, pos, tb)
        lk.lookat_rope(q, k, pos, tb, q_out=out)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0])
        del buf, q, k, v, out


def test_attend_packed_refuses():
    lk = Lookat(4, 2, 64, 64, 1, 16)
    q, k = (torch.zeros(5, h, 64, dtype=torch.float16, device="cuda") for h in (4, 2))
    s = i32([0, 5])
    assert lk.lookat_attend_packed(q[:0], k[:0], k[:0], i32([0, 0])).shape == (0, 4, 64)
    with pytest.raises(LookatError, match="UNSUPPORTED"):
        a = Lookat(2, 2, 24, 24, 1, 16)
        x = torch.zeros(5, 2, 24, dtype=torch.float16, device="cuda")
        a.lookat_attend_packed(x, x, x, s)
    with pytest.raises(LookatError, match="B=0"):
        lk.lookat_attend_packed(q, k, k, s[:1])
    with pytest.raises(LookatError, match="neither within heads"):
        lk.lookat_attend_packed(q, k, k, s, out=torch.zeros(1000, dtype=torch.float16, device="cuda").as_strided((5, 4, 64), (64, 64, 1)))
    with pytest.raises(LookatError, match="head_stride"):
        lk.lookat_attend_packed(q, torch.zeros(1000, dtype=torch.float16, device="cuda").as_strided((5, 2, 64), (136, 68, 1)), k, s)
    for bad in (dict(q=q.float()), dict(k=k[:4]), dict(v=k.cpu()), dict(starts=s.long())):
        with pytest.raises((TypeError, ValueError)):
            lk.lookat_attend_packed(**{**dict(q=q, k=k, v=k, starts=s), **bad})


def test_attend_packed_captured_replayed_and_on_two_streams():
    rng = np.random.default_rng(1)
    (q, k, v), starts = packed_inputs(rng, [200, 90, 310], 8, 2, 128, 128, first=0, behind=0)
    st = i32(starts)
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    lks = [Lookat(8, 2, 128, 128, 1, 16, stream=s) for s in side]
    outs = [torch.zeros(600, 8, 128, dtype=torch.float16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for lk, out in zip(lks, outs):                              # on streams of their own, whatever the current one is
        lk.lookat_attend_packed(q, k, v, st, out=out)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side[0]):
        lks[0].lookat_attend_packed(q, k, v, st, out=outs[0])
    st.copy_(i32([0, 1, 450, 600]))                             # other rows of as many tokens
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    want = Lookat(8, 2, 128, 128, 1, 16).lookat_attend_packed(q, k, v, st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want)


# ------------------------------------------------------------------------------------------------ packed appends
def random_cache(rng, n_pages, H, P, d_k, d_v, fmt):
    raw = [rng.integers(0, 127, (n_pages, H, P, d)).astype(np.uint8) for d in (d_k, d_v)]
    amax = [np.abs(rng.standard_normal((n_pages, H))).astype(np.float16).astype(np.float32) for _ in range(2)]
    return raw[0], amax[0], raw[1], amax[1]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("H,d_k,d_v,fused", [(3, 64, 64, True), (2, 128, 128, True), (1, 16, 256, False), (2, 80, 48, False), (5, 112, 112, True)])
@pytest.mark.parametrize("new,before", [([1] * 9, [5, 0, 16, 127, 128, 3, 31, 64, 200]), ([40, 0, 300, 1, 17], [0, 9, 13, 0, 250]), ([700], [0])])
def test_append_packed_is_the_oracles_bit_for_bit(fmt, P, H, d_k, d_v, fused, new, before):
    rng = np.random.default_rng(P + d_k + len(new))
    first, T = 2, 2 + sum(new) + 3
    lens = [a + b for a, b in zip(new, before)]
    need = [-(-n // P) for n in lens]
    n_pages = sum(need) + 2
    perm, tables, at = rng.permutation(n_pages), np.full((len(new), max(need)), -1, np.int32), 0
    for b, m in enumerate(need):
        tables[b, :m] = perm[at:at + m]
        at += m
    k, ka, v, va = random_cache(rng, n_pages, H, P, d_k, d_v, fmt)
    x = [(rng.standard_normal((T, H, d)) * np.exp(rng.standard_normal((T, H, 1)))).astype(np.float16) for d in (d_k, d_v)]
    x[0][first, 0, :3] = [np.nan, np.inf, -np.inf]
    gx = [torch.from_numpy(y).cuda() for y in x]
    if fused:
        gx = list(torch.cat(gx, dim=1).split([H, H], dim=1))
    else:
        gx = [y.transpose(0, 1).contiguous().transpose(0, 1) for y in gx]
    cache = Q8Cache(torch.from_numpy(k).cuda().view(DTYPE[fmt]), torch.from_numpy(ka).cuda(), torch.from_numpy(v).cuda().view(DTYPE[fmt]), torch.from_numpy(va).cuda())
    lk = Lookat(H, H, d_k, d_v, 1 if d_k <= 128 else 2, 16)
    starts = starts_of(new, first)
    lk.lookat_q8_append_packed(cache, gx[0], gx[1], i32(starts), i32(tables), i32(lens))
    assert finding(lk) == ""
    for y, raw, amax in ((x[0], k, ka), (x[1], v, va)):
        for b, n in enumerate(new):
            if n:
                part = y[starts[b]:starts[b + 1]].transpose(1, 0, 2)[None]
                q8.append(raw, amax, part, tables[b:b + 1], lens[b:b + 1], [n], fmt)
    assert np.array_equal(cache.k.view(torch.uint8).cpu().numpy(), k) and np.array_equal(cache.v.view(torch.uint8).cpu().numpy(), v)
    assert np.array_equal(cache.k_amax.cpu().numpy(), ka) and np.array_equal(cache.v_amax.cpu().numpy(), va)


def test_append_packed_many_rows_is_the_padded_append():
    """300 rows of 0 to 30 tokens, packed and padded: the same cache."""
    rng = np.random.default_rng(3)
    B, H, d, P = 300, 2, 64, 16
    new = rng.integers(0, 31, B)
    n = int(new.max())
    pages = PageState.empty(B, 8, 4 * B, P)
    caches = [Q8Cache.empty(4 * B, H, P, d, d) for _ in range(2)]
    lk = Lookat(H, H, d, d, 1, 16)
    padded = torch.randn(2, B, H, n, d, device="cuda").half()
    counts = i32(new)
    lk.lookat_pages_extend(pages, counts, None)
    lk.lookat_q8_append(caches[0], padded[0].contiguous(), padded[1].contiguous(), pages.tables, pages.seq_lens, counts)
    there = torch.arange(n, device="cuda")[None] < counts[:, None]
    k, v = (padded[i].permute(0, 2, 1, 3)[there].contiguous() for i in (0, 1))
    lk.lookat_q8_append_packed(caches[1], k, v, i32(starts_of(new)), pages.tables, pages.seq_lens)
    assert finding(lk) == ""
    for a, b in zip(caches[0].pools(), caches[1].pools()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_append_packed_findings_and_refusals():
    lk = Lookat(2, 2, 64, 64, 1, 16)
    cache = Q8Cache.empty(6, 2, 16, 64, 64)
    x = torch.randn(40, 2, 64, device="cuda").half()
    tables, lens = i32([[0, 1], [2, 3]]), i32([20, 20])
    lk.lookat_q8_append_packed(cache, x, x, i32([0, 20, 40]), tables, lens)
    assert finding(lk) == ""
    clean = [t.clone() for t in cache.pools()]
    for starts, row in (([0, 20, 41], 0), ([0, 20, 5], 0), ([-1, 20, 40], 1), ([0, 20, 2 ** 31 - 1], 0)):
        for t in cache.pools():
            t.zero_()
        lk = Lookat(2, 2, 64, 64, 1, 16)                        # (an error is reported until there is another)
        lk.lookat_q8_append_packed(cache, x, x, i32(starts), tables, lens)
        assert "out of range or order" in finding(lk)
        pages = [0, 1] if row == 0 else [2, 3]
        for got, want in zip(cache.pools(), clean):
            other = [p for p in range(6) if p not in pages]
            assert torch.equal(got[pages], want[pages]) and not got[other].float().any()
    lk.lookat_q8_append_packed(cache, x, x, i32([0, 20, 40]), i32([[0, 1], [2, 6]]), lens)
    assert "8-bit cache" in finding(lk)
    lk = Lookat(2, 2, 64, 64, 1, 16)
    lk.lookat_q8_append_packed(cache, x, x, i32([0, 20, 40]), tables, i32([20, 10]))       # more tokens than the row has
    assert "8-bit cache" in finding(lk)
    lk = Lookat(2, 2, 64, 64, 1, 16)
    lk.lookat_q8_append_packed(cache, x[:0], x[:0], i32([0, 0, 0]), tables, lens)
    assert finding(lk) == ""
    with pytest.raises(LookatError, match="token_stride"):
        lk.lookat_q8_append_packed(cache, torch.zeros(9000, dtype=torch.float16, device="cuda").as_strided((40, 2, 64), (132, 64, 1)), x, i32([0, 20, 40]), tables, lens)
    with pytest.raises(ValueError):
        lk.lookat_q8_append_packed(cache, x, x[:30], i32([0, 20, 40]), tables, lens)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
def test_append_packed_finds_bad_starts_behind_tokens_of_no_row(d, page):
    """Tokens of more than a page before the first row: nothing is appended for the first places."""
    cache = Q8Cache.empty(6, 2, page, d, d)
    x = torch.randn(page + 40, 2, d, device="cuda").half()
    tables, lens = i32([[0, 1], [2, 3]]), i32([20, 20])
    for starts, message in (([page, page + 20, page + 40], ""), ([page, page + 20, page + 41], "out of range or order"),
                            ([page + 20, page + 40, page], "out of range or order")):
        lk = Lookat(2, 2, d, d, 1, 16)
        lk.lookat_q8_append_packed(cache, x, x, i32(starts), tables, lens)
        found = finding(lk)
        assert message in found and bool(found) == bool(message)


# ------------------------------------------------------------------------------------------------ beam selection
GAP = 2e-5          # ranks closer than this are not asked to be told apart: fp32 exponentials and the differences in them, 2^-20 each at most


def beam_case(rng, G, W, V, L, done=0.15, first=False, masked=0.1, spread=2.5):
    logits = (rng.standard_normal((G * W, V)) * spread).astype(np.float32)
    logits[rng.random((G * W, V)) < masked] = -np.inf
    scores = (-5 * rng.random((G, W))).astype(np.float32)
    lengths = rng.integers(0, max(L, 1), (G, W)).astype(np.int32)
    finished = (rng.random((G, W)) < done).astype(np.int32)
    if first:
        scores[:, 0], scores[:, 1:] = 0, -np.inf
        lengths[:], finished[:] = 0, 0
    tokens = rng.integers(0, V, (G, W, L)).astype(np.int32) if L else None
    return scores, lengths, finished, tokens, logits


def check_beams(case, eos, penalty, logits_on_gpu=None, lk=None):
    scores, lengths, finished, tokens, logits = case
    want = serve.beam_select(scores, lengths, finished, tokens, logits, eos, penalty)
    assert want[6] > GAP, "the case does not tell its ranks apart"
    g = lambda x: None if x is None else torch.from_numpy(x).cuda()  # noqa: E731
    st = BeamState(g(scores), g(lengths), g(finished), g(tokens))
    x = torch.from_numpy(logits).cuda() if logits_on_gpu is None else logits_on_gpu
    lk = lk or Lookat(2, 2, 64, 64, 1, 16)
    ids, parents = lk.lookat_beam_select(st, x, eos=eos, length_penalty=penalty)
    torch.cuda.synchronize()
    assert parents.tolist() == want[5].tolist() and ids.tolist() == want[4].tolist()
    assert st.lengths.tolist() == want[1].tolist() and st.finished.tolist() == want[2].tolist()
    got, ref = st.scores.double().cpu().numpy(), want[0]
    assert np.array_equal(np.isfinite(got), np.isfinite(ref))
    live = np.isfinite(ref)
    # rounded once; sums of exponentials that are good to 2^-20
    assert (np.abs(got - ref)[live] <= np.abs(ref[live]) * 2.0 ** -24 + 2.0 ** -20).all()
    if tokens is not None:
        assert np.array_equal(st.tokens.cpu().numpy(), want[3])
    return st


@pytest.mark.parametrize("G,W,V,L", [(1, 1, 1, 4), (1, 1, 5000, 0), (3, 2, 50, 7), (8, 4, 50257, 33), (2, 32, 3000, 1), (5, 5, 4097, 300), (2, 16, 40001, 20), (1, 32, 20, 9),
                                     (40, 3, 1000, 16)])
@pytest.mark.parametrize("penalty,first,eos", [(0.0, False, 0), (0.7, False, -1), (1.0, True, 3)])
def test_beam_select(G, W, V, L, penalty, first, eos):
    if eos >= V:
        eos = V - 1
    rng = np.random.default_rng(G * 1000 + W + V)
    for _ in range(20):                                         # (on the CPU: a case whose ranks can be told apart)
        case = beam_case(rng, G, W, V, L, first=first)
        if serve.beam_select(*case, eos, penalty)[6] > GAP:
            break
    check_beams(case, eos, penalty)


@pytest.mark.parametrize("penalty,first,eos", [(0.0, False, 0), (0.7, False, -1), (1.0, True, 3)])
def test_beam_select_many_parts(penalty, first, eos):
    """More parts in a group than a CTA has threads."""
    rng = np.random.default_rng(5)
    for _ in range(20):                                         # (on the CPU: a case whose ranks can be told apart)
        case = beam_case(rng, 1, 32, 90001, 3, first=first)
        if serve.beam_select(*case, eos, penalty)[6] > GAP:
            break
    check_beams(case, eos, penalty)


def test_beam_select_many_parts_of_equal_logits():
    """Where every part's first is as good as any other, the lowest tokens of the first beam; and masked ones after the rest."""
    V = 90001
    for value in (0.0, -1e4, float(torch.finfo(torch.float32).min)):
        st = BeamState(torch.zeros(1, 32, device="cuda"), i32([[2] * 32]), i32([[0] * 32]))
        lk = Lookat(2, 2, 64, 64, 1, 16)
        ids, parents = lk.lookat_beam_select(st, torch.full((32, V), value, device="cuda"), length_penalty=0.5)
        assert finding(lk) == "" and ids.tolist() == list(range(32)) and parents.tolist() == [0] * 32
    scores, lengths, finished, tokens, logits = beam_case(np.random.default_rng(6), 1, 32, V, 3, done=0.0)
    logits[:] = np.finfo(np.float32).min
    logits[4, [9, 50000, 90000]], logits[30, [1, 60000]] = [2.0, 1.0, 0.5], [0.25, -1.0]
    check_beams((scores, lengths, finished, tokens, logits), 0, 0.0)


def test_beam_select_rows_at_any_alignment():
    """Rows of an odd vocabulary, dense and inside a wider buffer, at every alignment of 4 bytes."""
    rng = np.random.default_rng(5)
    G, W, V = 2, 3, 9001
    case = beam_case(rng, G, W, V, 5)
    states = []
    for off, stride in ((0, V), (1, V), (2, V + 2), (3, V + 7), (0, V + 3), (4, 9004)):
        buf = torch.full((G * W * stride + 8,), math.inf, device="cuda")      # what lies between the rows is not read
        view = buf[off:off + G * W * stride].as_strided((G * W, V), (stride, 1), off)
        view.copy_(torch.from_numpy(case[4]))
        st = check_beams(case, 7, 0.3, logits_on_gpu=view)
        states.append(st.scores)
    assert all(torch.allclose(s, states[0], rtol=0, atol=2e-6) for s in states)


def test_beam_select_equal_ranks_go_to_the_lowest_index():
    lk = Lookat(2, 2, 64, 64, 1, 16)
    for V in (7, 4096, 9001, 30011):
        logits = torch.zeros(6, V, device="cuda")
        st = BeamState(torch.zeros(2, 3, device="cuda"), i32([[4, 4, 4]] * 2), i32([[0, 0, 0]] * 2))
        ids, parents = lk.lookat_beam_select(st, logits, length_penalty=0.5)
        torch.cuda.synchronize()
        assert ids.tolist() == [0, 1, 2] * 2 and parents.tolist() == [0] * 3 + [3] * 3
        # the same logits and scores in every beam: equal ranks across beams, whatever the rows' alignment
        x = torch.randperm(V, device="cuda").float() * (8.0 / V)
        best = int(x.argmax())
        st = BeamState(torch.zeros(2, 3, device="cuda"), i32([[4, 4, 4]] * 2), i32([[0, 0, 0]] * 2))
        ids, parents = lk.lookat_beam_select(st, x.expand(6, V).contiguous())
        torch.cuda.synchronize()
        assert ids.tolist() == [best] * 6 and parents.tolist() == list(range(6))
        x[V // 2], x[V // 3] = 100.0, 100.0
        st = BeamState.empty(2, 3, 4)
        ids, parents = lk.lookat_beam_select(st, x.expand(6, V).contiguous())
        torch.cuda.synchronize()
        assert ids.view(2, 3)[:, :2].tolist() == [[V // 3, V // 2]] * 2 and parents.tolist() == [0] * 3 + [3] * 3


def test_beam_select_odd_rows():
    """Rows without a candidate, of one, with masks of the type's lowest value, with NaN and +inf; beams that do not count."""
    rng = np.random.default_rng(8)
    scores, lengths, finished, tokens, logits = beam_case(rng, 8, 3, 500, 6, done=0.0)
    low = np.finfo(np.float32).min
    logits[0:3] = -np.inf                                       # group 0: nothing at all
    logits[3] = -np.inf
    logits[3, 77] = -4.0                                        # group 1: one candidate in beam 0, none in the others
    logits[4:6] = -np.inf
    logits[6, :], logits[6, 9] = low, 1.0                       # group 2: masks of the lowest value
    logits[9, 400] = np.nan                                     # group 3: beams 0 and 1 have none
    logits[10, 3] = np.inf
    scores[4, 0], scores[4, 1] = np.nan, np.inf                 # group 4: only beam 2 counts
    finished[5] = 1                                             # group 5: all ended
    logits[18:21] = np.nan                                      # ended beams' logits do not matter
    scores[7] = -np.inf                                         # group 7: nothing counts
    finished[7, 1] = 1
    lengths[2, 1] = -5                                          # a length below zero is no place to write to
    check = (scores, lengths, finished, tokens, logits)
    with np.errstate(invalid="ignore", over="ignore"):
        check_beams(check, 4, 0.0)
        check_beams(check, 4, 2.0)


def test_beam_select_a_row_of_equal_lowest_values():
    """log of the row's size, not 0 or NaN."""
    low = np.finfo(np.float32).min
    st = BeamState(torch.zeros(1, 2, device="cuda"), i32([[0, 0]]), i32([[0, 0]]))
    x = torch.full((2, 64), low, device="cuda")
    Lookat(2, 2, 64, 64, 1, 16).lookat_beam_select(st, x)
    torch.cuda.synchronize()
    assert torch.allclose(st.scores.cpu(), torch.full((1, 2), -math.log(64)), rtol=1e-6, atol=0)


def test_beam_select_full_histories_and_large_values():
    rng = np.random.default_rng(9)
    scores, lengths, finished, tokens, logits = beam_case(rng, 3, 4, 200, 5, done=0.0, masked=0.0)
    lengths[:] = 5                                              # no room: the histories follow, the token is not written
    check_beams((scores, lengths, finished, tokens, logits), 0, 0.0)
    check_beams((scores, lengths, finished, tokens, logits * 1e4), 0, 0.0)
    check_beams((scores - 1e6, lengths, finished, tokens, logits), 0, 0.0)


def test_beam_select_captured_and_replayed():
    lk = Lookat(2, 2, 64, 64, 1, 16, stream=(side := torch.cuda.Stream()))
    G, W, V, steps = 4, 3, 12000, 5
    rng = np.random.default_rng(10)
    logits = torch.zeros(G * W, V, device="cuda")
    ids, parents = i32([0] * G * W), i32([0] * G * W)
    st, warm = BeamState.empty(G, W, steps), BeamState.empty(G, W, steps)
    torch.cuda.synchronize()
    lk.lookat_beam_select(warm, logits, eos=5, next_ids=ids, parents=parents)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        lk.lookat_beam_select(st, logits, eos=5, next_ids=ids, parents=parents)
    for _ in range(steps):
        x = (rng.standard_normal((G * W, V)) * 3).astype(np.float32)
        x[:, 5] += 6
        host = [t.cpu().numpy() for t in (st.scores, st.lengths, st.finished, st.tokens)]
        want = serve.beam_select(*host, x, 5, 0.0)
        logits.copy_(torch.from_numpy(x))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert want[6] > GAP and ids.tolist() == want[4].tolist() and parents.tolist() == want[5].tolist()
        assert np.array_equal(st.tokens.cpu().numpy(), want[3]) and st.finished.tolist() == want[2].tolist()


def test_beam_select_refuses():
    lk = Lookat(2, 2, 64, 64, 1, 16)
    st = BeamState.empty(2, 3, 4)
    x = torch.zeros(6, 10, device="cuda")
    for kw, what in ((dict(eos=10), "eos"), (dict(eos=-2), "eos"), (dict(length_penalty=-1.0), "length_penalty"), (dict(length_penalty=math.inf), "length_penalty")):
        with pytest.raises(LookatError, match=what):
            lk.lookat_beam_select(st, x, **kw)
    with pytest.raises(LookatError, match="beams=33"):
        lk.lookat_beam_select(BeamState.empty(1, 33, 0), torch.zeros(33, 10, device="cuda"))
    with pytest.raises(LookatError, match="logits_stride"):
        lk.lookat_beam_select(st, torch.zeros(20, device="cuda").as_strided((6, 10), (2, 1)))
    for bad in (x.half(), x.cpu(), x[:5], torch.zeros(6, 20, device="cuda")[:, ::2]):
        with pytest.raises((TypeError, ValueError)):
            lk.lookat_beam_select(st, bad)
    with pytest.raises(ValueError):
        BeamState(torch.zeros(2, 3, device="cuda"), i32([[0, 0, 0]]), i32([[0, 0, 0]] * 2))
