"""Calls of include/lookat_serve.h at the edges of what its header promises, each with the bound or the answer that it is held to."""
import math

import numpy as np
import pytest
import torch

from paper_2601_10155_b200.binding import BeamState, Lookat, LookatError, PageState, Q8Cache, RopeTable
from test_gpu_serve import beam_case, check_beams, finding, i32, starts_of

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ attention of packed prompts
@pytest.mark.parametrize("H,H_kv,d", [(4, 2, 96), (2, 1, 32), (1, 1, 256)])
@pytest.mark.parametrize("lens", [[1, 2, 3, 5, 90, 0, 17], [70, 100]])
def test_attend_packed_of_values_with_a_common_offset(H, H_kv, d, lens):
    """Whatever changes a weight (its rounding to fp16, 2^-11 of itself; errors of its score; the exponential, 2^-20) acts on what
    a value differs from the result by, since the sum is over the same weights: sum w (v - out) is 0.  The additions, L of
    them, are off by 2^-23 of their sum each, in the result and in the denominator.  Values lie in 1..2, where half a step of
    fp16 is 2^-11."""
    rng = np.random.default_rng(d + len(lens))
    starts, T = starts_of(lens), sum(lens)
    q, k = (torch.from_numpy((rng.standard_normal((T, h, d)) * s).astype(np.float16)).cuda() for h, s in ((H, 1.0), (H_kv, 1.0)))
    v = torch.from_numpy((1.75 + rng.uniform(-1, 1, (T, H_kv, d)) * 2.0 ** -5).astype(np.float16)).cuda()
    lk = Lookat(H, H_kv, d, d, 1 if d <= 128 else 2, 16)
    out = lk.lookat_attend_packed(q, k, v, i32(starts))
    assert finding(lk) == ""
    for lo, hi in zip(starts[:-1], starts[1:]):
        for h in range(H if hi > lo else 0):
            a, b, c = q[lo:hi, h].double(), k[lo:hi, h // (H // H_kv)].double(), v[lo:hi, h // (H // H_kv)].double()
            later = torch.ones((hi - lo, hi - lo), dtype=torch.bool, device="cuda").triu_(1)
            w = torch.softmax((a @ b.T * lk.scale).masked_fill(later, -math.inf), dim=1)
            want = w @ c
            reach = (a.abs() @ b.abs().T * lk.scale).masked_fill(later, 0).amax(dim=1, keepdim=True)
            apart = torch.einsum("tu,tud->td", w, (c[None] - want[:, None]).abs())
            rel = 1.01 * (2.0 ** -11 + 2 * reach * (d + 8) * 2.0 ** -23 + 2.0 ** -19)
            bound = 2.0 ** -11 + rel * apart + (2 * (hi - lo) + 4) * 2.0 ** -23 * want
            err = (out[lo:hi, h].double() - want).abs()
            assert bool((err <= bound).all()), f"off by up to {float((err / bound).max()):.4g} of the bound"


@pytest.mark.parametrize("d", [64, 32])
def test_attend_packed_reports_a_time_out_once(d):
    """The self-test's kernel has one wait that nothing ends and gives up after 4096 polls.  Without another attention call the
    time-out is in lookat_last_error."""
    lk = Lookat(2, 1, d, d, 1, 16)
    q, k, v = (torch.randn(90, h, d, device="cuda").half() for h in (2, 1, 1))
    starts = i32([0, 40, 90])
    want = lk.lookat_attend_packed(q, k, v, starts)
    assert finding(lk) == ""
    lk._check(lk._lib.lookat_selftest_timeout(lk._h))
    for _ in range(2):
        assert "gave up" in finding(lk)
    with pytest.raises(LookatError, match="gave up") as err:
        lk.lookat_attend_packed(q, k, v, starts)
    assert err.value.status == 5
    got = lk.lookat_attend_packed(q, k, v, starts)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_time_out_hides_no_other_finding():
    lk = Lookat(2, 1, 64, 64, 1, 16)
    q, k = (torch.randn(90, h, 64, device="cuda").half() for h in (2, 1))
    with pytest.raises(LookatError, match="B=0"):
        lk._check(lk._lib.lookat_attend_packed(lk._h, None, None, None, 90, 0, None, None))
    lk.lookat_attend_packed(q, k, k, i32([0, 100]))
    lk._check(lk._lib.lookat_selftest_timeout(lk._h))
    assert "out of range or order" in finding(lk) and "gave up" in finding(lk)


# ------------------------------------------------------------------------------------------------ beam selection
@pytest.mark.parametrize("G,W", [(1, 32), (200, 3), (70, 8)])
def test_beam_select_logits_that_rise_along_the_row(G, W):
    """Every renewal of the bar that candidates have to reach moves it, in parts of one batch of 4096 logits and of many; a bar
    above a part's W-th largest logit would lose a candidate."""
    rng = np.random.default_rng(W)
    V = 9 * 4096 + 77
    scores, lengths, finished, tokens, logits = beam_case(rng, G, W, V, 2, done=0.0, first=True, masked=0.0)
    rise = np.linspace(-20, 20, V)                              # a neighbour is 1e-3 away
    logits[:] = rise.astype(np.float32)
    logits[0] = np.where(np.arange(V) % 7 == 0, -np.inf, rise)
    check_beams((scores, lengths, finished, tokens, logits), -1, 0.0)


def test_beam_select_the_largest_length_penalties():
    """Norms of up to 2^868: beams of one length are ranked as without a penalty and keep their scores; a longer beam goes before
    a shorter one.  Penalties beyond that are refused: their norms could overflow, and rank times norm is then no score."""
    rng = np.random.default_rng(4)
    lk = Lookat(2, 2, 64, 64, 1, 16)
    x = torch.from_numpy(rng.standard_normal((6, 500)).astype(np.float32)).cuda()
    scores = torch.from_numpy((-1e-3 * rng.random((2, 3))).astype(np.float32)).cuda()
    for length in (0, 200, 2 ** 31 - 3):
        got = []
        for penalty in (0.0, 28.0):
            st = BeamState(scores.clone(), i32([[length] * 3] * 2), i32([[0, 0, 0]] * 2))
            ids, parents = lk.lookat_beam_select(st, x, length_penalty=penalty)
            assert finding(lk) == ""
            got.append((ids.tolist(), parents.tolist()))
            if penalty:                                         # rank times norm: one more rounding in fp64
                assert bool(((st.scores - plain).abs() <= plain.abs() * 2.0 ** -23).all())
            plain = st.scores
        assert got[0] == got[1]
    st = BeamState(torch.zeros(2, 3, device="cuda"), i32([[9, 199, 10]] * 2), i32([[0, 0, 0]] * 2))
    ids, parents = lk.lookat_beam_select(st, x, length_penalty=28.0)
    assert finding(lk) == "" and parents.tolist() == [1] * 3 + [4] * 3
    want = torch.log_softmax(x[1::3].double(), dim=1).topk(3)
    assert ids.tolist() == want.indices.reshape(-1).tolist()
    assert bool(((st.scores.double() - want.values).abs() <= want.values.abs() * 2.0 ** -24 + 2.0 ** -20).all())
    for penalty in (28.5, 150.0, 1e308, math.nan):
        with pytest.raises(LookatError, match="length_penalty"):
            lk.lookat_beam_select(st, x, length_penalty=penalty)


@pytest.mark.parametrize("kind", ["late", "flat", "spread", "large", "masked", "far", "rising far"])
def test_beam_select_sums_of_exponentials(kind):
    """Rows of five batches of logits in one part.  A term at distance d of the reference (at most 1 from the largest) is off by
    2^-22 (the exponential), 5 * 2^-24 (sixteen terms are added in fp32), 2^-24 d (the exponent's rounding) and 2^-26 d (log2(e)
    as an fp32 number) of itself; the rest is fp64, and the score is rounded once.
    late: one logit that holds all the weight, 8 to 17 above what stands in front of it.  flat: one logit, and all others 10 below,
    which weigh as much together.  masked: the first batches hold the type's lowest value.  far: logits above 2^20, or that get there."""
    rng = np.random.default_rng(7)
    G, W, V = 150, 4, 20000
    x = (rng.standard_normal((G * W, V)) * 2.5).astype(np.float32)
    if kind == "late":
        x[np.arange(G * W), rng.integers(4096, V, G * W)] = x[:, :4096].max(axis=1) + rng.uniform(8, 17, G * W).astype(np.float32)
    if kind == "flat":
        base = rng.uniform(-3, 3, G * W).astype(np.float32)
        x[:] = base[:, None]
        x[np.arange(G * W), rng.integers(0, V, G * W)] = base + np.float32(10)
    if kind == "large":
        x = (x + rng.uniform(-1e4, 1e4, (G * W, 1))).astype(np.float32)
    if kind == "masked":
        x[:, :9000] = np.finfo(np.float32).min
    if kind == "far":
        x = (x * 4 + rng.uniform(2e6, 3e6, (G * W, 1))).astype(np.float32)
    if kind == "rising far":
        x[:, 12000:] = (x[:, 12000:] * 4 + np.float32(2e6)).astype(np.float32)
        x[: G * W // 2, 17000] = np.float32(3e38)
    st = BeamState.empty(G, W, 0)
    ids, parents = Lookat(2, 2, 64, 64, 1, 16).lookat_beam_select(st, torch.from_numpy(x).cuda())
    torch.cuda.synchronize()
    assert parents.tolist() == [g * W for g in range(G) for _ in range(W)]
    got, ids = st.scores[:, 0].double().cpu().numpy(), ids.view(G, W)[:, 0].cpu().numpy()
    y = x[::W].astype(np.float64)
    d = y.max(axis=1, keepdims=True) - y
    p = np.exp(-d)
    total = p.sum(axis=1)
    want = -np.log(total)
    assert np.array_equal(ids, y.argmax(axis=1))
    bound = (10 + 1.25 * ((p * (d + 1)).sum(axis=1) / total)) * 2.0 ** -24 + np.abs(want) * 2.0 ** -24
    assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) / bound).max()


# ------------------------------------------------------------------------------------------------ results on other streams
def test_results_do_not_lie_in_memory_that_the_callers_stream_still_writes():
    """A context on a stream of its own; the caller's stream has freed blocks of just the results' sizes, which work that waits
    there is still to write."""
    side = torch.cuda.Stream()
    T, H, d = 64, 4, 64
    lk, tb = Lookat(H, H, d, d, 1, 16, stream=side), RopeTable(d)
    q, k, v = (torch.randn(T, H, d, device="cuda").half() for _ in range(3))
    pos, starts, logits = torch.arange(T, dtype=torch.int32, device="cuda"), i32([0, 20, T]), torch.randn(6, 50, device="cuda")
    beams = [BeamState.empty(2, 3, 0) for _ in range(2)]
    pages, cache = PageState.empty(2, 4, 8, 16), Q8Cache.empty(8, H, 16, d, d)
    torch.cuda.synchronize()
    lk.lookat_pages_extend(pages, i32([20, T - 20]), cache.pools())
    lk.lookat_q8_append_packed(cache, k, v, starts, pages.tables, pages.seq_lens)
    calls = [lambda: lk.lookat_rope(q, k, pos, tb), lambda: [lk.lookat_attend_packed(q, k, v, starts)],
             lambda: [lk.lookat_attend_q8(cache, q[:2], pages.tables, pages.seq_lens)]]
    selects = [lambda st=st: lk.lookat_beam_select(st, logits) for st in beams]
    for first, again in [(c, c) for c in calls] + [tuple(selects)]:
        want = first()
        torch.cuda.synchronize()
        blocks = [torch.empty_like(x) for x in want for _ in range(8)]
        torch.cuda.synchronize()
        torch.cuda._sleep(40_000_000)                           # tens of milliseconds
        for b in blocks:
            b.fill_(77)
        del b, blocks
        got = again()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
