"""Calls of include/lookat_serve.h at the edges of what its header promises, each with the bound or the answer that it is held to."""
import math

import numpy as np
import pytest
import torch

from paper_2601_10155_b200.binding import Lookat
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
