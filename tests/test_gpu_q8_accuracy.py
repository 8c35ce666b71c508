"""Accuracy of attention over the 8-bit paged cache where the weights of a row are of very different sizes: blocks of
zeros, a token that takes most of the weight, values at the end of fp16's range.  fp32 results are held to
oracle.q8.attend_rms_tolerance."""
import numpy as np
import pytest
import torch

from oracle import q8
from paper_2601_10155_b200.binding import Lookat, Q8Cache

pytestmark = pytest.mark.gpu

DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def quantise(x, P, fmt):
    """[n][H][d] as pages [n_pages][H][P][d] in order, and their amax; zeros behind the last token."""
    n, H, d = x.shape
    n_pages = -(-n // P)
    padded = np.zeros((n_pages * P, H, d))
    padded[:n] = x
    pages = padded.reshape(n_pages, P, H, d).transpose(0, 2, 1, 3)
    amax = np.abs(pages).max(axis=(2, 3)).astype(np.float16).astype(np.float32)
    a = np.where(amax > 0, amax, 1.0)[:, :, None, None]
    return q8.bytes_of(np.clip(q8.R[fmt] * pages / a, -q8.R[fmt], q8.R[fmt]), fmt), amax


def attend(rows, q, P, fmt, width=0, fp16=False):
    """rows: (k, v) of each row, [n][H][d].  (got, out, reach, the caches' parts and tables)"""
    parts, tables, at = [], [], 0
    for k, v in rows:
        parts.append(quantise(k, P, fmt) + quantise(v, P, fmt))
        tables.append(np.arange(at, at + parts[-1][0].shape[0]))
        at += parts[-1][0].shape[0]
    W = max(width, *(len(t) for t in tables))
    tables = np.array([np.concatenate([t, np.full(W - len(t), -1)]) for t in tables], np.int32)
    k, ka, v, va = (np.concatenate(x) for x in zip(*parts))
    lens = [len(r[0]) for r in rows]
    B, Hq, Lq, d = q.shape
    lk = Lookat(Hq, k.shape[1], d, v.shape[3], 1, 16)
    cache = Q8Cache(dev(k).view(DTYPE[fmt]), dev(ka), dev(v).view(DTYPE[fmt]), dev(va))
    got = lk.lookat_attend_q8(cache, dev(q), dev(tables), dev(np.array(lens, np.int32)), out_fp16=fp16)
    torch.cuda.synchronize()
    assert lk.lookat_last_error() == ""
    need = max(-(-n // P) for n in lens)
    out, _, reach = q8.attend(k, ka, v, va, q, tables[:, :need], lens, fmt, lk.scale)
    return got.double().cpu().numpy(), out, reach


def off(got, out):
    return float(np.linalg.norm(got - out) / np.linalg.norm(out))


def check(rows, q, P, fmt):
    got, out, reach = attend(rows, q, P, fmt)
    tol = q8.attend_rms_tolerance(reach, q.shape[3], max(len(r[0]) for r in rows))
    assert tol < 1e-4                                           # weights of 11 bits are 1e-4 and more off
    assert off(got, out) <= tol, f"off by {off(got, out):.2e}, allowed {tol:.2e}"


def a_row(rng, n, H, d):
    return rng.standard_normal((n, H, d)), rng.standard_normal((n, H, d))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4, 1e-5])
@pytest.mark.parametrize("Hq,H,Lq", [(2, 1, 1), (8, 1, 1), (4, 2, 5), (4, 2, 40)])
def test_blocks_of_zero_values_do_not_cost_the_others_their_bits(fmt, size, Hq, H, Lq):
    """V is zero in a page of tokens that weigh as much as the rest: small values elsewhere keep their accuracy."""
    rng = np.random.default_rng(41)
    k, v = a_row(rng, 300, H, 64)
    v *= size
    v[32:48] = 0
    v[-12:] = 0
    q = rng.standard_normal((1, Hq, Lq, 64)).astype(np.float16)
    check([(k, v)], q, 16, fmt)


@pytest.mark.parametrize("Lq", [1, 40])
def test_a_block_of_zero_values_that_takes_the_weight(Lq):
    """The tokens of the zero page outweigh the rest by 12 nats; and a row whose values are all zero gives zeros."""
    rng = np.random.default_rng(42)
    k, v = a_row(rng, 200, 1, 64)
    k[:, :, 0] = 0
    k[:16, :, 0] = 26.0
    v[:16] = 0
    v[16:] *= 1e-3
    q = rng.standard_normal((2, 2, Lq, 64)).astype(np.float16)
    q[..., 0] = 4.0
    check([(k, v), (k[:90], 0 * v[:90])], q, 16, "int8")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("small", [0.01, 0.0])
@pytest.mark.parametrize("n,Hq,H,Lq", [(4096, 2, 1, 1), (4096, 8, 1, 1), (4096, 8, 1, 2), (4096, 2, 1, 40), (32768, 4, 1, 1), (32768, 2, 1, 20)])
def test_a_token_that_takes_most_of_the_weight(fmt, small, n, Hq, H, Lq):
    """A first token 12 nats above the rest whose own values are small: the result is made of the many small weights."""
    rng = np.random.default_rng(43)
    k, v = a_row(rng, n, H, 64)
    k[:, :, 0] = 0
    k[0, :, 0] = 24.0                                           # 24 * 4 / 8 = 12
    k[0, :, 1:] = 0
    v[0] *= small
    q = rng.standard_normal((1, Hq, Lq, 64)).astype(np.float16)
    q[..., 0] = 4.0
    check([(k, v)], q, 64, fmt)


@pytest.mark.parametrize("Lq", [1, 40])
def test_a_last_token_far_above_the_ones_before(Lq):
    """The running maximum moves by many powers of two at once, and step by step."""
    rng = np.random.default_rng(44)
    k, v = a_row(rng, 1500, 1, 64)
    k[:, 0, 0] = np.linspace(0, 20, 1500)                       # scores rise by 10 nats over the row
    k[1400, 0, 0] = 60.0
    q = rng.standard_normal((1, 2, Lq, 64)).astype(np.float16)
    q[..., 0] = 4.0
    got, out, reach = attend([(k, v)], q, 32, "e4m3")
    assert off(got, out) <= q8.attend_rms_tolerance(reach, 64, 1500)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,Lq,P,Hq,H,d", [([1000], 1, 64, 8, 2, 128), ([3000, 70], 70, 64, 4, 1, 128), ([2500], 300, 16, 2, 2, 64),
                                              ([9000, 4097, 63], 1, 64, 8, 2, 128), ([5000, 7], 3, 16, 4, 1, 64), ([2000], 1, 32, 16, 1, 128)])
def test_fp32_results_of_ordinary_rows(fmt, lens, Lq, P, Hq, H, d):
    rng = np.random.default_rng(45)
    q = (0.9 * rng.standard_normal((len(lens), Hq, Lq, d))).astype(np.float16)
    check([a_row(rng, n, H, d) for n in lens], q, P, fmt)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("n,width", [(200, 0), (700, 64)])
@pytest.mark.parametrize("Hq,Lq", [(1, 1), (4, 60)])
def test_fp16_results_of_the_largest_values_stay_finite(fmt, n, width, Hq, Lq):
    """Every value is the largest fp16 number, so every mean of them is.  All tokens but the first weigh the same, about
    half of the first: where that weight is rounded up, the sum is up to 2^-11 above its denominator."""
    rng = np.random.default_rng(46)
    sign = np.where(rng.random(64) < 0.5, -1.0, 1.0)
    k, v = np.zeros((n, 1, 64)), np.tile(65504.0 * sign, (n, 1, 1))
    k[0, :, 0] = 1.0
    q = np.zeros((1, Hq, Lq, 64), np.float16)
    q[..., 0] = rng.uniform(0.85, 1.15, (1, Hq, Lq)) * 8 * np.log(2)
    got, out, _ = attend([(k, v)], q, 16, fmt, width=width, fp16=True)
    assert np.isfinite(got).all()
    # a weight's rounding, then the result's
    assert (np.abs(got - 65504.0 * sign) <= 65504 * 2.0 ** -10).all()


def test_a_query_that_is_not_a_number_reaches_its_own_result_only():
    rng = np.random.default_rng(47)
    k, v = a_row(rng, 100, 1, 64)
    q = rng.standard_normal((1, 2, 40, 64)).astype(np.float16)
    clean, out, _ = attend([(k, v)], q, 16, "int8", fp16=True)
    q[0, 1, 7, 3] = np.nan
    got, _, _ = attend([(k, v)], q, 16, "int8", fp16=True)
    assert np.isnan(got[0, 1, 7]).all()
    got[0, 1, 7] = clean[0, 1, 7]
    assert np.array_equal(got, clean)
