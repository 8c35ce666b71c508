"""The oracle of include/lookat_serve.h against hand-made cases, the host-side rotary table against it, and the refusals that
need no device."""
import ctypes
import math

import numpy as np
import pytest

from oracle import serve
from paper_2601_10155_b200 import binding, build

SCALINGS = [("none", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)), ("bands", dict(factor=8.0, original_len=8192.0, low=1.0, high=4.0)),
            ("ramp", dict(factor=16.0, original_len=4096.0, low=1.0, high=32.0)), ("ramp", dict(factor=1.0, original_len=100.0, low=1.0, high=1.01))]


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def table(lib, r, base, scaling, factor=1.0, original_len=0.0, low=1.0, high=32.0):
    cfg = binding.lookat_rope_config(r, ("none", "linear", "base", "bands", "ramp").index(scaling), base, factor, original_len, low, high)
    turns, amplitude = (ctypes.c_uint64 * 512)(), ctypes.c_float()
    return lib.lookat_rope_table(ctypes.byref(cfg), turns, ctypes.byref(amplitude)), list(turns[:max(r, 0) // 2]), amplitude.value


@pytest.mark.parametrize("scaling,kw", SCALINGS)
@pytest.mark.parametrize("r,base", [(4, 10000.0), (20, 10000.0), (64, 10000.0), (128, 500000.0), (1024, 1.5)])
def test_rope_table(lib, r, base, scaling, kw):
    st, turns, amplitude = table(lib, r, base, scaling, **kw)
    want, amp = serve.rope_frequencies(r, base, scaling, **kw)
    assert st == 0 and abs(amplitude - amp) <= amp * 2.0 ** -24
    # the oracle's fp64 powers are good to a few 2^-52 of themselves (the exponent's rounding times ln f <= 14); the fractions
    # of 2^64 to half a unit
    for t, f in zip(turns, want):
        assert abs(t * 2.0 ** -64 * 2 * math.pi - f) <= f * 2.0 ** -46 + 2 * math.pi * 2.0 ** -64


def test_rope_table_refuses(lib):
    good = dict(r=64, base=10000.0, scaling="ramp", factor=2.0, original_len=4096.0)
    assert table(lib, **good)[0] == 0
    for bad in (dict(r=0), dict(r=7), dict(r=1026), dict(r=-2), dict(base=1.0), dict(base=math.inf), dict(base=math.nan), dict(factor=0.5), dict(factor=math.nan),
                dict(original_len=0.0), dict(low=0.0), dict(high=1.0), dict(high=math.inf), dict(scaling="base", r=2)):
        assert table(lib, **{**good, **bad})[0] == 1, bad
    cfg = binding.lookat_rope_config(64, 5, 10000.0, 1.0, 0.0, 1.0, 32.0)
    out, amp = (ctypes.c_uint64 * 32)(), ctypes.c_float()
    assert lib.lookat_rope_table(ctypes.byref(cfg), out, ctypes.byref(amp)) == 1
    assert lib.lookat_rope_table(None, out, ctypes.byref(amp)) == 1


def test_calls_without_a_context_are_refused(lib):
    r = binding.lookat_rows(None, 0, 0)
    assert lib.lookat_rope(None, r, r, 1, None, None, 2, 0, 1.0, None, None) == 1
    assert lib.lookat_attend_packed(None, r, r, r, 1, 1, None, r) == 1
    assert lib.lookat_q8_append_packed(None, None, r, r, 1, 1, None, None, 1, None) == 1
    assert lib.lookat_beam_select(None, None, None, 1, 1, -1, 0.0, None, None) == 1


def test_rope_oracle_keeps_lengths_and_relative_positions():
    rng = np.random.default_rng(0)
    f, _ = serve.rope_frequencies(16, 100.0)
    turns = [round(x / (2 * math.pi) * 2 ** 64) for x in f]
    q, k = rng.standard_normal((2, 1, 1, 24))
    for inter in (False, True):
        dots = [float((serve.rope(q, [p + 5], turns, 1.0, inter) * serve.rope(k, [p], turns, 1.0, inter)).sum()) for p in (0, 3, 10 ** 6, -70)]
        assert np.allclose(dots, dots[0], atol=1e-12)
        assert np.array_equal(serve.rope(q, [9], turns, 1.0, inter)[..., 16:], q[..., 16:])
    assert np.allclose(serve.rope(np.array([[[1.0, 0.0]]]), [1], [2 ** 62], 1.0, False), [[[0.0, 1.0]]])      # a quarter turn


def test_attend_oracle_by_hand():
    q, k = np.zeros((3, 2, 4)), np.zeros((3, 1, 4))
    v = np.array([1.0, 3.0, 10.0]).reshape(3, 1, 1)
    out, mag, _ = serve.attend_packed(q, k, v, [0, 2, 3], 0.5)
    assert out[:, :, 0].tolist() == [[1, 1], [2, 2], [10, 10]] and np.array_equal(out, mag)


def test_beam_oracle_by_hand():
    half = math.log(0.5)
    s = np.array([[0.0, -0.1]])
    logits = np.log(np.array([[0.5, 0.25, 0.25], [0.5, 0.25, 0.25]])).astype(np.float32)
    tokens = np.array([[[7, 0], [8, 0]]])
    got = serve.beam_select(s, np.array([[1, 1]]), np.array([[0, 0]]), tokens, logits, 0, 0.0)
    assert np.allclose(got[0], [[half, half - 0.1]]) and got[1].tolist() == [[2, 2]] and got[2].tolist() == [[1, 1]]
    assert got[3].tolist() == [[[7, 0], [8, 0]]] and got[4].tolist() == [0, 0] and got[5].tolist() == [0, 1]
    # an ended beam competes as it is; equal ranks go to the lower index
    got = serve.beam_select(s, np.array([[1, 1]]), np.array([[1, 1]]), tokens, logits, 0, 0.0)
    assert np.allclose(got[0], s) and got[1].tolist() == [[1, 1]] and got[5].tolist() == [0, 1]
    logits[:] = 0
    got = serve.beam_select(np.zeros((1, 2)), np.array([[1, 1]]), np.array([[0, 0]]), tokens, logits, -1, 1.0)
    assert got[4].tolist() == [0, 1] and got[5].tolist() == [0, 0] and got[3].tolist() == [[[7, 0], [7, 1]]]
    # no candidate: the place keeps its row
    got = serve.beam_select(np.array([[-math.inf, -math.inf]]), np.array([[1, 1]]), np.array([[0, 1]]), tokens, logits, 2, 0.0)
    assert got[0].tolist() == [[-math.inf] * 2] and got[5].tolist() == [0, 1] and got[4].tolist() == [2, 2] and got[2].tolist() == [[0, 1]]
