"""Checks of the 8-bit cache's oracle against closed forms and torch's own e4m3 conversion (CPU)."""
import random

import numpy as np
import pytest
import torch

from oracle import q8


def test_e4m3_bytes_are_torchs():
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = every.view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    assert np.array_equal(q8.e4m3_values(), want, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 0.02, q8.e4m3_values()[:127],
                        (q8.e4m3_values()[:126] + q8.e4m3_values()[1:127]) / 2])     # the borders themselves
    got = q8.bytes_of(x, "e4m3")
    want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    same = got == want
    # fp32 holds the borders exactly; random fp64 values next to one may round to it first
    assert same[8000:].all() and (~same).sum() <= 2


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_token_by_token_stays_within_its_roundings(fmt):
    """Each growth of a block's amax rounds its earlier tokens once more: the error is at most half a step per rounding."""
    rng = np.random.default_rng(1)
    P, d, n = 16, 16, 40
    x = (rng.standard_normal((1, 2, n, d)) * np.exp(rng.standard_normal((1, 1, n, 1)))).astype(np.float16)
    tables = np.array([[3, 0, 2]], dtype=np.int32)
    raw, amax = np.full((4, 2, P, d), 0x55, np.uint8), np.full((4, 2), np.nan, np.float32)
    grown = np.zeros((2, n))
    for t in range(n):
        before = amax.copy()
        q8.append(raw, amax, x[:, :, t:t + 1], tables, [t + 1], [1], fmt)
        for h in range(2):
            p = tables[0, t // P]
            if t % P and amax[p, h] > before[p, h]:
                grown[h, t - t % P:t] += 1
    for t in range(n):
        for h in range(2):
            p = tables[0, t // P]
            a = float(amax[p, h])
            got = q8.values_of(raw[p, h, t % P], fmt) * a / q8.R[fmt]
            want = x[0, h, t].astype(np.float64)
            half = a / 254 if fmt == "int8" else np.maximum(np.abs(want) * 2.0 ** -4 * 1.1, a / 448 * 2.0 ** -10)
            assert (np.abs(got - want) <= (1 + grown[h, t]) * half * 1.0001).all()
    assert (raw[1] == 0x55).all() and (raw[2, :, n % P:] == 0x55).all()     # nothing else is written


def test_attend_reduces_to_plain_softmax():
    rng = np.random.default_rng(2)
    n, P, d = 37, 16, 16
    raw_k, raw_v = (rng.integers(0, 256, (4, 1, P, d)).astype(np.uint8) for _ in range(2))
    a = np.full((4, 1), 1.5, np.float32)
    q = rng.standard_normal((1, 2, 3, d)).astype(np.float16)
    out, mag, _ = q8.attend(raw_k, a, raw_v, a, q, np.array([[2, 1, 3]]), [n], "int8", 0.25)
    k = (raw_k.view(np.int8).astype(np.float64) * 1.5 / 127)[[2, 1, 3], 0].reshape(-1, d)[:n]
    v = (raw_v.view(np.int8).astype(np.float64) * 1.5 / 127)[[2, 1, 3], 0].reshape(-1, d)[:n]
    s = torch.from_numpy(q[0].astype(np.float64) @ k.T * 0.25)
    for i in range(3):
        s[:, i, n - 3 + i + 1:] = -np.inf
    want = torch.softmax(s, dim=-1).numpy() @ v
    assert np.abs(out[0] - want).max() < 1e-12 and (mag >= np.abs(out) - 1e-12).all()


def test_page_rules_keep_the_books():
    """Random extends, forks and compactions: every page is either free or counted exactly."""
    rnd = random.Random(3)
    B, W, n_pages, P = 6, 8, 60, 16
    st = dict(tables=[[-1] * W for _ in range(B)], seq_lens=[0] * B, refs=[0] * n_pages, free=list(range(n_pages)))
    refused = 0
    for step in range(300):
        kind = rnd.randrange(8)
        if kind < 5:
            _, ok = q8.extend(st, [rnd.choice([0, 1, 1, 5, 20]) for _ in range(B)], P, W)
            refused += not ok
        elif kind < 7:
            q8.fork(st, [rnd.randrange(-1, B) for _ in range(B)], P)
        else:
            remap = q8.compact(st, P)
            assert sorted(x for x in remap if x >= 0) == list(range(n_pages - len(st["free"])))
        count = [0] * n_pages
        for row, n in zip(st["tables"], st["seq_lens"]):
            for p in row[: -(-n // P)]:
                count[p] += 1
        assert count == st["refs"]
        assert sorted(st["free"]) == [p for p in range(n_pages) if not count[p]]
    assert refused
