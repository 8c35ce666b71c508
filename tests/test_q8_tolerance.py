"""The tolerance of fp32 attention results (oracle.q8.attend_rms_tolerance) on the CPU: plain fp32 arithmetic keeps well
inside it, softmax weights of 11 bits do not (what a kernel that lost their second halves would give)."""
import numpy as np
import pytest

from oracle import q8


def forms(rng, n, d, gap, chunk):
    """64-bit result, fp32 result (tokens summed in chunks), result with weights rounded to fp16, and the reach."""
    k, v = rng.standard_normal((n, d)), rng.standard_normal((n, d))
    q = 0.9 * rng.standard_normal(d)
    if gap:
        k[:, 0], q[0] = 0, 4.0
        k[0], v[0] = 0, 0
        k[0, 0] = gap * np.sqrt(d) / 4
    k, v, q = (x.astype(np.float32) for x in (k, v, q))
    s = k.astype(np.float64) @ q.astype(np.float64) / np.sqrt(d)
    w = np.exp(s - s.max())
    out = w @ v.astype(np.float64) / w.sum()
    s32 = (k @ q) * np.float32(1 / np.sqrt(d))
    w32 = np.exp(s32 - s32.max())
    sums = [w32[i:i + chunk] @ v[i:i + chunk] for i in range(0, n, chunk)]
    low = (w32 * np.float32(128)).astype(np.float16).astype(np.float64) @ v / (np.float64(128) * w32.astype(np.float64).sum())
    reach = (np.abs(k) @ np.abs(q)).max() / np.sqrt(d)
    return out, np.sum(sums, axis=0, dtype=np.float32) / w32.sum(dtype=np.float32), low, reach


@pytest.mark.parametrize("n,d,gap", [(1000, 128, 0), (3000, 128, 0), (9000, 128, 0), (2500, 64, 0), (5000, 64, 0), (4096, 64, 12), (32768, 64, 12)])
def test_the_tolerance_takes_fp32_and_refuses_fp16_weights(n, d, gap):
    rng = np.random.default_rng(n)
    out, full, low = (np.array(x) for x in zip(*[forms(rng, n, d, gap, 64)[:3] for _ in range(6)]))
    reach = max(forms(rng, n, d, gap, 64)[3] for _ in range(6))
    tol = q8.attend_rms_tolerance(reach, d, n)
    off = lambda x: np.linalg.norm(x - out) / np.linalg.norm(out)  # noqa: E731
    assert off(full) < tol / 4 and off(low) > 1.5 * tol, (off(full), off(low), tol)
