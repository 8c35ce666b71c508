"""The GPT-2 harness over the 8-bit paged cache: the prompt's cache bit for bit on the GPU's own keys and values, then
teacher-forced steps and beam forks against the decoder oracle (tolerances as in test_gpu_gpt2.py)."""
import numpy as np
import pytest
import torch

from oracle import gpt2 as ref
from oracle import q8
from paper_2601_10155_b200 import synth
from paper_2601_10155_b200.binding import LookatError, LookatGpt2

pytestmark = pytest.mark.gpu

DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def close(got, want, rel, what=""):
    got, want = np.asarray(got, dtype=np.float64), np.asarray(want, dtype=np.float64)
    scale = float(np.sqrt((want ** 2).mean())) + 1e-30
    excess = np.abs(got - want) - 1e-3 * np.abs(want)
    assert float(excess.max()) <= rel * scale, f"{what}: error {float(np.abs(got - want).max()):.3e} against scale {scale:.3e}"


class Q8Decoder:
    """The decoder oracle over per-row 8-bit caches (no pages are shared here: a fork copies)."""

    def __init__(self, w, caches, page, fmt):
        self.w, self.caches, self.page, self.fmt = w, caches, page, fmt      # per layer [k, ka, v, va] of dense rows' pages
        self.pos = None

    def step(self, ids):
        w, d = self.w, self.w.d_model
        x = ref.embed(w, np.asarray(ids)[:, None], self.pos)
        B = len(ids)
        for l, lw in enumerate(w.layers):
            qkv = ref.linear(ref.layer_norm(x, lw["ln1_g"], lw["ln1_b"]), lw["w_qkv"], lw["b_qkv"])
            q16, k16, v16 = (ref.split_heads(qkv[..., i * d:(i + 1) * d], w.n_head).astype(np.float16) for i in range(3))
            k, ka, v, va = self.caches[l]
            W = k.shape[0] // B
            tables = np.arange(B * W).reshape(B, W)
            lens = [self.pos + 1] * B
            q8.append(k, ka, k16, tables, lens, [1] * B, self.fmt)
            q8.append(v, va, v16, tables, lens, [1] * B, self.fmt)
            att, _, _ = q8.attend(k, ka, v, va, q16, tables, lens, self.fmt, 0.125)
            x = x + ref.linear(att.reshape(B, 1, d), lw["w_o"], lw["b_o"])
            x = ref.block_mlp(lw, x)
        self.pos += 1
        return x[:, 0]

    def fork(self, parents):
        for c in self.caches:
            for i in range(4):
                rows = c[i].reshape(len(parents), -1, *c[i].shape[1:])
                c[i] = rows[parents].reshape(c[i].shape).copy()


@pytest.mark.parametrize("fmt,page", [("int8", 16), ("e4m3", 32)])
def test_decoder_over_the_8_bit_cache(fmt, page):
    n_layer, n_head, B, T0, steps, vocab = 2, 4, 3, 70, 6, 500
    wd = synth.gpt2_weights(31, n_layer=n_layer, n_head=n_head, d_model=64 * n_head, vocab=vocab, n_pos=T0 + steps + 2, plain_init=False)
    ids = synth.token_ids(32, B, T0 + steps, vocab)
    w = ref.Gpt2Weights.from_dict(wd)
    cap = T0 + steps
    plain = LookatGpt2(wd, B, cap, 4, 16, fit_iters=1, keep_prompt_keys=True)
    gpu = LookatGpt2(wd, B, cap, 4, 16, fit_iters=1)
    with pytest.raises(LookatError, match="does not use"):
        gpu.lookat_gpt2_fork(torch.zeros(B, dtype=torch.int32, device="cuda"))
    gpu.lookat_gpt2_use_q8_cache(page, DTYPE[fmt])
    with pytest.raises(LookatError, match="once"):
        gpu.lookat_gpt2_use_q8_cache(page, DTYPE[fmt])
    h0 = plain.lookat_gpt2_prefill(dev(ids[:, :T0]), want_hidden=True)
    gpu.lookat_gpt2_prefill(dev(ids[:, :T0][::-1]))                          # another prompt first: its pages are freed
    h1 = gpu.lookat_gpt2_prefill(dev(ids[:, :T0]), want_hidden=True)
    assert torch.equal(h0, h1), "the prompt pass does not depend on the cache"
    W = -(-cap // page)
    caches = []
    for l in range(n_layer):
        _, _, values, keys = plain.lookat_gpt2_layer_state(l, T=T0)
        k, ka, v, va, tables, lens, refs, free, n_free = (t.cpu().numpy() for t in gpu.lookat_gpt2_q8_state(l))
        assert lens.tolist() == [T0] * B and int(n_free[0]) == B * W - B * -(-T0 // page)
        want = []
        for got, got_a, x in ((k, ka, keys), (v, va, values[:, :, :T0])):
            raw, a = np.zeros((B * W, n_head, page, 64), np.uint8), np.zeros((B * W, n_head), np.float32)
            dense = np.arange(B * W).reshape(B, W)
            q8.append(raw, a, x.cpu().numpy(), dense, [T0] * B, [T0] * B, fmt)
            for b in range(B):
                for i in range(-(-T0 // page)):
                    m = min(page, T0 - i * page)
                    assert np.array_equal(got[tables[b, i]][:, :m], raw[dense[b, i]][:, :m]), f"layer {l}"
                    assert np.array_equal(got_a[tables[b, i]], a[dense[b, i]])
            want += [raw, a]
        caches.append(want)
    dec = Q8Decoder(w, caches, page, fmt)
    dec.pos = T0
    for t in range(steps):
        if t in (2, 4):
            parents = [1, 1, 0] if t == 2 else [2, 0, 0]
            gpu.lookat_gpt2_fork(torch.tensor(parents, dtype=torch.int32, device="cuda"))
            dec.fork(parents)
        hid, logits, nxt = gpu.lookat_gpt2_decode(dev(ids[:, T0 + t]), want_hidden=True, want_logits=True, want_next=True)
        torch.cuda.synchronize()
        x = dec.step(ids[:, T0 + t])
        close(hid.cpu().numpy(), x, 2e-2, f"step {t}, residual stream")
        close(logits.cpu().numpy(), ref.logits_of(w, x), 2e-2, f"step {t}, logits")
    assert gpu.lookat_gpt2_position() == T0 + steps
    k, ka, v, va, tables, lens, refs, free, n_free = (t.cpu().numpy() for t in gpu.lookat_gpt2_q8_state(0))
    assert lens.tolist() == [cap] * B
    held = np.bincount(tables.reshape(-1), minlength=B * W)
    assert np.array_equal(held, refs) and int(n_free[0]) == int((refs == 0).sum())
