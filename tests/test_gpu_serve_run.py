"""Serving from the 8-bit paged cache, the operators of include/lookat_serve.h together with those around them: packed prompts in,
beams out; every stage against its oracle on what the GPU itself handed to it."""
import math

import numpy as np
import pytest
import torch

from oracle import q8, serve
from paper_2601_10155_b200 import synth
from paper_2601_10155_b200.binding import BeamState, Lookat, LookatGpt2, PageState, Q8Cache, RopeTable
from test_gpu_serve import attend_bound, attend_reference, i32, rope_bound, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,H,H_kv,d,interleaved", [("int8", 8, 2, 64, False), ("e4m3", 4, 4, 128, True)])
def test_prompts_in_beams_out(fmt, H, H_kv, d, interleaved):
    """One layer: a fused projection of packed prompts, rotary positions in place, exact attention, keys and values into the
    pages; then beams of two prompts: a token's projection, positions, append, attention, logits, selection, fork."""
    rng = np.random.default_rng(H + d)
    dm, V, W, P, lens, steps = 256, 700, 3, 16, [37, 90], 6
    G, heads = len(lens), H + 2 * H_kv
    w = lambda n, k: torch.from_numpy((rng.standard_normal((n, k)) / math.sqrt(k)).astype(np.float16)).cuda()  # noqa: E731
    w_qkv, w_out, w_vocab, table = w(heads * d, dm), w(dm, H * d), 4 * w(V, dm), w(V, dm) * 16
    lk, rope = Lookat(H, H_kv, d, d, 1, 16), RopeTable(d // 2, 10000.0)
    ids = rng.integers(0, V, sum(lens))
    starts, pos = i32(starts_of(lens)), i32(np.concatenate([np.arange(n) for n in lens]))
    x = table[torch.from_numpy(ids).cuda()].contiguous()
    qkv = lk.lookat_linear(x, w_qkv).view(-1, heads, d)
    q, k, v = qkv.split([H, H_kv, H_kv], dim=1)
    before = qkv.clone()
    lk.lookat_rope(q, k, pos, rope, interleaved=interleaved, q_out=q, k_out=k)
    att = lk.lookat_attend_packed(q, k, v, starts)
    # a row per beam: the prompts lie in every group's first row, its other rows are forks of it
    B = G * W
    pages = PageState.empty(B, 12, 80, P)
    cache = Q8Cache.empty(80, H_kv, P, d, d, dtype=torch.int8 if fmt == "int8" else torch.float8_e4m3fn)
    first = [0] * B
    for g, n in enumerate(lens):
        first[g * W] = n
    lk.lookat_pages_extend(pages, i32(first), cache.pools())
    row_starts = i32(starts_of(first))
    lk.lookat_q8_append_packed(cache, k, v, row_starts, pages.tables, pages.seq_lens)
    lk.lookat_pages_fork(pages, i32([b // W * W for b in range(B)]))
    torch.cuda.synchronize()
    assert lk.lookat_last_error() == ""
    for got, had, n in ((q, before[:, :H], H), (k, before[:, H:H + H_kv], H_kv)):
        had = had.cpu().numpy()
        want = serve.rope(had, pos.tolist(), rope.host, rope.amplitude, interleaved)
        assert (np.abs(got.double().cpu().numpy() - want) <= rope_bound(had, rope.amplitude)).all()
    want, mag, reach = attend_reference(q, k, v, starts.tolist(), lk.scale)
    assert bool(((att.double() - want).abs() <= attend_bound(want, mag, reach, d, max(lens), float(v.abs().max()))).all())
    assert lk.lookat_linear(att.view(-1, H * d), w_out).isfinite().all()
    # the cache that the oracle would hold, in the rows' own pages (forks share: tables name the same ones)
    host = [t.view(torch.uint8).cpu().numpy().copy() if i % 2 == 0 else t.cpu().numpy().copy() for i, t in enumerate(cache.pools())]
    ref = [np.zeros_like(t) for t in host]
    tables = pages.tables.cpu().numpy()
    for g, n in enumerate(lens):
        lo, hi = int(starts[g]), int(starts[g + 1])
        for i, t in ((0, k), (2, v)):
            q8.append(ref[i], ref[i + 1], t[lo:hi].cpu().numpy().transpose(1, 0, 2)[None], tables[g * W:g * W + 1], [n], [n], fmt)
    assert all(np.array_equal(a, b) for a, b in zip(host, ref))

    # ---- beams ----
    st = BeamState.empty(G, W, steps)
    tokens = torch.from_numpy(np.repeat([int(ids[int(starts[g + 1]) - 1]) for g in range(G)], W)).cuda()
    one = torch.ones(B, dtype=torch.int32, device="cuda")
    for step in range(steps):
        lk.lookat_pages_extend(pages, one, cache.pools())
        qkv = lk.lookat_linear(table[tokens.long()].contiguous(), w_qkv).view(B, heads, d)
        qn, kn, vn = qkv.split([H, H_kv, H_kv], dim=1)
        p = pages.seq_lens - 1
        qr, kr = lk.lookat_rope(qn, kn, p, rope, interleaved=interleaved)
        lk.lookat_q8_append_packed(cache, kr, vn, torch.arange(B + 1, dtype=torch.int32, device="cuda"), pages.tables, pages.seq_lens)
        out = lk.lookat_attend_q8(cache, qr, pages.tables, pages.seq_lens)
        logits = lk.lookat_linear(lk.lookat_linear(out.half().view(B, H * d), w_out), w_vocab, out_fp16=False)
        torch.cuda.synchronize()
        had = [t.cpu().numpy().copy() for t in (st.scores, st.lengths, st.finished, st.tokens)]
        rows = pages.tables.cpu().numpy(), pages.seq_lens.tolist()
        kc, ka, vc, va = (t.view(torch.uint8).cpu().numpy() if i % 2 == 0 else t.cpu().numpy() for i, t in enumerate(cache.pools()))
        ref_out, _, reach = q8.attend(kc, ka, vc, va, qr.cpu().numpy()[:, :, None], *rows, fmt, lk.scale)
        err = np.linalg.norm(out.double().cpu().numpy() - ref_out[:, :, 0]) / np.linalg.norm(ref_out)
        assert err <= q8.attend_rms_tolerance(reach, d, max(rows[1]))
        nxt, parents = lk.lookat_beam_select(st, logits, eos=5, length_penalty=0.6)
        lk.lookat_pages_fork(pages, parents)
        torch.cuda.synchronize()
        sel = serve.beam_select(*had, logits.cpu().numpy(), 5, 0.6)
        assert sel[6] > 2e-5 and nxt.tolist() == sel[4].tolist() and parents.tolist() == sel[5].tolist()
        assert np.array_equal(st.tokens.cpu().numpy(), sel[3])
        assert pages.tables[:, :].cpu().numpy()[:, 0].tolist() == [rows[0][p][0] for p in parents.tolist()]
        tokens = nxt
    assert lk.lookat_last_error() == ""
    assert pages.seq_lens.view(G, W).tolist() == [[n + steps] * W for n in lens]


def test_beam_search_with_the_gpt2_harness():
    """A batch of beams over the harness's 8-bit cache: selection between decode steps and forks.  Afterwards every beam's tokens,
    fed one by one to a fresh model, give the beam's score again."""
    G, W, T0, steps, vocab, n_head = 2, 3, 20, 5, 500, 4
    B = G * W
    wd = synth.gpt2_weights(31, n_layer=2, n_head=n_head, d_model=64 * n_head, vocab=vocab, n_pos=T0 + steps + 2, plain_init=False)
    ids = synth.token_ids(33, G, T0, vocab)
    prompt = torch.from_numpy(np.repeat(ids, W, axis=0)).cuda().int()

    def model():
        g = LookatGpt2(wd, B, T0 + steps, 4, 16, fit_iters=1)
        g.lookat_gpt2_use_q8_cache(16, torch.int8)
        g.lookat_gpt2_prefill(prompt[:, :T0 - 1].contiguous())
        return g

    gpu, lk, st = model(), Lookat(4, 4, 64, 64, 1, 16), BeamState.empty(G, W, steps)
    feed = prompt[:, T0 - 1].contiguous()
    for step in range(steps):
        _, logits, _ = gpu.lookat_gpt2_decode(feed, want_logits=True)
        torch.cuda.synchronize()
        had = [t.cpu().numpy().copy() for t in (st.scores, st.lengths, st.finished, st.tokens)]
        feed, parents = lk.lookat_beam_select(st, logits)
        gpu.lookat_gpt2_fork(parents)
        torch.cuda.synchronize()
        sel = serve.beam_select(*had, logits.cpu().numpy(), -1, 0.0)
        assert sel[6] > 2e-5 and feed.tolist() == sel[4].tolist() and parents.tolist() == sel[5].tolist()
    assert gpu.lookat_gpt2_last_error() == ""
    tokens, scores = st.tokens.view(B, steps), st.scores.view(B)
    assert len({tuple(t) for t in tokens[:W].tolist()}) == W
    again, total = model(), torch.zeros(B, dtype=torch.float64, device="cuda")
    feed = prompt[:, T0 - 1].contiguous()
    for step in range(steps):
        _, logits, _ = again.lookat_gpt2_decode(feed, want_logits=True)
        feed = tokens[:, step].contiguous()
        total += torch.log_softmax(logits.double(), dim=1).gather(1, feed.long()[:, None])[:, 0]
    # the same kernels on the same rows, the scores rounded once a step (2^-24 of at most 100) over sums good to 2^-20
    assert float((total - scores.double()).abs().max()) <= steps * (100 * 2.0 ** -24 + 2.0 ** -20)


def test_the_debug_build_serves_as_well():
    """The same calls in the library that checks codes."""
    x = torch.randn(300, 12, 64, device="cuda").half()
    q, k, v = x.split([8, 2, 2], dim=1)
    got = []
    for debug in (False, True):
        lk = Lookat(8, 2, 64, 64, 4, 16, debug=debug)
        a, b = lk.lookat_rope(q, k, torch.arange(300, dtype=torch.int32, device="cuda"), RopeTable(64))
        st = BeamState.empty(2, 2, 4)
        ids, _ = lk.lookat_beam_select(st, x.view(300, -1)[:4].float())
        got.append((a, b, lk.lookat_attend_packed(a, b, v, i32([0, 170, 300])), ids, st.scores))
        torch.cuda.synchronize()
        assert lk.lookat_last_error() == ""
    assert all(torch.equal(y, z) for y, z in zip(*got))
