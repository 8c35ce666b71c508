"""The GPT-2 harness over the 8-bit paged cache when something goes wrong between steps: nothing is lost silently."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_10155_b200 import synth
from paper_2601_10155_b200.binding import LookatError, LookatGpt2, _RawDeviceArray, lookat_page_state, lookat_q8_cache

pytestmark = pytest.mark.gpu

B, T0, VOCAB, PAGE = 3, 32, 300, 16
IDS = synth.token_ids(52, B, T0 + 8, VOCAB)
WEIGHTS = synth.gpt2_weights(51, n_layer=2, n_head=2, d_model=128, vocab=VOCAB, n_pos=T0 + 8, plain_init=False)


def ids(t):
    return torch.from_numpy(np.ascontiguousarray(IDS[:, t])).cuda()


def model(stream=None):
    m = LookatGpt2(WEIGHTS, B, T0 + 8, 4, 16, fit_iters=1, stream=stream)
    m.lookat_gpt2_use_q8_cache(PAGE)
    return m


def prompt(m):
    m.lookat_gpt2_prefill(torch.from_numpy(np.ascontiguousarray(IDS[:, :T0])).cuda())
    torch.cuda.synchronize()
    return m


def step(m, t):
    hidden, _, _ = m.lookat_gpt2_decode(ids(T0 + t), want_hidden=True)
    torch.cuda.synchronize()
    return hidden


def pages(m):
    """The model's own page state: tables, seq_lens, refs, free_list, n_free."""
    c, s = lookat_q8_cache(), lookat_page_state()
    m._check(m._lib.lookat_gpt2_q8_state(m._h, 0, ctypes.byref(c), ctypes.byref(s)))
    view = lambda p, *shape: torch.as_tensor(_RawDeviceArray(p, shape, "<i4"), device="cuda")  # noqa: E731
    return view(s.tables, s.B, s.max_pages), view(s.seq_lens, s.B), view(s.refs, s.n_pages), view(s.free_list, s.n_pages), view(s.n_free, 1)


def finding(m):
    torch.cuda.synchronize()
    return m.lookat_gpt2_last_error()


def test_findings_of_the_models_kernels_are_reported():
    m = prompt(model())
    tables = pages(m)[0]
    assert finding(m) == ""
    held = int(tables[1, 0])
    tables[1, 0] = 10000
    step(m, 0)
    with pytest.raises(LookatError, match="layer 9"):           # a refused call's own error comes first
        m.lookat_gpt2_q8_state(9)
    assert "outside its range" in finding(m)
    tables[1, 0] = held
    step(m, 1)
    assert finding(m) == ""


@pytest.mark.parametrize("bad", [-1, 3, 2 ** 31 - 1, -2 ** 31])
def test_a_parent_out_of_range_leaves_the_row_as_it_is(bad):
    """The harness's rows all have one length: a row cannot become empty between steps."""
    m, want = prompt(model()), prompt(model())
    step(m, 0), step(want, 0)
    parents = torch.tensor([2, bad, 2], dtype=torch.int32, device="cuda")
    m.lookat_gpt2_fork(parents)
    want.lookat_gpt2_fork(torch.tensor([2, 1, 2], dtype=torch.int32, device="cuda"))
    assert "outside its range" in finding(m) and finding(want) == ""
    assert parents.tolist() == [2, bad, 2]
    assert pages(m)[1].tolist() == [T0 + 1] * B
    for t in (1, 2):
        assert torch.equal(step(m, t), step(want, t))


def test_a_refused_step_does_not_make_later_ones_write_over_the_newest_token():
    """The free list runs out at a page border: the step is refused on the device and reported, nothing is written, and the
    steps after the pages are back take room again."""
    m = prompt(model())                                         # 32 tokens: the next one needs a page
    tables, seq_lens, refs, free_list, n_free = pages(m)
    before = [t.clone() for t in m.lookat_gpt2_q8_state(1)]
    free = int(n_free)
    n_free.zero_()
    step(m, 0)
    assert "too few free pages" in finding(m)
    n_free.fill_(free)
    for a, b in zip(before, m.lookat_gpt2_q8_state(1)):
        assert torch.equal(a, b)
    for t in (1, 2):
        step(m, t)
        assert finding(m) == "" and seq_lens.tolist() == [T0 + t] * B
    after = m.lookat_gpt2_q8_state(1)
    for b in range(B):                                          # the prompt's tokens are as they were
        for i in range(T0 // PAGE):
            for x, y in ((before[0], after[0]), (before[2], after[2])):
                assert torch.equal(x[before[4][b, i]], y[after[4][b, i]])


def attention_of(m):
    """The model's attention context (its address follows the configuration, three ints and the stream)."""
    at = ctypes.sizeof(m.cfg)
    at = (at + 12 + 7) // 8 * 8 + 8
    h = ctypes.c_void_p.from_address(m._h.value + at)
    assert m._lib.lookat_kernel_launches(h) == m.lookat_gpt2_kernel_launches() > 0
    return h


def test_a_step_that_failed_half_way_is_not_repeated_on_top_of_itself():
    """A time-out is found after the step has taken its pages (a self-test kernel's wait that nothing ends): the model then
    refuses steps and forks until the next prompt, and is as good as new after it."""
    m, want = prompt(model()), prompt(model())
    step(m, 0)
    m._lib.lookat_selftest_timeout(attention_of(m))
    torch.cuda.synchronize()
    with pytest.raises(LookatError, match="gave up"):
        step(m, 1)
    for _ in range(2):
        with pytest.raises(LookatError, match="prompt"):
            step(m, 1)
    with pytest.raises(LookatError, match="prompt"):
        m.lookat_gpt2_fork(torch.zeros(B, dtype=torch.int32, device="cuda"))
    prompt(m)
    for t in range(3):
        assert torch.equal(step(m, t), step(want, t))


def test_a_prompt_that_failed_half_way_leaves_nothing_to_continue():
    m, want = prompt(model()), prompt(model())
    step(m, 0)
    m._lib.lookat_selftest_timeout(attention_of(m))
    torch.cuda.synchronize()
    with pytest.raises(LookatError, match="gave up"):
        prompt(m)
    with pytest.raises(LookatError, match="prompt"):
        step(m, 1)
    prompt(m)
    for t in range(3):
        assert torch.equal(step(m, t), step(want, t))


def test_the_first_step_can_be_captured():
    """The workspaces are made with the cache, so no step and no fork has to allocate."""
    want = prompt(model())
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        m = prompt(model(stream=s))
        x, hidden, parents = ids(T0), torch.zeros(B, 128, device="cuda"), torch.arange(B, dtype=torch.int32, device="cuda")
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got, _, _ = m.lookat_gpt2_decode(x, want_hidden=True)
            hidden.copy_(got)
            m.lookat_gpt2_fork(parents)
        g.replay()
        s.synchronize()
        assert finding(m) == "" and torch.equal(hidden, step(want, 0))
        del g


def test_the_cache_replaces_codes_and_values():
    """Codebooks, codes and fp16 values are given back: the 8-bit cache takes less than they did."""
    cap = 1024
    step(prompt(model()), 0)                                    # (the kernels are loaded before memory is counted)
    w = synth.gpt2_weights(53, n_layer=4, n_head=8, d_model=512, vocab=50, n_pos=cap)
    torch.cuda.synchronize()
    m = LookatGpt2(w, 16, cap, 4, 16, fit_iters=1)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    m.lookat_gpt2_use_q8_cache(PAGE)
    torch.cuda.synchronize()
    # per layer: 16.8 MB of values and 2 MB of codes go, 16.8 MB of pages come; 16.8 MB of values for a prompt, once
    assert before - torch.cuda.mem_get_info()[0] < 20 << 20
    assert m.lookat_gpt2_layer_state(0)[:3] == (None, None, None)
    m.lookat_gpt2_prefill(torch.zeros(16, 40, dtype=torch.int32, device="cuda"))
    m.lookat_gpt2_decode(torch.zeros(16, dtype=torch.int32, device="cuda"))
    assert finding(m) == ""
