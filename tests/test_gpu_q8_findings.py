"""Findings and refusals of the 8-bit paged cache: what is out of range is reported, what is not is not."""
import numpy as np
import pytest
import torch

from oracle import q8
from paper_2601_10155_b200.binding import Lookat, LookatError, PageState, Q8Cache

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def state(tables, seq_lens, refs, free, page=16):
    n = len(refs)
    return PageState(i32(tables), i32(seq_lens), i32(refs), i32(list(free) + [-7] * (n - len(free))), i32([len(free)]), page)


def finding(lk):
    torch.cuda.synchronize()
    return lk.lookat_last_error()


def test_a_negative_count_is_zero_in_a_whole_step():
    """extend takes a negative count as 0 and leaves it as it is; append then takes it the same way, without a finding."""
    lk = Lookat(2, 2, 64, 64, 1, 16)
    cache, ps = Q8Cache.empty(6, 2, 16, 64, 64), PageState.empty(3, 2, 6, 16)
    x = torch.randn(3, 2, 5, 64, device="cuda").half()
    n_new = i32([5, -1, -2147483648])
    lk.lookat_pages_extend(ps, n_new, cache.pools())
    lk.lookat_q8_append(cache, x, x, ps.tables, ps.seq_lens, n_new)
    lk.lookat_attend_q8(cache, x[:, :, :1].contiguous(), ps.tables, ps.seq_lens)
    assert finding(lk) == ""
    assert ps.seq_lens.tolist() == [5, 0, 0] and n_new.tolist() == [5, -1, -2147483648]
    # a row that holds tokens keeps them, scales among them
    before = [t.clone() for t in cache.pools()]
    lk.lookat_q8_append(cache, 9 * x, 9 * x, ps.tables, ps.seq_lens, i32([-3, 0, -1]))
    assert finding(lk) == "" and all(torch.equal(a, b) for a, b in zip(before, cache.pools()))
    lk.lookat_q8_append(cache, x, x, ps.tables, ps.seq_lens, i32([6, 0, 0]))             # more than there are: still a finding
    assert "outside its range" in finding(lk)


def test_page_calls_without_pools():
    """None stands for no pools, as NULL does in C."""
    lk = Lookat(2, 2, 64, 64, 1, 16)
    ps = state([[0, -1], [1, -1]], [5, 16], [1, 1, 0, 0], [2, 3])
    lk.lookat_pages_extend(ps, i32([1, 1]), None)
    assert finding(lk) == "" and ps.tables.tolist() == [[0, -1], [1, 3]] and ps.seq_lens.tolist() == [6, 17]
    remap = i32([9] * 4)
    lk.lookat_pages_compact(ps, None, remap)
    assert finding(lk) == "" and remap.tolist() == [0, 1, -1, 2] and ps.tables.tolist() == [[0, -1], [1, 2]]


def test_two_findings_are_both_reported():
    lk = Lookat(2, 2, 64, 64, 1, 16)
    cache, ps = Q8Cache.empty(2, 2, 16, 64, 64), state([[0, -1]], [10], [1, 0], [1])
    q = torch.zeros(1, 2, 1, 64, dtype=torch.float16, device="cuda")
    lk.lookat_attend_q8(cache, q, i32([[7, 0]]), ps.seq_lens)
    lk.lookat_pages_extend(ps, i32([100]), [])
    first, second = finding(lk), finding(lk)
    assert "too few free pages" in first and "outside its range" in second


def test_compact_reports_a_length_out_of_range():
    lk = Lookat(2, 2, 64, 64, 1, 16)
    for bad in (-1, 33):
        ps = state([[0, 1], [2, -1]], [bad, 16], [1, 1, 1, 0], [3])
        lk.lookat_pages_compact(ps, [])
        assert "outside its range" in finding(lk)
        lk = Lookat(2, 2, 64, 64, 1, 16)
    ps = state([[0, 1], [2, -1]], [32, 0], [1, 1, 0, 0], [2, 3])
    lk.lookat_pages_compact(ps, [])
    assert finding(lk) == ""


def test_extend_reports_a_free_list_entry_out_of_range():
    for entry in (-3, 4, 2 ** 31 - 1):
        lk = Lookat(2, 2, 64, 64, 1, 16)
        ps = state([[0, -1], [1, -1]], [16, 16], [1, 1, 0, 0], [entry, 2])
        lk.lookat_pages_extend(ps, i32([1, 1]), [torch.zeros(4, 4, device="cuda")])
        assert "outside its range" in finding(lk)
        assert ps.refs.tolist() == [1, 1, 1, 0] and ps.tables[0].tolist() == [0, 2]


def test_lengths_beyond_the_table_are_taken_as_its_end():
    """Row 0 asks for more tokens than its table holds, row 1 for fewer than none: the first attends its whole table."""
    rng = np.random.default_rng(13)
    k, v = (rng.integers(-127, 128, (9, 2, 16, 64)).astype(np.int8) for _ in range(2))
    ka, va = (rng.uniform(0.5, 2, (9, 2)).astype(np.float32) for _ in range(2))
    tables = np.array([[3, 0, 8, 5, 2, 7, 1], [4, 6, 4, 4, 4, 4, 4]], np.int32)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    for L_q in (1, 6, 70):
        lk = Lookat(4, 2, 64, 64, 1, 16)
        q = rng.standard_normal((2, 4, L_q, 64)).astype(np.float16)
        got = lk.lookat_attend_q8(Q8Cache(dev(k), dev(ka), dev(v), dev(va)), dev(q), dev(tables), i32([100000, -3]))
        assert "outside its range" in finding(lk)
        out, _, reach = q8.attend(k.view(np.uint8), ka, v.view(np.uint8), va, q, tables, [112, 0], "int8", lk.scale)
        got = got.double().cpu().numpy()
        assert (got[1] == 0).all()
        assert np.linalg.norm(got[0] - out[0]) <= q8.attend_rms_tolerance(reach, 64, 112) * np.linalg.norm(out[0])


def test_a_refused_call_is_not_explained_by_an_earlier_finding():
    lk = Lookat(2, 2, 64, 64, 1, 16)
    cache, lens = Q8Cache.empty(2, 2, 16, 64, 64), i32([10])
    q = torch.zeros(1, 2, 1, 64, dtype=torch.float16, device="cuda")
    lk.lookat_attend_q8(cache, q, i32([[7, 0]]), lens)
    torch.cuda.synchronize()
    with pytest.raises(LookatError, match="L_q=0"):
        lk.lookat_attend_q8(cache, q[:, :, :0].contiguous(), i32([[0, 0]]), lens)
    assert "outside its range" in finding(lk)
    with pytest.raises(LookatError, match="L_q=0"):
        lk.lookat_attend_q8(cache, q[:, :, :0].contiguous(), i32([[0, 0]]), lens)
