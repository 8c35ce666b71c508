"""Findings and refusals of the 8-bit paged cache: what is out of range is reported, what is not is not."""
import numpy as np
import pytest
import torch

from oracle import q8
from paper_2601_10155_b200.binding import Lookat, PageState, Q8Cache

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def state(tables, seq_lens, refs, free, page=16):
    n = len(refs)
    return PageState(i32(tables), i32(seq_lens), i32(refs), i32(list(free) + [-7] * (n - len(free))), i32([len(free)]), page)


def finding(lk):
    torch.cuda.synchronize()
    return lk.lookat_last_error()


