"""What the binding of include/lookat_serve.h refuses before the library or a device is asked (no GPU needed)."""
import pytest
import torch

from paper_2601_10155_b200.binding import Lookat, RopeTable


def context_of_nothing(n_q_heads, n_kv_heads, d_k, d_v):
    """A Lookat without a library context: calls that are refused do not come that far."""
    lk = Lookat.__new__(Lookat)
    lk._h, lk._lib, lk.device = None, None, torch.device("cuda", 0)
    lk._shape = (n_q_heads, n_kv_heads, d_k, d_v)
    return lk


def test_rope_refuses_a_result_without_its_input():
    """The result would come back as it was, as if it had been filled."""
    lk = context_of_nothing(4, 2, 64, 64)
    table = RopeTable.__new__(RopeTable)
    table.device = lk.device
    q, k = torch.zeros(3, 4, 64, dtype=torch.float16), torch.zeros(3, 2, 64, dtype=torch.float16)
    positions = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="without its input"):
        lk.lookat_rope(q, None, positions, table, k_out=k)
    with pytest.raises(ValueError, match="without its input"):
        lk.lookat_rope(None, k, positions, table, q_out=q)
    with pytest.raises(ValueError, match="both None"):
        lk.lookat_rope(None, None, positions, table, q_out=q)
