"""Sizes and positions that do not fit the C ABI's fields are refused, not taken modulo 2^32 or 2^64 (no GPU needed:
the tensors hold one element, or none that is touched)."""
import pytest
import torch

import paper_1907_00641_amd as P

FAR = (1 << 32) + 5


def one(*shape):
    return torch.zeros(1).as_strided(shape, (0,) * len(shape))


def test_sizes_past_32_bits():
    q, k, v, lam = one(1, 2, 2, 2, 8), one(1, 2, 2, 2, 8), one(1, 2, 2, 8), torch.zeros(2)
    for args in ((one(1, FAR, 2, 2, 8), k, v, lam), (q, one(1, FAR, 2, 2, 8), one(1, FAR, 2, 8), lam),
                 (one(FAR, 2, 2, 2, 8), one(FAR, 2, 2, 2, 8), one(FAR, 2, 2, 8), lam),
                 (one(1, 2, FAR, 2, 8), k, v, one(FAR)), (q, k, one(1, 2, 2, FAR), lam),
                 (one(1, 2, 2, 2, FAR), one(1, 2, 2, 2, FAR), v, lam)):
        with pytest.raises(ValueError, match=r"2\^31"):
            P.pam_diff_attn_fwd(*args)
        with pytest.raises(ValueError, match=r"2\^31"):
            P.pam_diff_attn_bwd(*args, (None, None), args[0][:, :, :, 0])
    table = one(4, 4, 2)
    for args in ((one(1, FAR, 2, 8), None, table), (one(FAR, 1, 2, 8), None, table), (one(1, 2, FAR, 8), None, table),
                 (one(1, 2, 2, 8), one(1, 2, FAR, 8), table), (one(1, 2, 2, 8), None, one(4, FAR, 2))):
        with pytest.raises(ValueError, match=r"2\^31"):
            P.pam_rotary(*args)
    for start in (1 << 64, -(1 << 64), 1 << 62):
        with pytest.raises(ValueError, match=r"2\^62"):
            P.pam_rotary(one(1, 2, 2, 8), None, table, start=start)
    with pytest.raises(ValueError, match=r"2\^31"):
        P.pam_rotary_table(one(4).double(), coord=one(3, FAR))
    with pytest.raises(ValueError, match=r"2\^31"):
        P.pam_rotary_frequencies((1 << 32) + 8)
    with pytest.raises(ValueError, match=r"2\^31"):
        P.pam_norm_gate_fwd(one(3, FAR))
    with pytest.raises(ValueError, match=r"2\^31"):
        P.pam_norm_gate_bwd(one(3, FAR), grad_r=None, grad_h=None)
