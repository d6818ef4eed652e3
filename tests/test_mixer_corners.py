"""Calls of the operators around the attention that the binding refuses before the library would see something else (no GPU)."""
import pytest
import torch

from paper_2607_17419_b200 import binding as kb


@pytest.mark.parametrize("rotary_dim", [17, 33, 1, 63, -1, -2, -16, -64])
@pytest.mark.parametrize("given", [False, True])
def test_rotary_dim_that_is_no_number_of_pairs(rotary_dim, given):
    """Halved, 33 would be 32 and -64 nothing at all: another rotation than the one asked for."""
    q = torch.zeros(2, 4, 5, 64)
    inv_freq = [1.0] * max(0, rotary_dim // 2) if given else None
    for call in (lambda: kb.kata_fwd_norm_rope(q, q, inv_freq=inv_freq, rotary_dim=rotary_dim),
                 lambda: kb.kata_bwd_norm_rope(q, q, q, q, inv_freq=inv_freq, rotary_dim=rotary_dim)):
        with pytest.raises(ValueError, match="rotary_dim"):
            call()
    for even in (0, 16, 64):
        assert len(kb._rope_freq(q, 10000.0, None, even)) == even // 2
