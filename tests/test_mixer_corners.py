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


BIG = (1 << 32) + 2


@pytest.mark.parametrize("axis", [0, 1, 2])
def test_sizes_beyond_32_bits_are_refused(axis):
    """The argument structs hold 32 bits: 2^32 + 2 tokens must not become two of them."""
    def wide(*shape):
        return torch.zeros(1).expand(*shape)
    def rows(*shape):
        return torch.zeros(shape[-1]).expand(*shape)
    shape = [2, 2, 2]
    shape[axis] = BIG
    q = rows(*shape, 64)
    for make in (lambda: kb._rope_args(q, None, None, None, None, 0, (1.0,) * 8, False, 1e-6),
                 lambda: kb._ssm_args(q, q, q, wide(*shape), wide(shape[1]), None, None, False, None, q)):
        with pytest.raises(ValueError, match="32 bits"):
            make()
    if axis == 1:
        with pytest.raises(ValueError, match="32 bits"):          # heads of the keys alone
            kb._rope_args(rows(2, 2, 2, 64), rows(2, BIG, 2, 64), None, None, None, 0, (1.0,) * 8, False, 1e-6)
        with pytest.raises(ValueError, match="32 bits"):          # tokens
            kb._conv_args(rows(2, BIG, 64), torch.zeros(64, 4), None, True, None, None, None)
    if axis == 0:
        with pytest.raises(ValueError, match="32 bits"):
            kb._conv_args(rows(BIG, 2, 64), torch.zeros(64, 4), None, True, None, None, None)
