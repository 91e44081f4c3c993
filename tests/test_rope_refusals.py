"""More sequences than rotation counts in 32 bits, on the CPU: with row_starts their number is bounded by nothing else."""
import pytest

from test_chunk_refusals import ONE, append_call, rope_call
from test_kvq_refusals import lib  # noqa: F401


@pytest.mark.parametrize("B", [(1 << 30) + 1, (1 << 31) - 64, (1 << 31) - 1])
def test_more_sequences_than_are_counted(lib, B):  # noqa: F811
    """Starts near the 2^31st would be looked at under numbers that have become negative."""
    assert rope_call(lib, starts=ONE, B=B, N=4) == -2
    assert append_call(lib, 7, ONE, B=B, N=4) == -2                  # (7: row_starts)
    assert rope_call(lib, starts=ONE, B=1 << 30, N=0) == 0           # nothing to do, nothing launched


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-50, -1e-46])
def test_a_scale_that_32_bits_make_zero(scale):
    """The descriptor's zero stands for one."""
    import torch
    from paper_2512_14069_amd import binding as b
    with pytest.raises(ValueError):
        b.Rope(torch.ones(8), scale=scale)
    assert b.Rope(torch.ones(8), scale=1e-45).desc().scale != 0.0
