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
