"""Arguments of rotary positions and attention of chunks that the native half and ctypes have to agree on."""
import numpy as np
import pytest
import torch

from gpu_util import dev
from kvq_util import seed
from test_gpu_kvq import binding
from test_gpu_rope import frequencies

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T_max", [-1, -5, -2 ** 31])
@pytest.mark.parametrize("packed", [True, False])
def test_less_than_no_rows_are_refused(packed, T_max):
    """Direct calls (which the native half takes where it can) and prepared ones (which ctypes makes) alike; nothing is written."""
    b, D, H = binding(), 64, 2
    lead = (6,) if packed else (2, 3)
    x = lambda h: torch.ones(lead + (h, D), dtype=torch.bfloat16, device="cuda")                     # noqa: E731
    q, k, out = x(4), x(H), x(4)
    rows = dict(row_starts=dev(np.array([0, 3, 6], np.int32))) if packed else {}
    rope, c, tables, ctx = b.Rope(dev(frequencies(32))), b.KvqCache(4, 16, H, D), torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = b.new_workspace(b.radar_chunk_attention_kvq_workspace_bytes(b.kvq_chunk_desc(q, c, 2, 2, 3, 6)))
    for prepared in (False, True):
        for call in (lambda: b.radar_rope(q, k, rope, ctx_lens=ctx, T_max=T_max, q_out=out, prepared=prepared, **rows),
                     lambda: b.radar_chunk_attention_kvq(q, c, tables, ctx, T_max=T_max, out=out, workspace=ws, prepared=prepared, **rows)):
            with pytest.raises((ValueError, b.RadarError)):
                got = call()
                if prepared:
                    got()
    assert (out == 1).all()
