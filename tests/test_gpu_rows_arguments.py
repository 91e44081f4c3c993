"""Arguments of rotary positions and attention of chunks that the native half and ctypes have to agree on."""
import numpy as np
import pytest
import torch

from gpu_util import dev
from kvq_util import seed
from test_gpu_kvq import binding
from test_gpu_rope import frequencies
from test_gpu_support import _Both

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


@pytest.mark.parametrize("Hkv,N", [(2, 1), (1, 4), (1, 1)])
def test_strides_of_one_entry_say_nothing(Hkv, N, monkeypatch):
    """Keys and values whose strides differ only where an axis has one entry: the bytes of the same call over dense ones, by the native half and by ctypes."""
    b, rng, D = binding(), seed(995 + N), 64
    dense = [torch.from_numpy(rng.normal(size=(1, N, Hkv, D))).bfloat16().cuda() for _ in range(2)]
    k, v = dense[0], dense[1].as_strided((1, N, Hkv, D), (8 * D * N * Hkv, Hkv * D if N > 1 else 48 * D, D if Hkv > 1 else 16 * D, 1))
    assert torch.equal(v, dense[1]) and v.stride() != k.stride()
    rope, slots = b.Rope(dev(frequencies(32))), torch.arange(N, dtype=torch.int32, device="cuda")[None]

    def bytes_of(v):
        c = b.KvqCache(2, 16, Hkv, D)
        c.data.fill_(0xAA)
        b.radar_kvq_append_rope(c, None, k, v, slots, rope)
        return c.data
    want = bytes_of(dense[1])
    got = []
    _Both(b, monkeypatch)("append", lambda: got.append(bytes_of(v)) or got[-1:])
    assert len(got) == 2 and all(torch.equal(x, want) for x in got)
