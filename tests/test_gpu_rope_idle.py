"""Rows one behind the other in batches most of whose sequences have none: long stretches of starts that repeat between two rows of a workgroup."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_bits, bf16_dev, dev, host
from kvq_util import bf16, seed
from oracle import kvq
from test_gpu_kvq import binding
from test_gpu_rope import frequencies, turned

pytestmark = pytest.mark.gpu
D, P = 64, 32


def batch(rng, B, at, new):
    counts = np.zeros(B, np.int64)
    counts[at] = new
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    return starts, rng.integers(0, 5000, B).astype(np.int32), bf16(rng.normal(size=(int(starts[-1]), 3, D)))


@pytest.mark.parametrize("B,at,new", [(64, [0, 63], [1, 1]), (65, [0, 63, 64], [1, 1, 1]), (66, [1, 64, 65], [2, 1, 3]), (129, [0, 62, 63, 64, 126, 127, 128], [1] * 7), (200, [199], [5]),
                                      (700, [3, 66, 67, 68, 131, 650, 699], [1, 1, 1, 2, 1, 1, 2]), (9000, [0, 5, 100, 1000, 4000, 8000, 8998, 8999], [1] * 8),
                                      (9001, [0, 4500, 9000], [9, 6, 7]), (100000, [2, 70, 50000, 50100, 99999], [1, 2, 1, 2, 4]), (640, list(range(0, 640, 64)), [1] * 10)])
def test_a_rows_sequence_is_found_wherever_it_lies(B, at, new):
    b, rng = binding(), seed(970 + B)
    starts, ctx, (x, bits) = batch(rng, B, at, new)
    ctx[at[-1]] = -1 if len(at) > 1 and B % 2 else ctx[at[-1]]
    T = max(new)
    rope = b.Rope(dev(frequencies(P)))
    fresh = lambda h: torch.full((len(x), h, D), 3.0, dtype=torch.bfloat16, device="cuda")           # noqa: E731
    q, k, v = (bf16_dev(bits[:, h:h + 1]) for h in range(3))
    got, _ = b.radar_rope(q, None, rope, ctx_lens=dev(ctx), row_starts=dev(starts), T_max=T, q_out=fresh(1))
    rows = kvq.new_rows(B, T, ctx, starts)
    want = turned(np.full_like(bits, 0x4040), x, rows, None, ctx, frequencies(P), [0] * P, False, 1.0)
    assert np.array_equal(bf16_bits(got), want[:, :1])
    # and into the cache, whose slots go by the sequence too
    cache, R = np.full((1, 8, 1, kvq.chunk_bytes(16, D)), 0xAA, np.uint8), 16
    c = b.KvqCache(8, R, 1, D)
    c.data.copy_(dev(cache))
    slots, wide = np.full((B, T), -1, np.int32), lambda p: torch.from_numpy(p.view(np.int16)).view(torch.bfloat16).double().numpy()      # noqa: E731
    for place, (n, s, i) in enumerate(rows):
        slots[s, i] = (place * 7 + 3) % 128
        kvq.put(cache, R, D, 0, int(slots[s, i]), wide(want[n, 1:2].copy()), x[n, 2:])
    turned_q = b.radar_kvq_append_rope(c, q, k, v, dev(slots), rope, ctx_lens=dev(ctx), row_starts=dev(starts), q_out=fresh(1))
    assert torch.equal(turned_q, got) and np.array_equal(host(c.data), cache)


def test_idle_sequences_take_no_time_of_their_own():
    """Rows that lie 200000 sequences apart, and the same rows side by side.  A walk from one to the other, a load behind a load, would take 16 ms (80 ns a sequence); a search takes as
    many round trips as there are digits (ten microseconds or so)."""
    b, rng, B = binding(), seed(990), 200000
    rope, times = b.Rope(dev(frequencies(P))), []
    for at in ([0, 1, 2, 3], [0, 1, B - 2, B - 1]):
        starts, ctx, (_, bits) = batch(rng, B, at, [1, 1, 1, 1])
        q, dc, ds = bf16_dev(bits), dev(ctx), dev(starts)
        out = torch.empty_like(q)
        best = np.inf
        for _ in range(4):
            one, two = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            one.record()
            b.radar_rope(q, None, rope, ctx_lens=dc, row_starts=ds, T_max=1, q_out=out)
            two.record()
            two.synchronize()
            best = min(best, one.elapsed_time(two))
        times.append(best)
    assert times[1] < times[0] + 2.0, times                          # ms
