"""Attention over the paged 4-bit cache where several workgroups have parts of a unit and the last to arrive joins them: every number of parts that
calls are divided into, with the path that was taken read off the launches and the partial results."""
import numpy as np
import pytest
import torch

from gpu_util import bf16_dev, dev, host
from kvq_util import bf16, random_parents, seed
from test_gpu_kvq import binding, check_attention, gpu_cache, make_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,T,Hq,H,S,columns,joined", [
    (1, 1, 32, 8, 65536, 16, 32), (4, 1, 1, 1, 32768, 16, 32), (1, 1, 4, 1, 16384, 16, 16), (1, 20, 32, 8, 16384, 32, 8),
    (1, 60, 16, 2, 131072, 64, 16), (1, 20, 16, 8, 786432, 64, 32), (1, 20, 8, 4, 3 << 20, 64, 64)])
def test_parts_are_joined(B, T, Hq, H, S, columns, joined, D):
    """Planned for S rows; contexts that give every workgroup a step, that leave some without, that are one step long, and none."""
    b, rng, R = binding(), seed(400 + T + D + joined), 16
    tables, cache, _, _, _ = make_attention(rng, np.full(B, 2100), T, np.full(B, T), Hq, H, D, R)
    c = gpu_cache(cache, R, D)
    wide = np.full((B, S // R), -1, np.int32)
    wide[:, :tables.shape[1]] = tables
    wide, ws, units_of_one = dev(wide), None, -(-Hq // H * T // columns)
    units, slot = B * H * units_of_one, columns * (D + 2) * 4
    first = 16384 + -(-4 * B * H * -(-Hq // H * T // 16) // 256) * 256                              # counters, then a word for each unit of 16 columns
    for rows in (2100, 700, 20, 0, -1):
        ctx, nodes = np.full(B, rows, np.int32), np.full(B, T, np.int32)
        if B > 1:
            ctx[1:3] = [max(rows - 333, -1), -1]
        q, qb = bf16(rng.normal(size=(B, T, Hq, D)))
        par = random_parents(rng, B, T, nodes)
        if ws is None:
            ws = b.new_workspace(b.radar_tree_attention_kvq_workspace_bytes(b.kvq_attn_desc(bf16_dev(qb), c, wide.shape[1], S)))
        ws[first:] = 0xA5
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device="cuda")
        b.radar_profile_begin(8)
        b.radar_tree_attention_kvq(bf16_dev(qb), c, wide, dev(ctx), dev(par), dev(nodes), out=out, lse_out=lse, S_max=S, workspace=ws)
        launches = {name: v["calls"] for name, v in b.radar_profile_end().items()}
        assert launches == {"kvq_attention": 1}
        check_attention(q, cache, R, D, 0, tables, ctx, par, nodes, out, lse)
        assert (ws[:16384] == 0).all()
        written = (host(ws[first:first + units * joined * slot]).reshape(units, joined, slot) != 0xA5).any(-1)
        assert (host(ws[first + units * joined * slot:]) == 0xA5).all()
        for u in range(units):
            steps = -(-(ctx[u // (H * units_of_one)] + T) // 32) if ctx[u // (H * units_of_one)] >= 0 else 0
            parts = -(-steps // -(-steps // joined)) if steps else 0
            assert written[u].tolist() == [parts > 1 and x < parts for x in range(joined)]
