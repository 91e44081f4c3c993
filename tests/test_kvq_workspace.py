"""The workspace of attention over the paged 4-bit cache: the size asked for covers every smaller batch, tree and length (on the CPU)."""
import ctypes
import os
import random

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2512_14069_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build_library(force=False)
    return binding.load()


def attn_desc(B, T, S, Hq=32, H=8, D=128, R=16, split=0):
    from paper_2512_14069_amd import binding as b
    d = b.KvqAttnDesc()
    d.cache.n_blocks, d.cache.block_rows, d.cache.Hkv, d.cache.D, d.cache.layers = 1 << 20, R, H, D, 1
    d.B, d.T_max, d.Hq, d.max_blocks, d.S_max, d.rows_per_split = B, T, Hq, -(-S // R), S, split
    return d


def takes(lib, d, size):
    """Whether the call finds `size` enough (a workspace that is not aligned is refused after that)."""
    one, odd = ctypes.c_void_p(256), ctypes.c_void_p(260)
    rc = lib.radar_tree_attention_kvq(one, one, one, one, one, one, one, None, ctypes.byref(d), odd, size, None)
    assert rc in (-1, -3)
    return rc == -1


@pytest.mark.parametrize("Hq,H,D", [(32, 8, 128), (64, 8, 128), (4, 1, 64), (1, 1, 128), (16, 16, 64)])
def test_the_largest_shape_serves_smaller_ones(lib, Hq, H, D):
    rng = random.Random(Hq * 1000 + D)
    size = lambda d: lib.radar_tree_attention_kvq_workspace_bytes(ctypes.byref(d))                                              # noqa: E731
    for B, T, S in ((1, 1, 65536), (16, 60, 2100), (64, 1, 8192), (300, 64, 1 << 20), (2, 20, 60000)):
        most = size(attn_desc(B, T, S, Hq, H, D))
        lengths = [1, 31, 32, 2100, 40961, 64512] + [int(2 ** rng.uniform(0, 20)) for _ in range(200)]
        for n in lengths:
            if n > S:
                continue
            d = attn_desc(rng.choice([1, B, rng.randint(1, B)]), rng.choice([1, T, rng.randint(1, T)]), n, Hq, H, D, split=rng.choice([0, 0, 64, 4096]))
            assert 0 < size(d) <= most and takes(lib, d, most), (B, T, S, d.B, d.T_max, n)
            assert not takes(lib, d, size(d) - 1)
