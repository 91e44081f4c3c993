"""Inputs of the tests of the paged 4-bit cache."""
import numpy as np

from oracle import kvq
from paper_2512_14069_amd import synth


def bf16(x):
    """float -> the nearest bf16 values, as float64, and their bit patterns."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16()
    return t.double().numpy(), t.view(torch.int16).numpy().view(np.uint16)


def tables_for(rng, rows, R, spare=3, width=0):
    """Block tables [B,M] of sequences that hold so many rows each, from a pool in random order; its size."""
    need = [max(0, -(-n // R)) for n in rows]
    M = max(max(need), 1, width)
    n_blocks = sum(need) + spare
    ids = rng.permutation(n_blocks).astype(np.int32)
    table, at = np.full((len(rows), M), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, n_blocks


def random_cache(rng, layers, n_blocks, H, R, D):
    """Any codes, scales around one: bytes of rows N(0, about 1)."""
    c = rng.integers(0, 256, (layers, n_blocks, H, kvq.chunk_bytes(R, D)), dtype=np.uint8)
    c[..., R * D:] = rng.integers(124, 128, c[..., R * D:].shape, dtype=np.uint8)
    return c


def random_parents(rng, B, T, nodes):
    par = np.full((B, T), -1, np.int32)
    for b in range(B):
        for i in range(1, nodes[b]):
            par[b, i] = rng.integers(0, i)
    return par


def seed(n):
    return np.random.default_rng(synth.seed_for(91, n))
