"""Keys and values with the same layout whose strides differ where an axis has one entry only: the binding takes them, on the CPU as far as its checks go."""
import pytest
import torch


def layouts():
    x = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)                                     # noqa: E731
    tokens, one = x(1, 9, 2, 64), x(1, 1, 2, 64)
    yield one, tokens[:, -1:], dict()                                # a single token: the last of nine, and one alone
    yield x(3, 3, 2, 64)[:1], x(1, 3, 2, 64).as_strided((1, 3, 2, 64), (64, 128, 64, 1)), dict()      # one sequence
    yield x(4, 1, 64), x(4, 1, 64).as_strided((4, 1, 64), (64, 4096, 1)), dict(row_starts=torch.zeros(2, dtype=torch.int32))      # one head, rows one behind the other


@pytest.mark.parametrize("case", range(3))
def test_strides_of_one_entry_say_nothing(case):
    from paper_2512_14069_amd import binding as b
    k, v, rows = list(layouts())[case]
    assert k.stride() != v.stride()
    cache = b.KvqCache(4, 16, k.shape[-2], 64, device="cpu")
    slots = torch.zeros((1, k.shape[0] if rows else k.shape[1]), dtype=torch.int32)
    with pytest.raises((ValueError, RuntimeError), match="GPU tensor|HIP|CUDA"):                    # all that is wrong with them
        b.radar_kvq_append_rope(cache, None, k, v, slots, b.Rope(torch.ones(32)), **rows)


def test_strides_that_differ_are_refused():
    from paper_2512_14069_amd import binding as b
    x = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)                                     # noqa: E731
    cache, slots, rope = b.KvqCache(4, 16, 2, 64, device="cpu"), torch.zeros((2, 3), dtype=torch.int32), b.Rope(torch.ones(32))
    k = x(2, 3, 2, 64)
    for v in (x(2, 3, 4, 64)[:, :, :2], x(2, 3, 2, 128)[..., :64], x(2, 2, 3, 64).transpose(1, 2), x(2, 6, 2, 64)[:, ::2], x(2, 3, 2, 128)[..., ::2], x(2, 1, 2, 64).expand(2, 3, 2, 64)):
        assert v.shape == k.shape
        with pytest.raises(ValueError):
            b.radar_kvq_append_rope(cache, None, k, v, slots, rope)
