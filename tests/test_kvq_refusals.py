"""What the paged 4-bit cache's entry points refuse, on the CPU: status codes of the C calls, exceptions of the binding, and the
same under the sanitizers."""
import ctypes
import os

import pytest
import torch

import test_sanitizers


@pytest.fixture(scope="module")
def lib():
    from paper_2512_14069_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build_library(force=False)
    return binding.load()


ONE = ctypes.c_void_p(256)                                          # never dereferenced: every case is rejected first


def desc(**kw):
    from paper_2512_14069_amd import binding as b
    d = b.KvqDesc()
    for n, v in dict(dict(n_blocks=8, block_rows=16, Hkv=2, D=128, layers=2, layer_stride=0), **kw).items():
        setattr(d, n, v)
    return d


BAD_CACHE = [(dict(n_blocks=0), -1), (dict(Hkv=0), -1), (dict(D=96), -2), (dict(D=256), -2), (dict(block_rows=0), -1), (dict(block_rows=8), -2),
             (dict(block_rows=48), -2), (dict(block_rows=256), -2), (dict(Hkv=70000), -2), (dict(n_blocks=1 << 28), -2)]


def test_block_bytes(lib):
    from paper_2512_14069_amd import binding as b
    assert b.radar_kvq_block_bytes(16, 128) == 16 * 136 and b.radar_kvq_block_bytes(128, 64) == 128 * 68
    assert [b.radar_kvq_block_bytes(*x) for x in ((8, 128), (16, 32), (0, 64), (-16, 64), (24, 64))] == [0] * 5


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_no_call_takes_an_impossible_cache(lib, kw, want):
    from paper_2512_14069_amd import binding as b
    d = ctypes.byref(desc(**kw))
    assert lib.radar_kvq_append(ONE, ONE, ONE, ONE, 1, 0, 0, d, None) == want
    assert lib.radar_kvq_read(ONE, ONE, ONE, ONE, 1, d, None) == want
    assert lib.radar_kvq_commit(ONE, ONE, 4, ONE, ONE, ONE, 9, 1, None, d, None) == want
    a = b.KvqAttnDesc()
    a.cache = desc(**kw)
    a.B = a.T_max = a.S_max = 1
    a.Hq, a.max_blocks = 2, 4
    assert lib.radar_tree_attention_kvq(ONE, ONE, ONE, ONE, ONE, None, ONE, None, ctypes.byref(a), ONE, 1 << 30, None) == want
    assert lib.radar_tree_attention_kvq_workspace_bytes(ctypes.byref(a)) == 0


def test_rows(lib):
    d, odd = ctypes.byref(desc()), ctypes.c_void_p(264)
    append = lambda k=ONE, v=ONE, s=ONE, c=ONE, N=1, sn=0, sh=0, dd=d: lib.radar_kvq_append(k, v, s, c, N, sn, sh, dd, None)   # noqa: E731
    assert append(k=None) == append(v=None) == append(s=None) == append(c=None) == append(dd=None) == -1
    assert append(k=odd) == append(v=odd) == append(c=odd) == append(N=-1) == append(sn=12) == append(sh=-8) == append(sn=-128) == -1
    assert append(N=1 << 31) == append(N=1 << 26) == -2              # more lanes than a launch has
    assert append(N=0) == 0                                          # nothing to do, nothing launched
    read = lambda c=ONE, s=ONE, k=ONE, v=ONE, N=1, dd=d: lib.radar_kvq_read(c, s, k, v, N, dd, None)                             # noqa: E731
    assert read(c=None) == read(s=None) == read(k=None) == read(v=None) == read(dd=None) == read(k=odd) == read(N=-2) == -1
    assert read(dd=ctypes.byref(desc(layers=0))) == read(dd=ctypes.byref(desc(layer_stride=24))) == read(dd=ctypes.byref(desc(layer_stride=-16))) == -1
    assert read(dd=ctypes.byref(desc(layers=65536))) == -2
    assert read(N=0) == 0


def test_layers_do_not_share_memory(lib):
    from paper_2512_14069_amd import binding as b
    layer = 8 * 2 * 16 * 136
    for stride, layers, want in ((layer - 16, 2, -1), (16, 3, -1), (layer, 2, 0), (16, 1, 0)):
        assert lib.radar_kvq_read(ONE, ONE, ONE, ONE, 0, ctypes.byref(desc(layers=layers, layer_stride=stride)), None) == want
    assert lib.radar_kvq_commit(ONE, ONE, 4, ONE, ONE, ONE, 9, 1, None, ctypes.byref(desc(layer_stride=layer - 16)), None) == -1
    one = torch.zeros((1, 8, 2, 16 * 136), dtype=torch.uint8)
    with pytest.raises(ValueError, match="layers 0 bytes apart"):
        b.KvqCache(data=one.expand(3, -1, -1, -1))
    wide = torch.zeros((3, layer + 8), dtype=torch.uint8)[:, :layer].view(3, 8, 2, 16 * 136)
    with pytest.raises(ValueError, match="multiple of 16"):
        b.KvqCache(data=wide)
    assert b.KvqCache(data=torch.zeros((3, layer + 32), dtype=torch.uint8)[:, :layer].view(3, 8, 2, 16 * 136)).desc().layer_stride == layer + 32


def test_commit(lib):
    d, two = ctypes.byref(desc()), ctypes.c_void_p(512)
    commit = lambda c=ONE, t=ONE, M=4, ctx=ONE, n=ONE, p=ONE, P=9, B=1, out=two, dd=d: lib.radar_kvq_commit(c, t, M, ctx, n, p, P, B, out, dd, None)  # noqa: E731
    assert commit(c=None) == commit(t=None) == commit(ctx=None) == commit(n=None) == commit(p=None) == commit(dd=None) == -1
    assert commit(out=ONE) == -1                                     # the new lengths are not written over the old ones
    assert commit(M=0) == commit(P=0) == commit(B=0) == commit(c=ctypes.c_void_p(260)) == -1
    assert commit(P=65) == commit(B=65536) == -2
    assert commit(dd=ctypes.byref(desc(layers=0))) == commit(dd=ctypes.byref(desc(layer_stride=8))) == -1
    assert commit(dd=ctypes.byref(desc(layers=1 << 17, Hkv=65535))) == -2


def test_blocks(lib):
    from paper_2512_14069_amd import binding as b

    def call(null=None, **kw):
        d = b.KvqBlocksDesc()
        for n, v in dict(dict(B=2, T_max=8, max_blocks=4, n_blocks=9, block_rows=16), **kw).items():
            setattr(d, n, v)
        args = [ONE] * 10
        if null is not None:
            args[null] = None
        return lib.radar_kvq_blocks(*args, ctypes.byref(d), None)
    for i in (0, 2, 3, 4, 5, 6, 7, 8, 9):                            # n_new may be left out
        assert call(null=i) == -1
    assert lib.radar_kvq_blocks(*([ONE] * 10), None, None) == -1
    assert call(B=0) == call(T_max=0) == call(max_blocks=0) == call(n_blocks=0) == call(block_rows=0) == -1
    assert call(block_rows=17) == call(n_blocks=1 << 28) == call(B=1 << 16, max_blocks=1 << 16) == call(B=1 << 16, T_max=1 << 16) == -2


def test_attention(lib):
    from paper_2512_14069_amd import binding as b

    def call(ptr=None, at=None, ws=1 << 40, ws_at=ONE, **kw):
        a = b.KvqAttnDesc()
        a.cache = desc()
        for n, v in dict(dict(B=2, T_max=4, Hq=4, max_blocks=4, S_max=64), **kw).items():
            setattr(a, n, v)
        args = [ONE] * 8
        if ptr is not None:
            args[ptr] = at
        return lib.radar_tree_attention_kvq(*args, ctypes.byref(a), ws_at, ws, None)
    for i in (0, 1, 2, 4, 6):                                        # parents, n_nodes and lse_out may be left out
        assert call(i) == -1
    for i in (0, 1, 6):
        assert call(i, ctypes.c_void_p(264)) == -1
    assert call(ws_at=None) == call(ws_at=ctypes.c_void_p(260)) == -1 and call(ws=255) == -3
    assert lib.radar_tree_attention_kvq(*([ONE] * 8), None, ONE, 1 << 30, None) == -1
    assert call(B=0) == call(T_max=0) == call(Hq=0) == call(Hq=3) == call(max_blocks=0) == call(S_max=0) == -1
    assert call(S_max=65) == call(rows_per_split=32) == call(rows_per_split=-64) == call(softmax_scale=-1.0) == call(softmax_scale=float("nan")) == -1
    assert call(q_stride_t=12) == call(out_stride_h=4) == call(q_stride_b=-8) == -1
    assert call(T_max=65) == call(B=65536) == call(Hq=65538) == call(B=65535, T_max=64, Hq=64) == -2


def test_the_binding_raises():
    from paper_2512_14069_amd import binding as b
    cache = b.KvqCache(4, 16, 2, 128, device="cpu")
    assert tuple(cache.data.shape) == (1, 4, 2, 16 * 136)
    k, s = torch.zeros((3, 2, 128), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)                                                                  # noqa: E731
    with pytest.raises(ValueError, match="GPU tensor"):
        b.radar_kvq_append(cache, k, k, s)
    for bad in (lambda: b.KvqCache(4, 24, 2, 128, device="cpu"), lambda: b.KvqCache(4, 16, 2, 96, device="cpu"),
                lambda: b.KvqCache(data=torch.zeros((1, 4, 2, 100), dtype=torch.uint8)),
                lambda: b.KvqCache(data=torch.zeros((1, 4, 2176, 2), dtype=torch.uint8).transpose(2, 3)),
                lambda: b.radar_kvq_append(cache, k, k[:2], s), lambda: b.radar_kvq_append(cache, k, k, s[:2]),
                lambda: b.radar_kvq_append(cache, k.transpose(0, 1).contiguous().transpose(0, 1), k, s),
                lambda: b.radar_kvq_append(cache, k, k, s, layer=1), lambda: b.radar_kvq_append(cache, k, k, s, layer=-1),
                lambda: b.radar_kvq_append(cache, k[:1].expand(3, 2, 128), k[:1].expand(3, 2, 128), s),
                lambda: b.radar_kvq_append(cache, k[:, :1].expand(3, 2, 128), k[:, :1].expand(3, 2, 128), s),
                lambda: b.radar_kvq_read(cache, s, layer=3), lambda: b.radar_kvq_read(cache, s, k=k),
                lambda: b.radar_kvq_commit(cache, i32(2, 3), i32(3), i32(2), i32(2, 9)),
                lambda: b.radar_kvq_commit(cache, i32(2, 3), i32(2), i32(2), i32(3, 9)),
                lambda: b.radar_kvq_commit(cache, i32(2, 3), i32(2), i32(2), i32(9)),
                lambda: b.radar_tree_attention_kvq(torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16), cache, i32(1, 2), i32(1)),
                lambda: b.radar_tree_attention_kvq(torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16), cache, i32(2, 2), i32(1)),
                lambda: b.radar_tree_attention_kvq(torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16), cache, i32(1, 2), i32(2)),
                lambda: b.radar_tree_attention_kvq(torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16), cache, i32(1, 2), i32(1), parents=i32(2, 1)),
                lambda: b.radar_tree_attention_kvq(torch.zeros((1, 1, 4, 128), dtype=torch.bfloat16).expand(3, 2, 4, 128), cache, i32(3, 2), i32(3)),
                lambda: b.radar_tree_attention_kvq(torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16), cache, i32(1, 2), i32(1),
                                                   out=torch.zeros((1, 2, 1, 128), dtype=torch.bfloat16).expand(1, 2, 4, 128)),
                lambda: b.radar_kvq_blocks(i32(3), b.KvqTables(2, 4, 9, device="cpu"), 8),
                lambda: b.radar_kvq_blocks(i32(2), b.KvqTables(2, 4, 9, device="cpu"), 8, slots=i32(2, 7)),
                lambda: b.radar_kvq_blocks(i32(2), b.KvqTables(2, 4, 9, device="cpu"), 8, n_new=i32(1))):
        with pytest.raises(ValueError):
            bad()
    gap = torch.zeros((2, 5, 2, 128), dtype=torch.bfloat16)[:, :3]   # rows of two blocks, not evenly spaced
    with pytest.raises(ValueError, match="evenly"):
        b.radar_kvq_append(cache, gap, gap, torch.zeros(6, dtype=torch.int32))
    assert b._rows_stride(torch.zeros((2, 3, 9, 2, 128))[:, :, 4], "k") == 9 * 256
    t = b.KvqTables(2, 4, 9, device="cpu")
    assert t.free_blocks.tolist() == list(range(8, -1, -1)) and t.n_free.tolist() == [9] and (t.block_tables == -1).all()


def test_the_native_half_returns_none(lib):
    """Whatever it cannot take: tensors that are not on a GPU, other objects, too few of them, sizes that are none."""
    from paper_2512_14069_amd import binding as b
    n, i32 = b._native, torch.zeros((2, 2), dtype=torch.int32)
    cache, x = torch.zeros((1, 4, 2, 16 * 136), dtype=torch.uint8), torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    calls = ((n.kvq_blocks, [i32] * 10 + [8, 16]), (n.kvq_append, [cache, 16, 128, x, x, i32, 0]), (n.kvq_commit, [cache, 16, 128] + [i32] * 5),
             (n.tree_attention_kvq, [x, cache, 16, 128, i32, i32, None, None, 0, 0, None, None, i32, 0, 0.0]))
    for f, args in calls:
        assert f(*args) is None and f() is None
        for i in range(len(args)):
            assert f(*args[:i]) is None
            for other in (None, "no", 1 << 70, -1, object(), x, i32):
                assert f(*args[:i], other, *args[i + 1:]) is None


def test_under_sanitizers():
    if os.environ.get("RADAR_LIB_SANITIZE") == "1":
        pytest.skip("this is the sanitized run")
    from paper_2512_14069_amd import build
    build.build_library(force=False, sanitize=True)
    out = test_sanitizers.run_child([os.path.abspath(__file__)], {"RADAR_LIB_SANITIZE": "1"}, build.sanitizer_runtime())
    assert " passed" in out
