"""What rotary positions, rotated rows into the paged 4-bit cache and attention of chunks refuse, on the CPU: status codes of the C calls,
exceptions of the binding, and the same under the sanitizers."""
import ctypes
import os

import pytest
import torch

import test_sanitizers
from test_kvq_refusals import BAD_CACHE, ONE, desc, lib  # noqa: F401

TWO, ODD = ctypes.c_void_p(512), ctypes.c_void_p(264)


def rope_desc(**kw):
    from paper_2512_14069_amd import binding as b
    d = b.RopeDesc()
    axis = kw.pop("pair_axis", [])
    for n, v in dict(dict(B=2, T_max=3, N=6, Hq=4, Hkv=2, D=128, axes=1), **kw).items():
        setattr(d, n, v)
    d.pair_axis[:len(axis)] = axis
    return ctypes.byref(d)


def rope_call(lib, ptr=None, at=None, starts=None, n_new=None, dd=None, **kw):  # noqa: F811
    args = [ONE, ONE, TWO, TWO, ONE, ONE, ONE, starts, n_new]
    if ptr is not None:
        args[ptr] = at
    return lib.radar_rope(*args, rope_desc(**kw) if dd is None else dd, None)


def append_call(lib, ptr=None, at=None, cache=None, **kw):  # noqa: F811
    args = [ONE, ONE, ONE, TWO, ONE, ONE, ONE, None, None, ONE, ONE]
    if ptr is not None:
        args[ptr] = at
    return lib.radar_kvq_append_rope(*args, rope_desc(**kw), ctypes.byref(cache or desc()), None)


BAD_ROWS = [(dict(B=0), -1), (dict(T_max=0), -1), (dict(N=5), -1), (dict(N=-1), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(rotary_dim=-16), -1), (dict(rotary_dim=144), -1),
            (dict(axes=0), -1), (dict(interleaved=2), -1), (dict(interleaved=-1), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
            (dict(pair_axis=[0, 1]), -1), (dict(axes=3, pair_axis=[0] * 63 + [3]), -1), (dict(q_stride_n=12), -1), (dict(q_stride_h=-8), -1), (dict(kv_stride_n=4), -1),
            (dict(q_out_stride_h=20), -1), (dict(axes=5), -2), (dict(rotary_dim=24), -2), (dict(Hq=70000), -2), (dict(B=1 << 16, T_max=1 << 15, N=1 << 31), -2),
            (dict(B=1 << 14, T_max=1 << 16, N=1 << 30), -2)]


@pytest.mark.parametrize("kw,want", BAD_ROWS)
def test_no_call_takes_impossible_rows(lib, kw, want):  # noqa: F811
    assert rope_call(lib, **kw) == want
    if "Hkv" not in kw:
        assert append_call(lib, **kw) == want


def test_rope(lib):  # noqa: F811
    assert rope_call(lib, 0) == rope_call(lib, 2) == rope_call(lib, 1) == rope_call(lib, 3) == rope_call(lib, 4) == -1      # an output without its input, and so on
    assert lib.radar_rope(None, None, None, None, ONE, ONE, ONE, None, None, rope_desc(), None) == -1
    assert lib.radar_rope(ONE, ONE, TWO, TWO, ONE, ONE, ONE, None, None, None, None) == -1
    for i in (0, 1, 2, 3):
        assert rope_call(lib, i, ODD) == -1
    assert rope_call(lib, D=100) == rope_call(lib, D=272) == -2 and rope_call(lib, D=0) == -1
    assert rope_call(lib, starts=ONE, n_new=ONE, N=4) == -1          # rows one behind the other have no counts
    assert rope_call(lib, 2, ONE, q_stride_n=512, q_out_stride_n=1024) == rope_call(lib, 3, ONE, k_out_stride_h=256) == -1      # in place, with other strides
    assert rope_call(lib, starts=ONE, N=0) == 0                      # nothing to do, nothing launched


@pytest.mark.parametrize("kw,want", BAD_CACHE)
def test_no_call_takes_an_impossible_cache(lib, kw, want):  # noqa: F811
    from paper_2512_14069_amd import binding as b
    c = desc(**kw)
    assert append_call(lib, cache=c, D=c.D, Hkv=c.Hkv) == want
    a = b.KvqChunkDesc()
    a.cache = c
    a.B = a.T_max = a.N = a.S_max = 1
    a.Hq, a.max_blocks = 2, 4
    assert lib.radar_chunk_attention_kvq(ONE, ONE, ONE, ONE, None, None, TWO, None, ctypes.byref(a), ONE, 1 << 40, None) == want
    assert lib.radar_chunk_attention_kvq_workspace_bytes(ctypes.byref(a)) == 0


def test_append(lib):  # noqa: F811
    for i in (0, 1, 2, 3, 4, 9, 10):                                 # q without q_out, and what may not be left out
        assert append_call(lib, i) == -1
    for i in (0, 1, 2, 3, 10):
        assert append_call(lib, i, ODD) == -1
    assert append_call(lib, D=64) == append_call(lib, Hkv=3) == -1   # another cache's
    assert lib.radar_kvq_append_rope(*([ONE] * 3), TWO, *([ONE] * 3), None, None, ONE, ONE, None, ctypes.byref(desc()), None) == -1
    assert lib.radar_kvq_append_rope(*([ONE] * 3), TWO, *([ONE] * 3), None, None, ONE, ONE, rope_desc(), None, None) == -1


def test_chunk_attention(lib):  # noqa: F811
    from paper_2512_14069_amd import binding as b

    def call(ptr=None, at=None, ws=1 << 40, ws_at=ONE, starts=None, n_new=None, **kw):
        a = b.KvqChunkDesc()
        a.cache = desc()
        for n, v in dict(dict(B=2, T_max=4, N=8, Hq=4, max_blocks=4, S_max=64), **kw).items():
            setattr(a, n, v)
        args = [ONE, ONE, ONE, ONE, starts, n_new, TWO, None]
        if ptr is not None:
            args[ptr] = at
        return lib.radar_chunk_attention_kvq(*args, ctypes.byref(a), ws_at, ws, None)
    for i in (0, 1, 2, 3, 6):
        assert call(i) == -1
    for i in (0, 1, 6):
        assert call(i, ODD) == -1
    assert call(6, ONE) == -1                                        # over its own queries
    assert call(ws_at=None) == call(ws_at=ctypes.c_void_p(260)) == -1 and call(ws=255) == -3
    assert lib.radar_chunk_attention_kvq(ONE, ONE, ONE, ONE, None, None, TWO, None, None, ONE, 1 << 30, None) == -1
    assert call(B=0) == call(T_max=0) == call(N=-1) == call(N=7) == call(Hq=0) == call(Hq=3) == call(max_blocks=0) == call(S_max=0) == -1
    assert call(starts=ONE, n_new=ONE) == -1
    assert call(S_max=65) == call(rows_per_split=32) == call(rows_per_split=-64) == call(softmax_scale=-1.0) == call(softmax_scale=float("nan")) == -1
    assert call(q_stride_t=12) == call(out_stride_h=4) == call(q_stride_b=-8) == -1
    assert call(B=65536, N=4 * 65536) == call(Hq=65538) == call(starts=ONE, N=1 << 31) == -2
    assert call(starts=ONE, N=(1 << 27), Hq=4) == call(B=4, T_max=1 << 25, N=1 << 27) == -2      # more blocks of columns than a launch has
    assert call(starts=ONE, N=0) == 0


def test_one_workspace_serves_any_shape(lib):  # noqa: F811
    from paper_2512_14069_amd import binding as b
    sizes = set()
    for B, T, N, S in ((1, 1, 1, 64), (64, 1, 64, 1 << 20), (1, 1 << 20, 1 << 20, 1 << 20), (16, 2000, 30000, 1 << 16), (60000, 7, 70000, 1 << 10)):
        a = b.KvqChunkDesc()
        a.cache = desc(n_blocks=1 << 16)
        a.B, a.T_max, a.N, a.Hq, a.max_blocks, a.S_max = B, T, N, 4, 1 << 16, S
        sizes.add(b.radar_chunk_attention_kvq_workspace_bytes(a))
    assert len(sizes) == 1 and sizes.pop() % 256 == 0


def test_the_binding_raises():
    from paper_2512_14069_amd import binding as b
    cache = b.KvqCache(4, 16, 2, 128, device="cpu")
    inv = torch.ones(64)
    rope = b.Rope(inv)
    x = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)                                     # noqa: E731
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)                                      # noqa: E731
    q, k, s = x(2, 3, 4, 128), x(2, 3, 2, 128), i32(2, 3)
    for call in (lambda: b.radar_rope(q, k, rope), lambda: b.radar_kvq_append_rope(cache, q, k, k, s, rope), lambda: b.radar_chunk_attention_kvq(q, cache, i32(2, 4), i32(2))):
        with pytest.raises((ValueError, RuntimeError), match="GPU tensor|HIP|CUDA"):
            call()
    for bad in (lambda: b.Rope(torch.ones(0)), lambda: b.Rope(torch.ones(129)), lambda: b.Rope(torch.ones(2, 8)), lambda: b.Rope(inv, pair_axis=[0] * 63),
                lambda: b.Rope(inv, axes=2, pair_axis=[0] * 63 + [2]), lambda: b.Rope(inv, scale=0.0), lambda: b.Rope(inv, pair_axis=[-1] * 64),
                lambda: b.radar_rope(None, None, rope), lambda: b.radar_rope(q, x(2, 4, 2, 128), rope), lambda: b.radar_rope(q, x(2, 3, 2, 64), rope),
                lambda: b.radar_rope(q[..., :64], None, rope), lambda: b.radar_rope(q, None, rope, positions=i32(7)), lambda: b.radar_rope(q, None, rope, positions=i32(2, 6)),
                lambda: b.radar_rope(q, None, rope, ctx_lens=i32(3)), lambda: b.radar_rope(q, None, rope, n_new=i32(3)), lambda: b.radar_rope(q, None, rope, T_max=4),
                lambda: b.radar_rope(q, None, rope, row_starts=i32(3)), lambda: b.radar_rope(q[0], None, rope), lambda: b.radar_rope(q[0], None, rope, row_starts=i32(1)),
                lambda: b.radar_rope(q[0], None, rope, row_starts=i32(3), n_new=i32(2)), lambda: b.radar_rope(q, None, rope, q_out=k),
                lambda: b.radar_rope(q[:, :1].expand(2, 3, 4, 128), None, rope), lambda: b.radar_rope(q[:, :, :1].expand(2, 3, 4, 128), None, rope),
                lambda: b.radar_rope(x(2, 5, 4, 128)[:, :3], None, rope), lambda: b.radar_rope(x(2, 3, 128, 4).transpose(2, 3), None, rope),
                lambda: b.radar_kvq_append_rope(cache, q, k, k[:1], s, rope), lambda: b.radar_kvq_append_rope(cache, q, x(2, 3, 3, 128), x(2, 3, 3, 128), s, rope),
                lambda: b.radar_kvq_append_rope(cache, q, k, k, i32(6), rope), lambda: b.radar_kvq_append_rope(cache, q, k, k, i32(2, 4), rope),
                lambda: b.radar_kvq_append_rope(cache, q, k, k, i32(3, 3), rope), lambda: b.radar_kvq_append_rope(cache, q, k, k, s, rope, layer=1),
                lambda: b.radar_kvq_append_rope(cache, q[0], k[0], k[0], s, rope, row_starts=i32(4)),
                lambda: b.radar_chunk_attention_kvq(x(2, 3, 4, 64), cache, i32(2, 4), i32(2)), lambda: b.radar_chunk_attention_kvq(q, cache, i32(3, 4), i32(2)),
                lambda: b.radar_chunk_attention_kvq(q, cache, i32(2, 4), i32(3)), lambda: b.radar_chunk_attention_kvq(q, cache, i32(2, 4), i32(2), n_new=i32(3)),
                lambda: b.radar_chunk_attention_kvq(q[0], cache, i32(2, 4), i32(2)), lambda: b.radar_chunk_attention_kvq(q[0], cache, i32(2, 4), i32(2), row_starts=i32(2)),
                lambda: b.radar_chunk_attention_kvq(q, cache, i32(2, 4), i32(2), out=q[:, :2]), lambda: b.radar_chunk_attention_kvq(q, cache, i32(2, 4), i32(2), layer=3),
                lambda: b.radar_chunk_attention_kvq(q, cache, i32(2, 4), i32(2), lse_out=torch.zeros(2, 3)),
                lambda: b.radar_chunk_attention_kvq(q, cache, i32(2, 4), i32(2), out=x(2, 1, 4, 128).expand(2, 3, 4, 128))):
        with pytest.raises(ValueError):
            bad()
    empty = x(0, 4, 128)                                             # no rows: nothing to do
    assert b.radar_chunk_attention_kvq(empty, cache, i32(2, 4), i32(2), row_starts=i32(3)).shape == empty.shape
    assert b.radar_chunk_attention_kvq(empty, cache, i32(2, 4), i32(2), row_starts=i32(3), prepared=True)().shape == empty.shape


def test_the_native_half_returns_none(lib):  # noqa: F811
    """Whatever it cannot take: tensors that are not on a GPU, other objects, too few of them, sizes that are none."""
    from paper_2512_14069_amd import binding as b
    n, i32 = b._native, torch.zeros((2, 2), dtype=torch.int32)
    x, cache, rope = torch.zeros((1, 3, 2, 128), dtype=torch.bfloat16), torch.zeros((1, 4, 2, 16 * 136), dtype=torch.uint8), b.Rope(torch.ones(64))
    turn = list(rope._native(None, None, None, None, 0))
    calls = ((n.rope, turn + [x, x, x, x]), (n.kvq_append_rope, turn + [x, x, x, x, i32, cache, 16, 128, 0]),
             (n.chunk_attention_kvq, [x, cache, 16, 128, i32, i32, None, None, 0, 0, 0, None, None, i32, 0, 0.0]))
    for f, args in calls:
        assert f(*args) is None and f() is None
        for i in range(len(args)):
            assert f(*args[:i]) is None
            for other in (None, "no", b"", 1 << 70, -1, object(), x, i32):
                assert f(*args[:i], other, *args[i + 1:]) is None


FAKE = r"""
import sys
import warnings

import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2512_14069_amd import binding as b

warnings.simplefilter("ignore")
b.load()
n = b._native
with FakeTensorMode():                      # tensors that say they are on a GPU; there is none to allocate on or take a stream from
    i = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
    h = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    inv, cache = torch.empty(32, device="cuda"), torch.empty((1, 4, 2, 16 * 68), dtype=torch.uint8, device="cuda")
    turn = (inv, 2, bytes(32), 0, 1.0, i(2, 6), i(2), None, None, 0)
    packed = (inv, 1, bytes(32), 1, 0.5, i(6), i(2), i(3), None, 4)
    q, k, ends = h(2, 3, 4, 64), h(2, 3, 2, 64), (i(2, 3), cache, 16, 64, 0)
    calls = [(n.rope, turn + (q, k, h(2, 3, 4, 64), h(2, 3, 2, 64))), (n.rope, turn + (q, None, q, None)), (n.rope, packed + (h(6, 4, 64), h(6, 2, 64)) * 2),
             (n.kvq_append_rope, turn + (q, k, h(2, 3, 4, 64), k) + ends), (n.kvq_append_rope, turn + (None, k, None, k) + ends),
             (n.chunk_attention_kvq, (q, cache, 16, 64, i(2, 4), i(2), None, i(2), 0, 0, 0, None, None, None, 0, 0.0)),
             (n.chunk_attention_kvq, (h(6, 4, 64), cache, 16, 64, i(2, 4), i(2), i(3), None, 4, 0, 9, h(6, 4, 64), None, None, 0, 0.0))]
sparse = torch.sparse_coo_tensor(torch.zeros((1, 1), dtype=torch.long), torch.ones(1), (4,))
for f, args in calls:
    print(f.__name__, flush=True)
    assert f(*args) is None
    for at in range(len(args)):
        for other in (None, "text", torch.zeros(1), torch.zeros(2, dtype=torch.int8), sparse, 1 << 40, b"12"):
            assert f(*args[:at], other, *args[at + 1:]) is None
print("done")
"""


def test_nothing_leaves_the_native_half_but_none(lib):  # noqa: F811
    """In a process of its own: a C++ exception of torch's that escaped would end it."""
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-W", "ignore", "-c", FAKE], cwd=root, env=dict(os.environ, HIP_VISIBLE_DEVICES="-1", PYTHONPATH=root), capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("done"), (r.returncode, r.stdout[-500:], r.stderr[-2000:])


def test_under_sanitizers():
    if os.environ.get("RADAR_LIB_SANITIZE") == "1":
        pytest.skip("this is the sanitized run")
    from paper_2512_14069_amd import build
    build.build_library(force=False, sanitize=True)
    out = test_sanitizers.run_child([os.path.abspath(__file__)], {"RADAR_LIB_SANITIZE": "1"}, build.sanitizer_runtime())
    assert " passed" in out
