"""What the calls on bounds, selections and lists hand to the library, and what they and the library refuse,
without a GPU."""
import ctypes as C
import os

import pytest
import torch

D = 128
BF = torch.bfloat16


@pytest.fixture(scope="module")
def package():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2609_25782_gb300
    return paper_2609_25782_gb300


def make_pool(package, native, hq=8, hkv=2, layers=3, blocks=5):
    """A pool without arenas or a handle, and library calls that only note their arguments. native: through the module
    in C, to functions that note theirs as well."""
    p = package.Pool.__new__(package.Pool)
    p.device, p.handle, p.Hq, p.Hkv, p.D, p.L, p.bt, p.num_hot_blocks = torch.device("cpu"), None, hq, hkv, D, layers, 16, blocks
    p._bf16, p._i32, p._f32 = BF, torch.int32, torch.float32
    p._out_flags = {torch.float32: 0, BF: package.kvtier.KV_DECODE_OUT_BF16}
    p._index = -1
    p.bounds_bytes = layers * hkv * blocks * (2 * D + 2)
    p.calls = []
    p._select = p._sparse = lambda *a: p.calls.append(a) or 0
    p._calls, p.native = None, 0
    if native:
        if package.kvtier._calls is None:
            pytest.skip("built without Python's headers")
        i32, i64, ptr = C.c_int32, C.c_int64, C.c_void_p

        def note(*a):
            p.native += 1
            return p.calls.append(a) or 0
        select = C.CFUNCTYPE(C.c_int, ptr, i32, ptr, i64, ptr, ptr, ptr, i32, i32, i32, i32, i32, ptr, ptr, ptr)(note)
        sparse = C.CFUNCTYPE(C.c_int, ptr, i32, ptr, i64, ptr, ptr, i64, ptr, i32, ptr, ptr, i32, i32, C.c_float, ptr,
                             C.c_uint32, ptr)(note)
        p.keep = select, sparse
        p._calls = package.kvtier._calls.Calls(77, -1, hq, hkv, p.bounds_bytes, BF, torch.int32, torch.float32,
                                               *map(package.kvtier.address, p.keep))
    return p


@pytest.mark.parametrize("cc", [None, "", "gcc", "env gcc -g", "env 'CCACHE_DIR=/a b' gcc"])
def test_the_module_is_built_by_any_compiler_command(package, monkeypatch, tmp_path, cc):
    """CC as make and others take it, words and quotes; the file is named for this Python."""
    import importlib.machinery
    import subprocess

    from paper_2609_25782_gb300 import _build
    if not os.path.exists(_build.PYTHON_H):
        pytest.skip("built without Python's headers")
    monkeypatch.delenv("CC", raising=False)
    if cc is not None:
        monkeypatch.setenv("CC", cc)
    subprocess.run(_build.calls_command(str(tmp_path / "calls.so")), check=True)
    assert (tmp_path / "calls.so").exists()
    tagged = importlib.machinery.EXTENSION_SUFFIXES[0]
    assert _build.CALLS.endswith("_calls" + tagged) and package.kvtier._calls.__file__.endswith("_calls" + tagged)


BOTH = pytest.mark.parametrize("native", [False, True])


def arguments(pool, B=3, top=4, **other):
    a = dict(q=torch.zeros(B, pool.Hq, D, dtype=BF), k=torch.zeros(B, pool.Hkv, D, dtype=BF),
             v=torch.zeros(B, pool.Hkv, D, dtype=BF), tables=torch.zeros(B, 6, dtype=torch.int32),
             lens=torch.zeros(B, dtype=torch.int32), B=B, width=6,
             selected=torch.zeros(B, pool.Hkv, top, dtype=torch.int32), out=torch.zeros(B, pool.Hq, D),
             scores=torch.zeros(B, pool.Hkv, 6), bounds=torch.zeros(pool.bounds_bytes, dtype=torch.int8), stream=None)
    a.update(other)
    return a


def select(pool, **other):
    a = arguments(pool, **other)
    pool.calls.clear()
    pool.select_blocks(1, a["q"], a["bounds"], a["tables"], a["lens"], a["B"], a["width"], a["selected"], 1, 2,
                       a["scores"], a["stream"])
    return pool.calls[0]


def attend(pool, **other):
    a = arguments(pool, **other)
    pool.calls.clear()
    pool.sparse_attention(1, a["q"], a["selected"], a["tables"], a["lens"], a["B"], a["width"], 0.5, a["out"], a["k"],
                          a["v"], a["stream"])
    return pool.calls[0]


def refused(pool, f, **other):
    pool.calls.clear()
    with pytest.raises(ValueError):
        f(pool, **other)
    assert not pool.calls, other


@BOTH
def test_strides_and_shapes_reach_the_library(package, native):
    pool = make_pool(package, native)
    qkv = torch.zeros(3, 12, D, dtype=BF)
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    got = select(pool, q=q)
    assert got[2:4] == (q.data_ptr(), 12 * D) and got[7:12] == (3, 6, 1, 2, 4)
    assert select(pool, scores=None)[13] is None
    got = attend(pool, q=q, k=k, v=v)
    assert got[2:7] == (q.data_ptr(), 12 * D, k.data_ptr(), v.data_ptr(), 12 * D) and got[8] == 4 and got[15] == 0
    assert attend(pool, out=torch.zeros(3, 8, D, dtype=BF))[15] == package.kvtier.KV_DECODE_OUT_BF16
    assert attend(pool, k=None, v=None)[4:7] == (None, None, 0)
    # a single row's stride means nothing
    one = torch.zeros(1, 8, D, dtype=BF).expand(4, 8, D)[:1]
    assert attend(pool, B=1, q=one)[3] == 0
    for stream, handle in ((None, None), (1234, 1234), (0, 0)):
        assert (select(pool, stream=stream)[-1] or 0) == (attend(pool, stream=stream)[-1] or 0) == (handle or 0)
    assert pool.native == (12 if native else 0)


@BOTH
@pytest.mark.parametrize("error", [KeyboardInterrupt, SystemExit, MemoryError])
def test_an_interrupt_during_the_checks_is_not_lost(package, native, error):
    """It comes up once, where a tensor is asked for something; an error of another kind is the checks' own to find."""
    pool = make_pool(package, native)

    class Once(torch.Tensor):
        left = 0

        @property
        def dtype(self):
            if Once.left:
                Once.left -= 1
                raise Once.error("once")
            return super().dtype
    a = arguments(pool)
    for f, names in ((select, ("q", "tables", "lens", "selected", "scores")), (attend, ("q", "k", "v", "tables", "lens", "selected", "out"))):
        for name in names:
            x = a[name].as_subclass(Once)
            Once.left, Once.error = 1, error
            pool.calls.clear()
            with pytest.raises(error):
                f(pool, **dict(a, **{name: x}))
            assert not pool.calls and not Once.left, name
            if native:
                Once.left, Once.error = 1, TypeError     # (without the module the checks pass it on)
                assert f(pool, **dict(a, **{name: x}))[1:] == f(pool, **a)[1:] and not Once.left


@BOTH
def test_numpy_numbers_are_numbers(package, native):
    """The module in C leaves them to the checks in Python; the library gets the same numbers."""
    import numpy as np
    pool = make_pool(package, native)
    a = arguments(pool)
    for kind in (np.int64, np.int32):
        pool.native = 0
        for f in (select, attend):
            assert f(pool, **dict(a, B=kind(3), width=kind(6)))[1:] == f(pool, **a)[1:]
        pool.calls.clear()
        pool.select_blocks(kind(1), a["q"], a["bounds"], a["tables"], a["lens"], kind(3), 6, a["selected"], kind(1), kind(2), a["scores"])
        assert pool.calls[0][1:] == select(pool, **a)[1:]
        pool.calls.clear()
        pool.sparse_attention(kind(1), a["q"], a["selected"], a["tables"], a["lens"], 3, kind(6), np.float32(0.5), a["out"], a["k"], a["v"])
        assert pool.calls[0][1:] == attend(pool, **a)[1:]
        assert pool.native == (4 if native else 0)       # the plain calls
        refused(pool, select, **dict(a, B=kind(2)))
        refused(pool, attend, **dict(a, width=kind(7)))


@BOTH
def test_tensors_that_the_library_would_misread(package, native):
    pool = make_pool(package, native)
    i32 = torch.int32
    wide = torch.zeros(3, 16, 2 * D, dtype=BF)
    for f in (select, attend):
        f(pool)
        f(pool, tables=torch.zeros(18, dtype=i32), lens=torch.zeros(9, dtype=i32))
        for q in (torch.zeros(3, 8, D), torch.zeros(2, 8, D, dtype=BF), torch.zeros(3, 8, 64, dtype=BF), wide[:, :8, :D],
                  wide[:, :8, ::2], torch.zeros(1, 8, D, dtype=BF).expand(3, 8, D), wide[:, ::2, :D]):
            refused(pool, f, q=q)
        for tables in (torch.zeros(3, 6, dtype=torch.int64), torch.zeros(3, 5, dtype=i32),
                       torch.zeros(3, 9, dtype=i32)[:, :6]):
            refused(pool, f, tables=tables)
        for lens in (torch.zeros(2, dtype=i32), torch.zeros(3, dtype=torch.int64), torch.zeros(6, dtype=i32)[::2]):
            refused(pool, f, lens=lens)
        for selected in (torch.zeros(3, 2, 4, dtype=torch.int64), torch.zeros(3, 2, 4, 1, dtype=i32),
                         torch.zeros(3, 4, 4, dtype=i32), torch.zeros(2, 2, 4, dtype=i32),
                         torch.zeros(3, 2, 8, dtype=i32)[:, :, :4]):
            refused(pool, f, selected=selected)
    for bounds in (torch.zeros(pool.bounds_bytes - 1, dtype=torch.int8), torch.zeros(2 * pool.bounds_bytes, dtype=torch.int8)[::2]):
        refused(pool, select, bounds=bounds)
    for scores in (torch.zeros(3, 2, 5), torch.zeros(3, 2, 6, dtype=BF), torch.zeros(3, 2, 7)[:, :, :6]):
        refused(pool, select, scores=scores)
    kv = torch.zeros(3, 4, D, dtype=BF)
    for kk, vv in ((kv[:, :2], kv[:, :2].contiguous()), (None, kv[:, :2]), (kv[:, :2], None),
                   (kv, kv), (kv[:, :2].float(), kv[:, :2].float())):
        refused(pool, attend, k=kk, v=vv)
    for out in (torch.zeros(3, 8, D, dtype=torch.float16), torch.zeros(3, 8, D + 1)[:, :, :D], torch.zeros(2, 8, D)):
        refused(pool, attend, out=out)


@BOTH
def test_tensors_on_another_device(package, native):
    pool = make_pool(package, native)

    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1
    a = arguments(pool)
    for f, names in ((select, ("q", "tables", "lens", "selected", "bounds", "scores")),
                     (attend, ("q", "k", "v", "tables", "lens", "selected", "out"))):
        for name in names:
            refused(pool, f, **{name: a[name].as_subclass(Elsewhere)})


def test_lists_of_a_compaction(package, monkeypatch):
    pool = make_pool(package, False)
    calls = []
    monkeypatch.setattr(package.kvtier, "session_compact", lambda *a: calls.append(a))
    i32 = torch.int32
    for keep, strides in ((torch.zeros(9, dtype=i32), (0, 0)), (torch.zeros(3, 2, 9, dtype=i32), (18, 9)),
                          (torch.zeros(3, 2, 12, dtype=i32)[:, :, 2:11], (24, 12)),
                          (torch.zeros(1, 1, 9, dtype=i32).expand(3, 2, 9), (0, 0)),
                          (torch.zeros(2, 3, 9, dtype=i32).transpose(0, 1), (9, 27))):
        pool.session_compact(4, keep, 7)
        assert calls[-1][1:2] + calls[-1][3:] == (4, *strides, 9, 7, None)
    n = len(calls)
    for keep in (torch.zeros(9, dtype=torch.int64), torch.zeros(2, 3, 9, dtype=i32), torch.zeros(2, 9, dtype=i32),
                 torch.zeros(18, dtype=i32)[::2], torch.zeros(1, dtype=i32).expand(9)):
        with pytest.raises(ValueError):
            pool.session_compact(4, keep, 7)
    assert len(calls) == n


def test_what_the_library_refuses(package):
    kv = package.kvtier
    cfg = kv.make_config(num_layers=2, num_hot_blocks=8, cold_bytes=1 << 20, flags=kv.KV_POOL_HOST_LOGIC_ONLY)
    pool = kv.kv_pool_create(cfg)
    assert kv.kv_bounds_bytes(cfg) == 2 * 4 * 8 * 258

    def code(f, *a):
        with pytest.raises(kv.KVError) as e:
            f(*a)
        return e.value.code

    bad, state = kv.KV_ERR_INVALID_ARG, kv.KV_ERR_BAD_STATE
    good = dict(layer=-1, tables=4, lens=4, since=4, B=2, width=4, bounds=256)
    for want, change in ((state, {}), (state, dict(since=None)), (state, dict(layer=1)), (bad, dict(layer=2)),
                         (bad, dict(layer=-2)), (bad, dict(tables=None)), (bad, dict(lens=None)), (bad, dict(since=2)),
                         (bad, dict(tables=6)), (bad, dict(bounds=None)), (bad, dict(bounds=128)), (bad, dict(B=0)),
                         (bad, dict(B=4097)), (bad, dict(width=0)), (bad, dict(B=4096, width=1 << 19))):
        a = dict(good, **change)
        assert code(kv.kv_pool_block_bounds, pool, *(a[x] for x in ("layer", "tables", "lens", "since", "B", "width", "bounds"))) == want, change
    good = dict(layer=0, q=16, q_stride=0, bounds=256, tables=4, lens=4, B=2, width=4, first=1, last=1, top=2, selected=4,
                scores=None)
    for want, change in ((state, {}), (state, dict(q_stride=32 * 128 + 8)), (state, dict(first=0, last=0, top=1)),
                         (bad, dict(layer=-1)), (bad, dict(layer=2)), (bad, dict(q=8)), (bad, dict(q=None)),
                         (bad, dict(bounds=16)), (bad, dict(selected=None)), (bad, dict(selected=2)), (bad, dict(scores=2)),
                         (bad, dict(q_stride=8)), (bad, dict(q_stride=32 * 128 + 4)), (bad, dict(q_stride=-8)),
                         (bad, dict(first=-1)), (bad, dict(last=-1)), (bad, dict(first=2)), (bad, dict(top=0)),
                         (bad, dict(first=2 ** 31 - 1, last=2 ** 31 - 1)), (bad, dict(width=49153)), (bad, dict(B=65536))):
        a = dict(good, **change)
        assert code(kv.select_blocks, pool, *(a[x] for x in ("layer", "q", "q_stride", "bounds", "tables", "lens", "B", "width",
                                                             "first", "last", "top", "selected", "scores"))) == want, change
    good = dict(layer=0, q=16, q_stride=0, k=16, v=32, kv_stride=0, selected=4, top=3, tables=4, lens=4, B=2, width=4,
                scale=1.0, out=16, flags=0)
    for want, change in ((state, {}), (state, dict(k=None, v=None)), (state, dict(scale=-2.0)), (bad, dict(k=None)),
                         (bad, dict(v=None)), (bad, dict(q=8)), (bad, dict(k=8)), (bad, dict(out=8)), (bad, dict(out=None)),
                         (bad, dict(selected=None)), (bad, dict(top=0)), (bad, dict(kv_stride=4)), (bad, dict(kv_stride=128)),
                         (bad, dict(scale=float("nan"))), (bad, dict(scale=float("inf"))), (bad, dict(scale=-3e38)), (bad, dict(flags=1)),
                         (bad, dict(flags=4)), (bad, dict(layer=-1)), (bad, dict(width=0)), (bad, dict(B=0))):
        a = dict(good, **change)
        assert code(kv.sparse_attention, pool, *(a[x] for x in ("layer", "q", "q_stride", "k", "v", "kv_stride", "selected",
                                                                "top", "tables", "lens", "B", "width", "scale", "out", "flags"))) == want, change
    assert code(kv.sparse_attention, None, 0, 16, 0, None, None, 0, 4, 1, 4, 4, 1, 1, 1.0, 16) == bad
    kv.kv_pool_destroy(pool)
