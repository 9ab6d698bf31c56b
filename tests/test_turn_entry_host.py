"""What Pool.prefill_attention and Pool.tree_attention hand to the library, and what they refuse,
without a GPU: tensors on the CPU and a library call that only notes its arguments."""
import pytest
import torch

D = 128


@pytest.fixture(scope="module")
def package():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2609_25782_gb300
    return paper_2609_25782_gb300


def make_pool(package, hq=8, hkv=2):
    """A pool without arenas or a handle."""
    p = package.Pool.__new__(package.Pool)
    p.device, p.handle, p.Hq, p.Hkv, p.D = torch.device("cpu"), None, hq, hkv, D
    p._bf16, p._i32, p._masks = torch.bfloat16, torch.int32, (torch.int64, torch.uint64)
    p._out_flags = {torch.float32: 0, torch.bfloat16: package.kvtier.KV_DECODE_OUT_BF16}
    p._index = -1                      # the device number that tensors on the CPU give
    p.calls = []
    p._prefill = p._tree = lambda *a: p.calls.append(a) or 0
    return p


def arguments(pool, n, sessions=1, kind="prefill", **other):
    a = dict(q=torch.zeros(n, pool.Hq, D).bfloat16(), k=torch.zeros(n, pool.Hkv, D).bfloat16(),
             v=torch.zeros(n, pool.Hkv, D).bfloat16(), cu=torch.zeros(sessions + 1, dtype=torch.int32),
             tables=torch.zeros(sessions, 4, dtype=torch.int32), lens=torch.zeros(sessions, dtype=torch.int32),
             B=sessions, width=4, out=torch.zeros(n, pool.Hq, D), stream=None,
             masks=torch.zeros(n, dtype=torch.int64))
    a.update(other)
    return a


def call(pool, kind, a):
    """The strides that reach the library: (q's, k's and v's)."""
    pool.calls.clear()
    if kind == "prefill":
        pool.prefill_attention(0, a["q"], a["k"], a["v"], a["cu"], a["tables"], a["lens"], a["B"], a["width"], 0.1,
                               a["out"], a["stream"])
    else:
        pool.tree_attention(0, a["q"], a["k"], a["v"], a["masks"], a["cu"], a["tables"], a["lens"], a["B"],
                            a["width"], 0.1, a["out"], a["stream"])
    (got,) = pool.calls
    assert got[2] == a["q"].data_ptr() and got[4] == a["k"].data_ptr() and got[5] == a["v"].data_ptr()
    return got[3], got[6]


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_tokens_that_share_storage_are_refused(package, kind):
    """The library takes a stride of 0 for rows one after the other: eight tokens expanded from one would be
    read from eight times their storage."""
    pool = make_pool(package)
    q, kv = torch.zeros(1, 8, D).bfloat16().expand(8, 8, D), torch.zeros(1, 2, D).bfloat16().expand(8, 2, D)
    assert q.stride(0) == kv.stride(0) == 0
    for other in (dict(q=q), dict(k=kv, v=kv), dict(q=q, k=kv, v=kv)):
        with pytest.raises(ValueError):
            call(pool, kind, arguments(pool, 8, **other))
    assert not pool.calls
    assert call(pool, kind, arguments(pool, 8)) == (8 * D, 2 * D)
    qkv = torch.zeros(8, 12, D).bfloat16()
    assert call(pool, kind, arguments(pool, 8, q=qkv[:, :8], k=qkv[:, 8:10], v=qkv[:, 10:])) == (12 * D, 12 * D)
    # a single token's stride means nothing
    call(pool, kind, arguments(pool, 1, q=q[:1], k=kv[:1], v=kv[:1]))


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_strides_that_mean_nothing_are_not_compared(package, kind):
    """A single token's stride, and a single head's: k may be contiguous and v a view."""
    pool = make_pool(package)
    qkv = torch.zeros(8, 12, D).bfloat16()
    call(pool, kind, arguments(pool, 1, v=qkv[:1, 10:]))
    call(pool, kind, arguments(pool, 1, k=qkv[:1, 8:10]))
    one = make_pool(package, hq=4, hkv=1)
    whole = torch.zeros(8, 6 * D).bfloat16()
    k = torch.as_strided(whole, (8, 1, D), (6 * D, D, 1), 4 * D)
    v = torch.as_strided(whole, (8, 1, D), (6 * D, 6 * D, 1), 5 * D)
    assert k.stride() != v.stride()
    assert call(one, kind, arguments(one, 8, k=k, v=v))[1] == 6 * D
    # strides that do mean something
    two = torch.zeros(8, 2, 2 * D).bfloat16()
    for other in (dict(v=qkv[:, 10:]), dict(v=two[:, :, :D]), dict(v=torch.zeros(8, 2, 2 * D).bfloat16()[:, :, ::2])):
        with pytest.raises(ValueError):
            call(pool, kind, arguments(pool, 8, **other))
    with pytest.raises(ValueError):
        call(pool, kind, arguments(pool, 1, v=two[:1, :, :D]))


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_offsets_tables_and_lengths_that_the_library_would_misread(package, kind):
    """32-bit integers, contiguous, as many as the call reads; a wider or longer buffer is no fault."""
    pool = make_pool(package)
    i32 = torch.int32

    def good(**other):
        return call(pool, kind, arguments(pool, 6, 2, **other))

    def bad(**other):
        with pytest.raises(ValueError):
            good(**other)
        assert not pool.calls
    good()
    good(cu=torch.zeros(9, dtype=i32), lens=torch.zeros(5, dtype=i32), tables=torch.zeros(3, 9, dtype=i32))
    good(tables=torch.zeros(8, dtype=i32))
    good(cu=torch.zeros(6, dtype=i32)[1:4])
    for name, n in (("cu", 3), ("lens", 2), ("tables", 8)):
        bad(**{name: torch.zeros(n, dtype=torch.int64)})         # what cumsum of 32-bit integers gives
        bad(**{name: torch.zeros(n, dtype=torch.float32)})
        bad(**{name: torch.zeros(n - 1, dtype=i32)})
        bad(**{name: torch.zeros(2 * n, dtype=i32)[::2]})
        bad(**{name: torch.zeros(1, dtype=i32).expand(n)})
    bad(tables=torch.zeros(2, 9, dtype=i32)[:, :4])              # columns of a wider table
    if kind == "tree":
        good(masks=torch.zeros(6, dtype=torch.uint64))
        for masks in (torch.zeros(6, dtype=torch.float64), torch.zeros(5, dtype=torch.int64),
                      torch.zeros(6, dtype=i32), torch.zeros(12, dtype=torch.int64)[::2]):
            bad(masks=masks)


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_tensors_on_another_device_are_refused(package, kind):
    """A host address would fault in the kernel: here the pool is on device 0, the tensors are not."""
    pool = make_pool(package)
    a = arguments(pool, 6, 2)
    call(pool, kind, a)

    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1
    for name in ("q", "k", "v", "cu", "tables", "lens", "out") + (("masks",) if kind == "tree" else ()):
        with pytest.raises(ValueError):
            call(pool, kind, dict(a, **{name: a[name].as_subclass(Elsewhere)}))
    pool._index = 0
    with pytest.raises(ValueError):
        call(pool, kind, a)
    assert not pool.calls


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_streams_as_in_the_other_calls(package, kind):
    """None (the legacy default stream), a torch stream, or a stream's handle as an integer."""
    pool = make_pool(package)

    class Stream:
        cuda_stream = 77
    for stream, handle in ((None, None), (Stream(), 77), (1234, 1234), (0, 0)):
        call(pool, kind, arguments(pool, 3, stream=stream))
        assert pool.calls[0][-1] == handle
