"""What a pool allocates and sets up, and when, without a GPU: the pool runtime over a stand-in for the
CUDA runtime (fake_cuda.cpp) that notes allocations and fails when told to."""
import atexit
import ctypes as C
import functools
import os
import shutil
import subprocess
import tempfile

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_25782_gb300", "csrc")
SMS = 152


def cuda_include():
    nvcc = os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    return os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")


@pytest.fixture(scope="module")
def kv():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_25782_gb300 import kvtier
    return kvtier


@functools.cache
def built():
    d = tempfile.mkdtemp()
    so = os.path.join(d, "pool.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-I", CSRC, "-I", cuda_include(),
                    os.path.join(HERE, "fake_cuda.cpp"), os.path.join(CSRC, "pool.cpp"), "-o", so], check=True)
    atexit.register(shutil.rmtree, d)
    return so


@pytest.fixture()
def fake(kv, tmp_path):
    """A pool runtime of the test's own: a copy of the library has its variables at their start."""
    x = C.CDLL(shutil.copy(built(), tmp_path / "pool.so"))
    for name in ("prefill_attention", "tree_attention", "decode_attention", "kv_pool_create", "kv_pool_destroy"):
        getattr(x, name).argtypes = getattr(kv.lib, name).argtypes
    x.fake_allocations.restype = x.part_bytes.restype = C.c_int64
    x.fake_allocations.argtypes = [C.c_void_p, C.c_int64]
    x.kv_last_error.restype = C.c_char_p
    return x


def allocations(fake):
    out = (C.c_int64 * 64)()
    return list(out[:fake.fake_allocations(out, 64)])


def create(kv, fake):
    cfg = kv.make_config(num_layers=2, num_hot_blocks=64, max_sessions=2, max_batch=2, max_context=512,
                         hot_base=1 << 20, cold_base=1 << 21, cold_bytes=1 << 20)
    pool = C.c_void_p()
    assert fake.kv_pool_create(C.byref(cfg), C.byref(pool)) == kv.KV_OK
    return pool


def turn(fake, pool, width, kind="prefill"):
    """A call on 4 tokens of one session whose table holds `width` blocks of 16 tokens."""
    a = 256
    if kind == "prefill":
        return fake.prefill_attention(pool, 0, a, 0, a, a, 0, a, 4, a, a, 1, width, 0.1, a, 0, None)
    return fake.tree_attention(pool, 0, a, 0, a, a, 0, a, a, 4, a, a, 1, width, 0.1, a, 0, None)


def decode(fake, pool):
    return fake.decode_attention(pool, 0, 256, 256, 256, 1, 32, 0.1, 256, None)


def test_a_pool_that_decodes_holds_no_workspace_for_prompts(kv, fake):
    pool = create(kv, fake)
    first = allocations(fake)
    assert len(first) == 1 and first[0] < fake.part_bytes(SMS)
    assert decode(fake, pool) == kv.KV_OK and fake.fake_decodes() == 1
    assert turn(fake, pool, 8) == kv.KV_OK               # 128 tokens: no partial results
    assert allocations(fake) == first and not fake.fake_has_part()
    assert turn(fake, pool, 9) == kv.KV_OK and fake.fake_has_part()
    assert allocations(fake) == first + [fake.part_bytes(SMS)]
    for kind in ("prefill", "tree"):
        assert turn(fake, pool, 32, kind) == kv.KV_OK and turn(fake, pool, 4, kind) == kv.KV_OK
    assert len(allocations(fake)) == 2 and fake.fake_turns() == 6
    assert fake.kv_pool_destroy(pool) == kv.KV_OK and fake.fake_live() == 0


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_no_room_for_the_workspace(kv, fake, kind):
    """The call fails and leaves nothing behind, no error for a later launch either; the next one may go on."""
    pool = create(kv, fake)
    fake.fake_fail_malloc()
    assert turn(fake, pool, 32, kind) == kv.KV_ERR_CUDA and b"workspace" in fake.kv_last_error()
    assert fake.fake_turns() == 0 and fake.fake_last_error() == 0 and fake.fake_live() == 1
    assert decode(fake, pool) == kv.KV_OK
    assert turn(fake, pool, 32, kind) == kv.KV_OK and fake.fake_turns() == 1
    assert fake.kv_pool_destroy(pool) == kv.KV_OK and fake.fake_live() == 0


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_a_first_call_that_a_graph_records(kv, fake, kind):
    """Only in the relaxed mode may a thread that records allocate; the mode is put back."""
    pool = create(kv, fake)
    before, mode = fake.fake_strict_mallocs(), fake.fake_mode()
    assert turn(fake, pool, 32, kind) == kv.KV_OK and fake.fake_strict_mallocs() == before
    assert fake.fake_mode() == mode
    assert fake.kv_pool_destroy(pool) == kv.KV_OK


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_a_turn_kernel_that_cannot_run_does_not_keep_a_pool_from_decoding(kv, fake, kind):
    """Its preparation fails where the compiler gave it other registers than its warps' shares presume."""
    invalid_configuration = 9
    fake.fake_turn_status(invalid_configuration)
    pool = create(kv, fake)
    assert decode(fake, pool) == kv.KV_OK
    for width in (4, 32):
        assert turn(fake, pool, width, kind) == kv.KV_ERR_CUDA
        assert fake.fake_turns() == 0 and fake.fake_live() == 1 and fake.fake_last_error() == 0
    fake.fake_turn_status(0)
    assert turn(fake, pool, 32, kind) == kv.KV_OK and fake.fake_turns() == 1
    assert fake.kv_pool_destroy(pool) == kv.KV_OK and fake.fake_live() == 0
