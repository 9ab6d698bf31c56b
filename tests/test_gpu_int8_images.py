"""8-bit cold images: codes, exponents and what is read back, against the definition in 64 bits.

Nothing here has a tolerance: the one rounding is to nearest even in exact arithmetic, and the
value of a code is exactly a bf16, so codes, exponents and bf16 bits are compared as they are.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

D = 128


def definition(x):
    """(codes, exponents, values) of rows x [..., D], float64 holding bf16 values."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    top = np.max(np.where(finite, np.abs(x), 0.0), axis=-1)
    _, e = np.frexp(top)                                 # top = m * 2^e, m in [0.5, 1)
    E = np.where(top > 0, np.maximum(1, e - 1 + 127), 1)
    scaled = np.ldexp(np.where(finite, x, 0.0), (133 - E)[..., None])
    codes = np.clip(np.rint(scaled), -127, 127)
    values = np.where(finite, np.ldexp(codes, (E - 133)[..., None]), np.nan)
    return np.where(finite, codes, -128).astype(np.int8), E.astype(np.uint8), values


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def same_values(t, want):
    return np.array_equal(f64(t), want, equal_nan=True)


def make_pool(L, hkv, bt, tokens, sessions=2, lru=False, seed=5):
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_25782_gb300 import Pool
    return Pool(num_layers=L, num_hot_blocks=-(-tokens // bt), cold_bytes=sessions * (tokens + 2) * L * 2 * hkv * 129
                + 1024, num_q_heads=hkv, num_kv_heads=hkv, block_tokens=bt, max_sessions=sessions,
                max_batch=1, max_context=tokens, alloc_seed=seed, lru_residency=lru, cold_int8=True)


def logical(pool, sid, t):
    """The session's hot tokens, [L][2][Hkv][t][D]."""
    row = torch.as_tensor(pool.session_block_table(sid), device="cuda", dtype=torch.int64)
    got = pool.hot_view()[row].permute(1, 2, 3, 0, 4, 5)
    return got.reshape(pool.L, 2, pool.Hkv, -1, D)[:, :, :, :t]


def image_of(pool, sid, t):
    codes, exps = pool.image_int8(sid)
    return codes[:, :, :, :t].cpu().numpy(), exps[:, :, :, :t].cpu().numpy()


def rows_of_every_kind(L, t, hkv, seed):
    """Rows whose largest values span bf16's exponents, subnormals and zeros, with ties, the
    rounding that would reach 128, and values that are not finite among them."""
    r = np.random.RandomState(seed)
    x = r.standard_normal((2, L, t, hkv, D)) * np.exp2(r.randint(-140, 125, (2, L, t, hkv, 1)).astype(np.float64))
    k = torch.from_numpy(np.clip(x, -3e38, 3e38)).to(torch.bfloat16)
    flat = k.view(-1, D)
    kinds = torch.from_numpy(r.randint(0, 10, flat.shape[0]))
    flat[kinds == 0] = 0.0
    flat[kinds == 1, 7] = float("inf")
    flat[kinds == 2, 127] = float("nan")
    flat[kinds == 3, 0] = float("-inf")
    for j, v in enumerate((1.9921875, -1.9921875, 1.0, 0.5 / 64, 1.5 / 64, -2.5 / 64, 126.5 / 64)):
        flat[kinds == 4, j] = v                          # 127.5, 64, 0.5, 1.5, 2.5, 126.5 steps
    flat[kinds == 4, 7:] = 0.0
    flat[kinds == 5] = float("nan")                      # a row with nothing finite
    return k.cuda()


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("hkv,t", [(1, 1), (2, 7), (4, 8), (3, 65), (8, 130)])
def test_pause_and_resume_follow_the_definition(cuda_dev, bt, hkv, t):
    L = 2
    pool = make_pool(L, hkv, bt, t)
    kv = rows_of_every_kind(L, t, hkv, seed=t * 10 + hkv)
    sid = pool.session_create(t)
    pool.session_append(sid, kv[0].contiguous(), kv[1].contiguous())
    pool.session_pause(sid)
    codes, exps, values = definition(f64(kv.permute(1, 0, 3, 2, 4)))
    got_codes, got_exps = image_of(pool, sid, t)
    assert np.array_equal(got_codes, codes) and np.array_equal(got_exps, exps)
    pool.hot.fill_(3.0)
    pool.session_resume(sid)
    assert same_values(logical(pool, sid, t), values)
    assert pool.check_device() == 0


@pytest.mark.parametrize("lru", [False, True])
@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("t1,t2", [(7, 8), (8, 9), (23, 25), (57, 71), (64, 120)])
def test_tokens_are_quantised_once(cuda_dev, bt, lru, t1, t2):
    """A second pause writes the new tokens alone; what came back goes out as it came."""
    from paper_2609_25782_gb300 import kvtier
    L, hkv = 2, 2
    pool = make_pool(L, hkv, bt, t2, lru=lru)
    kv = torch.randn(2, L, t2, hkv, D, device="cuda",
                     generator=torch.Generator(device="cuda").manual_seed(2)).bfloat16()
    codes, exps, values = definition(f64(kv.permute(1, 0, 3, 2, 4)))
    sid, other = pool.session_create(t2), pool.session_create(t2)
    row_bytes = L * 2 * hkv * (D + 1)
    assert kvtier.kv_image_token_bytes(kvtier.make_config(num_layers=L, num_kv_heads=hkv, num_q_heads=hkv,
                                       num_hot_blocks=1, flags=kvtier.KV_POOL_COLD_INT8)) == row_bytes
    for a, b in ((0, t1), (t1, t2)):
        pool.session_append(sid, kv[0, :, a:b].contiguous(), kv[1, :, a:b].contiguous())
        before = pool.stats()["bytes_packed"]
        pool.session_pause(sid)
        zeros = torch.zeros_like(kv[0])
        pool.session_append(other, zeros, zeros)         # takes every block
        assert pool.stats()["bytes_packed"] - before == (b - a) * row_bytes
        got_codes, got_exps = image_of(pool, sid, b)
        assert np.array_equal(got_codes, codes[:, :, :, :b]) and np.array_equal(got_exps, exps[:, :, :, :b])
        pool.session_destroy(other)
        pool.shuffle_free(b)
        before = pool.stats()["bytes_unpacked"]
        pool.session_resume(sid)
        assert pool.stats()["bytes_unpacked"] - before == b * row_bytes
        assert same_values(logical(pool, sid, b), values[:, :, :, :b])
        other = pool.session_create(t2)
    assert pool.check_device() == 0


def test_packing_what_was_read_back_changes_nothing(cuda_dev):
    L, hkv, t, bt = 1, 4, 40, 16
    pool = make_pool(L, hkv, bt, 2 * 48)                # three blocks for each of two sessions
    kv = rows_of_every_kind(L, t, hkv, seed=3)
    kv[~torch.isfinite(kv)] = 1.0
    a, b = pool.session_create(t), pool.session_create(t)
    pool.session_append(a, kv[0].contiguous(), kv[1].contiguous())
    pool.session_pause(a)
    pool.session_resume(a)
    back = logical(pool, a, t)                           # [L][2][Hkv][t][D]
    pool.session_append(b, back[:, 0].transpose(1, 2).contiguous(), back[:, 1].transpose(1, 2).contiguous())
    pool.session_pause(b)
    pool.session_resume(b)
    assert torch.equal(logical(pool, b, t).view(torch.int16), back.view(torch.int16))
    assert pool.check_device() == 0


@pytest.mark.parametrize("lru", [False, True])
def test_images_the_caller_fills_and_moves_that_stride(cuda_dev, lru):
    """A session created paused reads the codes that the caller wrote, exponents 0 to 255 and code
    -128 among them; after a decode call on another stream the move's CTAs stride over its chunks."""
    L, hkv, t, bt = 8, 4, 7201, 16
    pool = make_pool(L, hkv, bt, t, sessions=1, lru=lru)
    sid = pool.session_create_paused(t, t)
    r = np.random.RandomState(0)
    codes = r.randint(-127, 128, (L, 2, hkv, t, D)).astype(np.int8)
    exps = r.randint(0, 249, (L, 2, hkv, t)).astype(np.uint8)
    codes[0, 0, 0, :50, :5] = -128
    to_codes, to_exps = pool.image_int8(sid)
    to_codes.copy_(torch.from_numpy(codes))
    to_exps.copy_(torch.from_numpy(exps))
    q = torch.zeros(1, hkv, D, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    out = torch.empty(1, hkv, D, device="cuda")
    pool.decode_attention(0, q, table, one, 1, 1, 1.0, out)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    pool.session_resume(sid, side)
    side.synchronize()
    values = np.where(codes == -128, np.nan, np.ldexp(codes.astype(np.float64), exps.astype(int)[..., None] - 133))
    assert same_values(logical(pool, sid, t), values)
    assert pool.check_device() == 0


@pytest.mark.slow
def test_image_offsets_past_32_bits(cuda_dev):
    """An image whose codes pass 2^32 bytes: the last runs' rows and exponents."""
    L, hkv, cap, t, bt = 48, 8, 45000, 50, 16
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_25782_gb300 import Pool
    rows = L * 2 * hkv * cap
    assert rows * D > 1 << 32
    pool = Pool(num_layers=L, num_hot_blocks=4, cold_bytes=rows * 129 + 512, num_q_heads=hkv, num_kv_heads=hkv,
                block_tokens=bt, max_sessions=1, max_batch=1, max_context=cap, cold_int8=True)
    sid = pool.session_create(cap)
    kv = torch.randn(2, L, t, hkv, D, device="cuda").bfloat16()
    pool.session_append(sid, kv[0].contiguous(), kv[1].contiguous())
    pool.session_pause(sid)
    codes, exps, values = definition(f64(kv.permute(1, 0, 3, 2, 4)))
    got_codes, got_exps = image_of(pool, sid, t)
    assert np.array_equal(got_codes, codes) and np.array_equal(got_exps, exps)
    pool.session_resume(sid)
    assert same_values(logical(pool, sid, t), values)


def test_views_refuse_the_other_kind(cuda_dev):
    pool = make_pool(1, 1, 16, 16)
    sid = pool.session_create(16)
    with pytest.raises(ValueError):
        pool.image(sid)
    import __graft_entry__
    from paper_2609_25782_gb300 import Pool
    plain = Pool(num_layers=1, num_hot_blocks=1, cold_bytes=1 << 16, max_sessions=1, max_batch=1, max_context=16)
    with pytest.raises(ValueError):
        plain.image_int8(plain.session_create(16))
