"""Accounting of 8-bit cold images on host-logic pools, without a GPU."""
import pytest


@pytest.fixture(scope="module")
def kv():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_25782_gb300 import kvtier
    return kvtier


def host_pool(kv, cold_bytes, flags=0):
    cfg = kv.make_config(num_layers=3, num_kv_heads=4, num_hot_blocks=20, max_sessions=4, max_context=400,
                         cold_bytes=cold_bytes, flags=kv.KV_POOL_HOST_LOGIC_ONLY | flags)
    return kv.kv_pool_create(cfg), cfg


def test_image_bytes_per_token(kv):
    pool, cfg = host_pool(kv, 0, kv.KV_POOL_COLD_INT8)
    assert kv.kv_image_token_bytes(cfg) == 3 * 2 * 4 * 129
    assert kv.kv_token_bytes(cfg) == 3 * 2 * 4 * 256
    kv.kv_pool_destroy(pool)
    pool, cfg = host_pool(kv, 0)
    assert kv.kv_image_token_bytes(cfg) == kv.kv_token_bytes(cfg)
    kv.kv_pool_destroy(pool)


def test_cold_space_and_counters(kv):
    """An arena of two 8-bit images of 100 tokens holds those, and no third; moves count image bytes."""
    per = 3 * 2 * 4 * 129
    image = -(-100 * per // 256) * 256
    pool, _ = host_pool(kv, 2 * image, kv.KV_POOL_COLD_INT8)
    a, _b = kv.session_create(pool, 100), kv.session_create(pool, 100)
    with pytest.raises(kv.KVError) as e:
        kv.session_create(pool, 100)
    assert e.value.code == kv.KV_ERR_NO_COLD_SPACE
    kv.session_append(pool, a, None, None, 37, None)
    kv.session_pause(pool, a, None)
    kv.session_resume(pool, a, None)
    kv.session_append(pool, a, None, None, 5, None)
    kv.session_pause(pool, a, None)
    s = kv.kv_pool_get_stats(pool)
    assert (s["bytes_packed"], s["bytes_unpacked"]) == (42 * per, 37 * per)
    assert s["bytes_appended"] == 42 * 3 * 2 * 4 * 256
    assert s["cold_bytes_used"] == 2 * image
    kv.kv_pool_destroy(pool)


def test_residency_counts_image_bytes(kv):
    per = 3 * 2 * 4 * 129
    pool, _ = host_pool(kv, 1 << 24, kv.KV_POOL_COLD_INT8 | kv.KV_POOL_LRU_RESIDENCY)
    a, b = kv.session_create(pool, 320), kv.session_create(pool, 320)
    kv.session_append(pool, a, None, None, 200, None)    # 13 of 20 blocks
    kv.session_append(pool, b, None, None, 160, None)    # 10: three of a's leave
    s = kv.kv_pool_get_stats(pool)
    assert s["blocks_evicted"] == 3 and s["bytes_packed"] == 48 * per
    kv.session_pause(pool, b, None)
    kv.session_pause(pool, a, None)
    kv.session_resume(pool, a, None)                     # three of b's leave, a's come back
    s = kv.kv_pool_get_stats(pool)
    assert s["bytes_unpacked"] == 48 * per and s["bytes_packed"] == 96 * per
    kv.kv_pool_destroy(pool)
