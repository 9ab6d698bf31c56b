"""Reservation of several positions per session, and refusals, without a GPU."""
import random

import pytest


@pytest.fixture(scope="module")
def kv():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_25782_gb300 import kvtier
    return kvtier


def host_pool(kv, nb=40, flags=0, bt=16):
    cfg = kv.make_config(num_layers=2, num_hot_blocks=nb, block_tokens=bt, alloc_seed=7, max_sessions=8,
                         max_context=4096, cold_bytes=1 << 30, flags=kv.KV_POOL_HOST_LOGIC_ONLY | flags)
    return kv.kv_pool_create(cfg)


def state(kv, pool, sids):
    rows = [(tuple(kv.session_block_table(pool, s)), kv.session_info(pool, s).tokens,
             kv.session_info(pool, s).num_blocks) for s in sids]
    return rows, kv.kv_pool_free_list(pool), kv.kv_pool_get_stats(pool)


@pytest.mark.parametrize("lru", [False, True])
@pytest.mark.parametrize("bt", [16, 64])
def test_counts_pop_as_single_positions_do(kv, lru, bt):
    """n positions at once give the tokens that n single reservations give; one member's blocks come in
    the same order."""
    flags = kv.KV_POOL_LRU_RESIDENCY if lru else 0
    a, b = host_pool(kv, flags=flags, bt=bt), host_pool(kv, flags=flags, bt=bt)
    r = random.Random(1)
    for p in (a, b):
        kv.session_create(p, 400)
    for _ in range(12):
        n = r.choice([1, 2, 15, 16, 17, 33])
        kv.kv_pool_batch_reserve_tokens(a, [0], [n], None, 1 << 20, None)
        for _ in range(n):
            kv.kv_pool_batch_reserve(b, [0], None, 1 << 20, None)
        ra, rb = state(kv, a, [0]), state(kv, b, [0])
        assert ra[0] == rb[0] and ra[1] == rb[1]
        assert ra[2]["bytes_appended"] == rb[2]["bytes_appended"]
        if ra[0][0][1] > 350:
            break
    for p in (a, b):
        kv.kv_pool_destroy(p)


def test_members_pop_in_batch_order_and_zero_counts_keep_their_place(kv):
    pool = host_pool(kv)
    order = kv.kv_pool_free_list(pool)[::-1]
    sids = [kv.session_create(pool, 500) for _ in range(3)]
    kv.kv_pool_batch_reserve_tokens(pool, sids, [20, 1, 40], None, 100, None)
    assert [kv.session_block_table(pool, s) for s in sids] == [order[:2], order[2:3], order[3:6]]
    kv.kv_pool_batch_reserve_tokens(pool, sids, [0, 15, 9], None, 100, None)
    assert [kv.session_block_table(pool, s) for s in sids] == [order[:2], order[2:3], order[3:6] + order[6:7]]
    assert [kv.session_info(pool, s).tokens for s in sids] == [20, 16, 49]
    kv.kv_pool_destroy(pool)


def test_refusals_change_nothing(kv):
    pool = host_pool(kv, nb=6)
    sids = [kv.session_create(pool, 60), kv.session_create(pool, 200)]
    kv.kv_pool_batch_reserve_tokens(pool, sids, [30, 17], None, 100, None)
    before = state(kv, pool, sids)
    for counts, width, code in (([31, 1], 100, kv.KV_ERR_INVALID_ARG),      # past the capacity
                                ([-1, 1], 100, kv.KV_ERR_INVALID_ARG), ([1, 100], 5, kv.KV_ERR_INVALID_ARG),
                                ([1, 80], 100, kv.KV_ERR_NO_HOT_BLOCKS)):
        with pytest.raises(kv.KVError) as e:
            kv.kv_pool_batch_reserve_tokens(pool, sids, counts, None, width, None)
        assert e.value.code == code
        assert state(kv, pool, sids) == before
    with pytest.raises(ValueError):
        kv.kv_pool_batch_reserve_tokens(pool, sids, [1], None, 100, None)
    empty = kv.session_create(pool, 60)
    with pytest.raises(kv.KVError) as e:
        kv.kv_pool_batch_reserve_tokens(pool, [empty], [0], None, 100, None)
    assert e.value.code == kv.KV_ERR_INVALID_ARG
    with pytest.raises(kv.KVError) as e:
        kv.kv_pool_batch_reserve_tokens(pool, [sids[0], sids[0]], [1, 1], None, 100, None)
    assert e.value.code == kv.KV_ERR_INVALID_ARG
    kv.session_pause(pool, sids[0], None)
    with pytest.raises(kv.KVError) as e:
        kv.kv_pool_batch_reserve_tokens(pool, [sids[0]], [1], None, 100, None)
    assert e.value.code == kv.KV_ERR_BAD_STATE
    kv.kv_pool_destroy(pool)


def test_eviction_makes_room_for_a_turn(kv):
    pool = host_pool(kv, nb=10, flags=kv.KV_POOL_LRU_RESIDENCY)
    a, b = kv.session_create(pool, 300), kv.session_create(pool, 300)
    kv.kv_pool_batch_reserve_tokens(pool, [a], [100], None, 100, None)      # 7 blocks
    kv.kv_pool_batch_reserve_tokens(pool, [b], [90], None, 100, None)       # 6: three of a's leave
    assert kv.kv_pool_get_stats(pool)["blocks_evicted"] == 3
    assert kv.session_block_table(pool, a)[:3] == [-1, -1, -1]
    kv.kv_pool_destroy(pool)


def test_attention_refuses_host_pools_after_its_arguments(kv):
    pool = host_pool(kv)
    for f in (lambda layer: kv.prefill_attention(pool, layer, 256, 0, 256, 256, 0, 256, 4, 256, 256, 1, 1, 1.0, 256),
              lambda layer: kv.tree_attention(pool, layer, 256, 0, 256, 256, 0, 256, 256, 4, 256, 256, 1, 1, 1.0,
                                              256)):
        with pytest.raises(kv.KVError) as e:
            f(0)
        assert e.value.code == kv.KV_ERR_BAD_STATE
        with pytest.raises(kv.KVError) as e:
            f(-1)
        assert e.value.code == kv.KV_ERR_INVALID_ARG
    kv.kv_pool_destroy(pool)
