"""Forks, truncation and compaction: placement, holders of shared blocks, images and refusals, without a GPU."""
import random

import pytest


@pytest.fixture(scope="module")
def kv():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_25782_gb300 import kvtier
    return kvtier


def host_pool(kv, nb=60, lru=False, bt=16, sessions=10, cold=1 << 30, L=2):
    cfg = kv.make_config(num_layers=L, num_hot_blocks=nb, block_tokens=bt, alloc_seed=7, max_sessions=sessions,
                         max_context=4096, cold_bytes=cold,
                         flags=kv.KV_POOL_HOST_LOGIC_ONLY | (kv.KV_POOL_LRU_RESIDENCY if lru else 0))
    return kv.kv_pool_create(cfg)


def live(kv, pool, sessions=10):
    out = []
    for s in range(sessions):
        try:
            kv.session_info(pool, s)
            out.append(s)
        except kv.KVError:
            pass
    return out


def state(kv, pool):
    rows = {}
    for s in live(kv, pool):
        i = kv.session_info(pool, s)
        rows[s] = (i.state, i.num_blocks, i.tokens, i.capacity, i.cold_valid, tuple(kv.session_block_table(pool, s)))
    return rows, kv.kv_pool_free_list(pool), kv.kv_pool_get_stats(pool)


def check(kv, pool, nb, lru, bt):
    rows, free, st = state(kv, pool)
    held = [b for r in rows.values() for b in r[5] if b >= 0]
    assert len(free) == len(set(free)) and not set(free) & set(held)
    assert sorted(set(held) | set(free)) == list(range(nb))
    assert st["free_blocks"] == len(free) and st["used_blocks"] == len(set(held))
    if lru:
        assert len(held) == len(set(held))               # one owner
    for s, (state_, blocks, tokens, cap, cold, row) in rows.items():
        assert tokens <= cap and cold <= tokens and blocks == sum(b >= 0 for b in row)
        if state_ == kv.KV_SESSION_ACTIVE or lru:
            assert len(row) == -(-tokens // bt)
        if not lru and tokens % bt and row:              # a block that may be written has one holder
            assert held.count(row[-1]) == 1


def reserve(kv, pool, sid, n):
    kv.kv_pool_batch_reserve_tokens(pool, [sid], [n], None, 1 << 20, None)


def refused(kv, code, f, *a):
    with pytest.raises(kv.KVError) as e:
        f(*a)
    assert e.value.code == code, e.value


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("tokens", [0, 1, 63, 64, 65, 128, 200])
def test_fork_shares_full_blocks(kv, tokens, bt):
    pool = host_pool(kv, bt=bt)
    p = kv.session_create(pool, 400)
    reserve(kv, pool, p, 200)
    row, free = kv.session_block_table(pool, p), kv.kv_pool_free_list(pool)[::-1]
    kids = kv.session_fork(pool, p, tokens, 300, 3)
    assert kids == [1, 2, 3]
    full, part = tokens // bt, tokens % bt > 0
    for i, k in enumerate(kids):
        info = kv.session_info(pool, k)
        assert (info.state, info.tokens, info.capacity, info.cold_valid) == (kv.KV_SESSION_ACTIVE, tokens, 300, 0)
        assert kv.session_block_table(pool, k) == row[:full] + free[i:i + 1] * part
    assert kv.session_block_table(pool, p) == row
    check(kv, pool, 60, False, bt)
    before = len(kv.kv_pool_free_list(pool))
    kv.session_destroy(pool, p)                          # what the forks hold stays
    assert len(kv.kv_pool_free_list(pool)) == before + len(row) - full
    for k in kids:
        kv.session_pause(pool, k, None)
        check(kv, pool, 60, False, bt)
    assert len(kv.kv_pool_free_list(pool)) == 60
    for k in kids:
        kv.session_resume(pool, k, None)                 # blocks of their own now
    check(kv, pool, 60, False, bt)
    rows = [b for k in kids for b in kv.session_block_table(pool, k)]
    assert len(rows) == len(set(rows)) == 3 * -(-tokens // bt)
    kv.kv_pool_destroy(pool)


def test_fork_of_a_fork_and_growth(kv):
    pool = host_pool(kv)
    p = kv.session_create(pool, 400)
    reserve(kv, pool, p, 100)
    a, = kv.session_fork(pool, p, 100, 400, 1)
    reserve(kv, pool, a, 60)
    b, c = kv.session_fork(pool, a, 150, 400, 2)
    rp, ra, rb, rc = (kv.session_block_table(pool, s) for s in (p, a, b, c))
    assert ra[:6] == rp[:6] and rb[:9] == ra[:9] == rc[:9] and len({ra[9], rb[9], rc[9], rp[6], ra[6]}) == 5
    for s in (a, p, c):
        kv.session_destroy(pool, s)
        check(kv, pool, 60, False, 16)
    reserve(kv, pool, b, 100)
    assert kv.session_block_table(pool, b)[:10] == rb
    check(kv, pool, 60, False, 16)
    kv.kv_pool_destroy(pool)


def test_fork_in_residency_mode_owns_its_blocks(kv):
    pool = host_pool(kv, nb=30, lru=True)
    p, o = kv.session_create(pool, 400), kv.session_create(pool, 400)
    reserve(kv, pool, o, 160)                            # 10 blocks
    reserve(kv, pool, p, 130)                            # 9
    kids = kv.session_fork(pool, p, 130, 130, 2)         # 18: 7 of o's leave
    st = kv.kv_pool_get_stats(pool)
    assert st["blocks_evicted"] == 7 and kv.session_info(pool, o).num_blocks == 3
    check(kv, pool, 30, True, 16)
    assert all(kv.session_info(pool, k).num_blocks == 9 for k in kids)
    # a parent whose blocks have left: read from its image
    kv.kv_pool_batch_reserve_tokens(pool, [o], [0], None, 100, None)
    assert kv.session_info(pool, p).num_blocks < 9
    third, = kv.session_fork(pool, p, 100, 100, 1)
    assert kv.session_info(pool, third).num_blocks == 7
    check(kv, pool, 30, True, 16)
    refused(kv, kv.KV_ERR_NO_HOT_BLOCKS, kv.session_fork, pool, p, 130, 130, 4)
    kv.kv_pool_destroy(pool)


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("int8", [False, True])
def test_what_a_fork_reads_from_an_image_counts(kv, int8, bt):
    """bytes_unpacked: evicted blocks of the parent, once for each new session, by the image's bytes a token."""
    cfg = kv.make_config(num_layers=2, num_hot_blocks=30, block_tokens=bt, alloc_seed=7, max_sessions=10, max_context=4096,
                         cold_bytes=1 << 30, flags=kv.KV_POOL_HOST_LOGIC_ONLY | kv.KV_POOL_LRU_RESIDENCY |
                         (kv.KV_POOL_COLD_INT8 if int8 else 0))
    pool = kv.kv_pool_create(cfg)
    token = 2 * 2 * 4 * (129 if int8 else 256)
    p, o = kv.session_create(pool, 10 * bt), kv.session_create(pool, 30 * bt)
    reserve(kv, pool, p, 6 * bt + 5)
    kv.session_fork(pool, p, 6 * bt + 5, 7 * bt, 1)      # nothing has left yet
    assert kv.kv_pool_get_stats(pool)["bytes_unpacked"] == 0
    kv.session_truncate(pool, 2, 0)
    reserve(kv, pool, o, 27 * bt)                        # 3 free: p's first four blocks leave
    assert kv.session_block_table(pool, p)[:4] == [-1] * 4 and kv.session_info(pool, p).num_blocks == 3
    kv.session_truncate(pool, o, 15 * bt)
    kv.session_fork(pool, p, 6 * bt + 5, 7 * bt, 1)      # four blocks from the image
    assert kv.kv_pool_get_stats(pool)["bytes_unpacked"] == 4 * bt * token
    kv.session_truncate(pool, 3, 0)
    kv.session_fork(pool, p, 2 * bt + 3, 7 * bt, 2)      # a part of the third one
    assert kv.kv_pool_get_stats(pool)["bytes_unpacked"] == (4 * bt + 2 * (2 * bt + 3)) * token
    before = kv.kv_pool_get_stats(pool)["bytes_unpacked"]
    refused(kv, kv.KV_ERR_NO_HOT_BLOCKS, kv.session_fork, pool, p, 6 * bt + 5, 7 * bt, 5)
    assert kv.kv_pool_get_stats(pool)["bytes_unpacked"] == before
    check(kv, pool, 30, True, bt)
    kv.kv_pool_destroy(pool)


def test_fork_refusals_change_nothing(kv):
    pool = host_pool(kv, nb=8, sessions=4, cold=800 * 4096)       # images of 800 tokens
    p = kv.session_create(pool, 200)
    reserve(kv, pool, p, 100)                            # 7 blocks, one free
    before = state(kv, pool)
    for code, a in ((kv.KV_ERR_INVALID_ARG, (p, 101, 200, 1)), (kv.KV_ERR_INVALID_ARG, (p, -1, 200, 1)),
                    (kv.KV_ERR_INVALID_ARG, (p, 50, 49, 1)), (kv.KV_ERR_INVALID_ARG, (p, 50, 5000, 1)),
                    (kv.KV_ERR_INVALID_ARG, (p, 0, 0, 1)), (kv.KV_ERR_INVALID_ARG, (p, 50, 200, 0)),
                    (kv.KV_ERR_INVALID_ARG, (2, 50, 200, 1)), (kv.KV_ERR_INVALID_ARG, (-1, 0, 200, 1)),
                    (kv.KV_ERR_NO_HOT_BLOCKS, (p, 100, 200, 2)), (kv.KV_ERR_INVALID_ARG, (p, 96, 100, 4)),
                    (kv.KV_ERR_NO_COLD_SPACE, (p, 96, 400, 2))):
        refused(kv, code, kv.session_fork, pool, *a)
        assert state(kv, pool) == before, a
    kv.session_pause(pool, p, None)
    refused(kv, kv.KV_ERR_BAD_STATE, kv.session_fork, pool, p, 50, 200, 1)
    kv.kv_pool_destroy(pool)


@pytest.mark.parametrize("lru", [False, True])
def test_truncate_gives_back_in_order(kv, lru):
    pool = host_pool(kv, lru=lru)
    s = kv.session_create(pool, 400)
    reserve(kv, pool, s, 200)
    row, free = kv.session_block_table(pool, s), kv.kv_pool_free_list(pool)
    for t in (200, 199, 193, 192, 100, 1, 0):
        kv.session_truncate(pool, s, t)
        assert kv.session_info(pool, s).tokens == t
        n = -(-t // 16)
        assert kv.session_block_table(pool, s) == row[:n]
        assert kv.kv_pool_free_list(pool) == free + row[n:][::-1]
        check(kv, pool, 60, lru, 16)
    reserve(kv, pool, s, 170)                            # the same blocks again
    assert kv.session_block_table(pool, s) == row[:11]
    for bad in (-1, 171):
        refused(kv, kv.KV_ERR_INVALID_ARG, kv.session_truncate, pool, s, bad)
    kv.kv_pool_destroy(pool)


def test_truncate_into_a_shared_block(kv):
    pool = host_pool(kv, nb=9)
    p = kv.session_create(pool, 200)
    reserve(kv, pool, p, 128)
    k, = kv.session_fork(pool, p, 128, 200, 1)           # all shared
    rows = kv.session_block_table(pool, p)
    spare, = kv.kv_pool_free_list(pool)
    kv.session_truncate(pool, k, 100)
    assert kv.session_block_table(pool, k) == rows[:6] + [spare] and kv.session_block_table(pool, p) == rows
    check(kv, pool, 9, False, 16)
    before = state(kv, pool)
    refused(kv, kv.KV_ERR_NO_HOT_BLOCKS, kv.session_truncate, pool, k, 90)
    assert state(kv, pool) == before
    kv.session_truncate(pool, k, 80)                     # a block's end: nothing to copy
    assert kv.session_block_table(pool, k) == rows[:5] and kv.kv_pool_free_list(pool) == [spare]
    kv.session_truncate(pool, p, 60)
    assert kv.session_block_table(pool, p) == rows[:3] + [spare]
    check(kv, pool, 9, False, 16)
    kv.kv_pool_destroy(pool)


@pytest.mark.parametrize("lru", [False, True])
def test_truncate_of_a_paused_session(kv, lru):
    pool = host_pool(kv, lru=lru)
    s = kv.session_create(pool, 300)
    reserve(kv, pool, s, 150)
    kv.session_pause(pool, s, None)
    kv.session_truncate(pool, s, 70)
    info = kv.session_info(pool, s)
    assert (info.state, info.tokens) == (kv.KV_SESSION_PAUSED, 70) and info.cold_valid == (0 if lru else 70)
    kv.session_resume(pool, s, None)
    assert len(kv.session_block_table(pool, s)) == 5
    reserve(kv, pool, s, 30)
    kv.session_pause(pool, s, None)
    assert kv.session_info(pool, s).cold_valid == (0 if lru else 100)
    kv.session_truncate(pool, s, 0)
    kv.session_resume(pool, s, None)
    reserve(kv, pool, s, 5)
    check(kv, pool, 60, lru, 16)
    kv.kv_pool_destroy(pool)


def test_truncation_and_compaction_limit_what_the_image_holds(kv):
    """Packed bytes: what a pause writes again."""
    pool = host_pool(kv)
    s = kv.session_create(pool, 300)
    token = 2 * 2 * 4 * 128 * 2
    reserve(kv, pool, s, 150)
    kv.session_pause(pool, s, None)
    kv.session_resume(pool, s, None)
    assert kv.kv_pool_get_stats(pool)["bytes_packed"] == 150 * token
    kv.session_truncate(pool, s, 101)
    reserve(kv, pool, s, 9)
    kv.session_pause(pool, s, None)
    assert kv.kv_pool_get_stats(pool)["bytes_packed"] == 159 * token
    kv.session_resume(pool, s, None)
    kv.session_compact(pool, s, 256, 0, 0, 20, 50)
    assert kv.session_info(pool, s).cold_valid == 50
    kv.session_pause(pool, s, None)
    assert kv.kv_pool_get_stats(pool)["bytes_packed"] == 179 * token
    kv.kv_pool_destroy(pool)


def test_eviction_writes_what_a_compaction_changed(kv):
    """Residency mode: blocks in the image count again from the prefix on."""
    pool = host_pool(kv, nb=10, lru=True)
    token = 2 * 2 * 4 * 128 * 2
    s, o = kv.session_create(pool, 160), kv.session_create(pool, 160)
    reserve(kv, pool, s, 100)                            # 7 blocks
    reserve(kv, pool, o, 160)                            # all of s leaves
    assert kv.kv_pool_get_stats(pool)["bytes_packed"] == 100 * token and kv.session_info(pool, s).num_blocks == 0
    kv.session_compact(pool, s, 256, 0, 0, 30, 40)       # comes back, 70 tokens of it stay
    assert kv.session_info(pool, s).tokens == 70 and kv.session_info(pool, s).num_blocks == 5
    packed = kv.kv_pool_get_stats(pool)["bytes_packed"]
    kv.kv_pool_batch_reserve_tokens(pool, [o], [0], None, 100, None)
    # 40 tokens of s were in the image and stay valid: the third block's 8 others, and all behind them
    assert kv.kv_pool_get_stats(pool)["bytes_packed"] - packed == 30 * token
    check(kv, pool, 10, True, 16)
    kv.kv_pool_destroy(pool)


@pytest.mark.parametrize("lru", [False, True])
def test_compact_keeps_its_blocks(kv, lru):
    pool = host_pool(kv, lru=lru)
    s = kv.session_create(pool, 400)
    reserve(kv, pool, s, 300)
    row = kv.session_block_table(pool, s)
    free = kv.kv_pool_free_list(pool)
    kv.session_compact(pool, s, 256, 0, 0, 90, 37)
    assert kv.session_info(pool, s).tokens == 127 and kv.session_block_table(pool, s) == row[:8]
    assert kv.kv_pool_free_list(pool) == free + row[8:][::-1]
    kv.session_compact(pool, s, 256, 0, 0, 90, 37)       # everything: nothing changes
    assert kv.session_block_table(pool, s) == row[:8]
    kv.session_compact(pool, s, None, 0, 0, 0, 37)       # nothing behind the prefix
    assert kv.session_info(pool, s).tokens == 37 and kv.session_block_table(pool, s) == row[:3]
    check(kv, pool, 60, lru, 16)
    kv.kv_pool_destroy(pool)


def test_compact_replaces_shared_blocks(kv):
    pool = host_pool(kv, nb=20)
    p = kv.session_create(pool, 200)
    reserve(kv, pool, p, 160)                            # 10
    k, = kv.session_fork(pool, p, 150, 200, 1)           # 9 shared, one its own
    row, mine = kv.session_block_table(pool, p), kv.session_block_table(pool, k)
    free = kv.kv_pool_free_list(pool)[::-1]              # 9
    kv.session_compact(pool, k, 256, 0, 0, 100, 20)      # blocks 1..7 are written: 7 new ones
    assert kv.session_block_table(pool, k) == row[:1] + free[:7]
    assert kv.session_block_table(pool, p) == row
    check(kv, pool, 20, False, 16)
    before = state(kv, pool)
    refused(kv, kv.KV_ERR_NO_HOT_BLOCKS, kv.session_compact, pool, kv.session_fork(pool, p, 160, 200, 1)[0], 256,
            0, 0, 100, 0)
    kv.session_destroy(pool, 2)
    assert state(kv, pool)[0] == before[0] and mine[9] in kv.kv_pool_free_list(pool)
    kv.kv_pool_destroy(pool)


def test_compact_refusals_change_nothing(kv):
    pool = host_pool(kv)
    s = kv.session_create(pool, 200)
    reserve(kv, pool, s, 100)
    before = state(kv, pool)
    for a in ((s, 256, 0, 0, -1, 0), (s, 256, 0, 0, 10, -1), (s, 256, 0, 0, 60, 41), (s, 256, -1, 0, 10, 0),
              (s, 256, 0, -4, 10, 0), (s, 256, 0, 0, 1, 2 ** 63 - 1), (s, 258, 0, 0, 10, 0), (5, 256, 0, 0, 10, 0), (s, 256, 1 << 41, 0, 10, 0)):
        refused(kv, kv.KV_ERR_INVALID_ARG, kv.session_compact, pool, *a)
        assert state(kv, pool) == before, a
    kv.session_pause(pool, s, None)
    refused(kv, kv.KV_ERR_BAD_STATE, kv.session_compact, pool, s, 256, 0, 0, 10, 0)
    kv.kv_pool_destroy(pool)


@pytest.mark.parametrize("lru", [False, True])
def test_failing_device_calls_change_nothing(kv, lru):
    pool = host_pool(kv, lru=lru)
    p = kv.session_create(pool, 300)
    reserve(kv, pool, p, 200)
    if not lru:
        kv.session_fork(pool, p, 192, 300, 1)
    calls = (lambda: kv.session_fork(pool, p, 150, 300, 2), lambda: kv.session_truncate(pool, p, 90),
             lambda: kv.session_compact(pool, p, 256, 0, 0, 50, 20))
    for f in calls:
        n = 0
        while True:
            before = state(kv, pool)
            kv.kv_pool_inject_cuda_failure(pool, n + 1)
            try:
                f()
                break
            except kv.KVError as e:
                assert e.code == kv.KV_ERR_CUDA
                assert state(kv, pool) == before
                check(kv, pool, 60, lru, 16)
            n += 1
        kv.kv_pool_inject_cuda_failure(pool, 0)
        assert n >= 1
        check(kv, pool, 60, lru, 16)
    kv.kv_pool_destroy(pool)


@pytest.mark.parametrize("lru", [False, True])
@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("how", ["compact", "truncate", "mixed"])
def test_sessions_that_grow_together_get_their_blocks_again(kv, lru, bt, how):
    """Several sessions give back blocks; one reservation for all, in any order, returns each one's."""
    pool = host_pool(kv, nb=40, lru=lru, bt=bt)
    n = [9 * bt + 3, 12 * bt, 7 * bt + 1]
    sids = [kv.session_create(pool, 1000) for _ in n]
    kv.kv_pool_batch_reserve_tokens(pool, sids, n, None, 1 << 20, None)
    rows, free = [kv.session_block_table(pool, s) for s in sids], kv.kv_pool_free_list(pool)
    for order in ((0, 1, 2), (2, 1, 0), (1, 2, 0), (0, 2, 1)):
        for i, s in enumerate(sids):
            if how == "truncate" or how == "mixed" and i == 1:
                kv.session_truncate(pool, s, 2 * bt + 5)
            else:
                kv.session_compact(pool, s, 256, 0, 0, 2 * bt, 5)
        kv.kv_pool_batch_reserve_tokens(pool, [sids[i] for i in order], [n[i] - 2 * bt - 5 for i in order], None, 1 << 20, None)
        assert [kv.session_block_table(pool, s) for s in sids] == rows and kv.kv_pool_free_list(pool) == free
        check(kv, pool, 40, lru, bt)
    kv.kv_pool_destroy(pool)


def test_blocks_that_were_given_back_go_by_the_free_list_else(kv):
    """A single session, sessions that gave nothing back, an ended one's id: the order of pops as it was."""
    pool = host_pool(kv)
    a, b = kv.session_create(pool, 400), kv.session_create(pool, 400)
    kv.kv_pool_batch_reserve_tokens(pool, [a, b], [96, 96], None, 1 << 20, None)
    rows = [kv.session_block_table(pool, s) for s in (a, b)]
    kv.session_truncate(pool, a, 48)
    kv.session_truncate(pool, b, 80)
    free = kv.kv_pool_free_list(pool)[::-1]
    assert free[:4] == rows[1][5:] + rows[0][3:]
    c, d = kv.session_create(pool, 400), kv.session_create(pool, 400)
    kv.kv_pool_batch_reserve_tokens(pool, [c, d], [16, 16], None, 1 << 20, None)
    assert [kv.session_block_table(pool, s) for s in (c, d)] == [free[0:1], free[1:2]]
    reserve(kv, pool, a, 32)
    assert kv.session_block_table(pool, a) == rows[0][:3] + free[2:4]
    kv.session_truncate(pool, a, 16)                     # four blocks with its mark
    kv.session_destroy(pool, a)
    assert kv.session_create(pool, 400) == a
    free = kv.kv_pool_free_list(pool)[::-1]
    kv.kv_pool_batch_reserve_tokens(pool, [b, a], [32, 32], None, 1 << 20, None)
    assert kv.session_block_table(pool, b)[5:] == free[:2] and kv.session_block_table(pool, a) == free[2:4]
    # fewer than were given back: what the free list has next, each one's own among it
    kv.session_truncate(pool, b, 64)
    kv.session_truncate(pool, a, 0)
    free = kv.kv_pool_free_list(pool)[::-1]
    mine = kv.session_block_table(pool, b)
    kv.kv_pool_batch_reserve_tokens(pool, [b, a, c], [1, 33, 16], None, 1 << 20, None)
    assert kv.session_block_table(pool, a)[:2] == free[:2] and kv.session_block_table(pool, b) == mine + [free[2]]
    check(kv, pool, 60, False, 16)
    kv.kv_pool_destroy(pool)


@pytest.mark.parametrize("lru", [False, True])
@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("seed", range(4))
def test_random_calls_keep_the_invariants(kv, lru, bt, seed):
    nb = 40 if bt == 16 else 14
    pool, r = host_pool(kv, nb=nb, lru=lru, bt=bt, sessions=10, cold=4500 * 4096 * 2), random.Random(seed)
    done = {}
    for _ in range(600):
        sids = live(kv, pool)
        op = r.choice(["create", "grow", "grow", "fork", "fork", "truncate", "compact", "pause", "resume", "destroy",
                       "append"])
        s = r.choice(sids) if sids and r.random() < 0.97 else r.randrange(-1, 11)
        before = state(kv, pool)
        try:
            if op == "create":
                kv.session_create(pool, r.randrange(1, 500))
            elif op == "grow":
                reserve(kv, pool, s, r.choice([0, 1, 5, bt, 70]))
            elif op == "append":
                kv.session_append(pool, s, 256, 256, r.choice([1, 20]))
            elif op == "fork":
                t = kv.session_info(pool, s).tokens
                kv.session_fork(pool, s, r.choice([t, t // 2, t // bt * bt, t + 1]), r.choice([t, 500]),
                                r.choice([1, 1, 2, 3]))
            elif op == "truncate":
                kv.session_truncate(pool, s, r.randrange(0, kv.session_info(pool, s).tokens + 2))
            elif op == "compact":
                t = kv.session_info(pool, s).tokens
                prefix = r.randrange(0, t + 1)
                kv.session_compact(pool, s, 256, 0, 0, r.randrange(0, t - prefix + 2), prefix)
            else:
                getattr(kv, f"session_{op}")(pool, s, *(() if op == "destroy" else (None,)))
            done[op] = done.get(op, 0) + 1
        except kv.KVError as e:
            assert e.code in (kv.KV_ERR_INVALID_ARG, kv.KV_ERR_BAD_STATE, kv.KV_ERR_NO_HOT_BLOCKS,
                              kv.KV_ERR_NO_COLD_SPACE)
            if not (lru and op == "compact"):            # (its blocks may have come back)
                assert state(kv, pool) == before, op
        check(kv, pool, nb, lru, bt)
    assert all(done.get(x, 0) > 5 for x in ("fork", "truncate", "compact", "pause", "resume"))
    kv.kv_pool_destroy(pool)
