"""Which of the pool's moves wait for which, without a GPU: the pool runtime over a stand-in for the CUDA runtime
(fake_streams.cpp) that notes launches, event records and waits. Each move's reads and writes of blocks' rows have to
come behind those that they would disturb, whatever streams they are on."""
import atexit
import ctypes as C
import functools
import os
import random
import shutil
import subprocess
import tempfile

import pytest

from test_pool_setup_host import CSRC, HERE, cuda_include

LAUNCH, RECORD, WAIT, HOST_WAIT = 1, 2, 3, 4
BT = 16


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
                    os.path.join(HERE, "fake_streams.cpp"), *(os.path.join(CSRC, x) for x in ("pool.cpp", "pages.cpp", "sparse.cpp")),
                    "-o", so], check=True)
    atexit.register(shutil.rmtree, d)
    return so


class Refused(Exception):
    pass


class Pool:
    """A simple-mode pool, what its moves read and write, and when: a clock per stream, which a wait brings up to what
    the event has seen."""

    def __init__(self, kv, path, nb=60, sessions=10, **more):
        x = self.x = C.CDLL(path)
        for name in set(kv.EXPORTS) - {"decode_attention_noalloc"}:      # (a file of its own)
            getattr(x, name).argtypes = getattr(kv.lib, name).argtypes
        x.fake_calls.argtypes, x.fake_calls.restype, x.fake_events.restype = [C.c_void_p, C.c_int64], C.c_int64, C.c_int64
        x.kv_last_error.restype = C.c_char_p
        cfg = kv.make_config(num_layers=2, num_hot_blocks=nb, max_sessions=sessions, max_batch=sessions, max_context=1024,
                             hot_base=1 << 20, cold_base=1 << 21, cold_bytes=1 << 30, block_tokens=BT, **more)
        self.kv, self.h = kv, C.c_void_p()
        assert x.kv_pool_create(C.byref(cfg), C.byref(self.h)) == kv.KV_OK
        self.clocks, self.events, self.host = {}, {}, {}
        self.past = {}                                   # block -> [(row from, to, writes, stream, tick, what)]
        self.grown = {}                                  # session -> the clock of its last reservation's writes
        self.moves = {}                                  # session -> the clock of all that read or wrote for it

    def call(self, name, *a):
        rc = getattr(self.x, name)(self.h, *a)
        self.replay()
        if rc:
            raise Refused(rc, self.x.kv_last_error())

    def info(self, sid):
        out = self.kv.kv_session_info()
        assert self.x.session_info(self.h, sid, C.byref(out)) == 0
        return out

    def row(self, sid):
        out, n = (C.c_int32 * 256)(), C.c_int32()
        assert self.x.session_block_table(self.h, sid, out, 256, C.byref(n)) == 0
        return list(out[:n.value])

    # order ----------------------------------------------------------------------------
    def clock(self, stream):
        return self.clocks.setdefault(stream, {})

    @staticmethod
    def merge(into, other):
        for s, t in other.items():
            into[s] = max(into.get(s, 0), t)

    def tick(self, stream):
        c = self.clock(stream)
        self.merge(c, self.host)
        c[stream] = c.get(stream, 0) + 1

    def replay(self):
        out = (C.c_int64 * 3000)()
        n = self.x.fake_calls(out, 1000)
        assert n <= 1000
        self.launches, self.first = 0, None              # the stream's clock behind the first launch
        self.waits = out[0:3 * n:3].count(WAIT)
        for what, stream, event in zip(out[0:3 * n:3], out[1:3 * n:3], out[2:3 * n:3]):
            if what == LAUNCH:
                self.tick(stream)
                self.launches += 1
                self.first = self.first or dict(self.clock(stream))
            elif what == RECORD:
                self.merge(self.clock(stream), self.host)
                self.events[event] = dict(self.clock(stream))
            elif what == WAIT:
                self.merge(self.clock(stream), self.events[event])
            else:
                self.merge(self.host, self.events[event])

    def synchronise(self):
        for c in self.clocks.values():
            self.merge(self.host, c)

    def touch(self, stream, sid, blocks, first, end, writes, what, clock=None):
        """Rows of a session's tokens [first, end), which lie in `blocks`, by the stream's newest launch (or that of `clock`)."""
        c = clock or self.clock(stream)
        self.merge(self.moves.setdefault(sid, {}), c)
        for j in range(first // BT, -(-end // BT)):
            lo, hi = max(first, j * BT) - j * BT, min(end, (j + 1) * BT) - j * BT
            past = self.past.setdefault(blocks[j], [])
            for l, h, w, s, t, other in past:
                if l < hi and lo < h and (w or writes):
                    assert c.get(s, 0) >= t, f"{what} on stream {stream} does not wait for {other} on stream {s}"
            past.append((lo, hi, writes, stream, c.get(stream, 0), what))

    def caller_orders(self, sid, stream):
        if sid in self.grown:
            self.merge(self.clock(stream), self.grown[sid])

    # the calls --------------------------------------------------------------------------
    def create(self, n=512):
        sid = C.c_int32()
        self.call("session_create", n, C.byref(sid))
        return sid.value

    def append(self, sid, n, st):
        T = self.info(sid).tokens
        self.call("session_append", sid, 256, 256, n, st)
        self.touch(st, sid, self.row(sid), T, T + n, True, f"append({sid})")

    def reserve(self, sids, n, st):
        """A reservation and, behind it on the stream, the kernel that writes the tokens."""
        T = [self.info(s).tokens for s in sids]
        B = len(sids)
        self.call("kv_pool_batch_reserve_tokens", (C.c_int32 * B)(*sids), (C.c_int32 * B)(*[n] * B), B, 256, 64, 256, st)
        self.tick(st)
        for s, t in zip(sids, T):
            self.touch(st, s, self.row(s), t, t + n, True, f"reserved tokens({s})")
            self.grown[s] = dict(self.clock(st))

    def pause(self, sid, st):
        self.caller_orders(sid, st)
        i, row = self.info(sid), self.row(sid)
        self.call("session_pause", sid, st)
        if i.tokens > i.cold_valid:
            self.touch(st, sid, row, i.cold_valid, i.tokens, False, f"pause({sid})")

    def resume(self, sid, st):
        self.call("session_resume", sid, st)
        self.touch(st, sid, self.row(sid), 0, self.info(sid).tokens, True, f"resume({sid})")

    def fork(self, sid, n, tokens, st):
        self.caller_orders(sid, st)
        out = (C.c_int32 * n)()
        self.call("session_fork", sid, tokens, 512, n, out, st)
        for k in out if tokens % BT else ():
            self.touch(st, sid, self.row(sid), tokens // BT * BT, tokens, False, f"fork of {sid}")
            self.touch(st, k, self.row(k), tokens // BT * BT, tokens, True, f"fork to {k}")
        return list(out)

    def truncate(self, sid, tokens, st):
        self.caller_orders(sid, st)
        old = self.row(sid)
        self.call("session_truncate", sid, tokens, st)
        row = self.row(sid)
        if row and row[-1] != old[len(row) - 1]:
            self.touch(st, sid, old, tokens // BT * BT, tokens, False, f"truncation of {sid}")
            self.touch(st, sid, row, tokens // BT * BT, tokens, True, f"truncation of {sid}")

    def compact(self, sid, n, prefix, st):
        self.caller_orders(sid, st)
        T, old = self.info(sid).tokens, self.row(sid)
        self.call("session_compact", sid, 256, 0, 0, n, prefix, st)
        if not n or prefix + n == T:
            return
        row = self.row(sid)
        first = prefix if row[prefix // BT] == old[prefix // BT] else prefix // BT * BT
        past, self.past = self.past, {b: list(x) for b, x in self.past.items()}
        self.touch(st, sid, old, first, T, False, f"compaction of {sid}")
        read, self.past = self.past, past
        self.touch(st, sid, row, first, prefix + n, True, f"compaction of {sid}")
        for b, x in read.items():                        # (its own reads and writes are one kernel's)
            self.past.setdefault(b, []).extend(y for y in x if y not in self.past[b])

    def destroy(self, sid):
        """The caller has waited for the session's own work, and for nothing else."""
        self.merge(self.host, self.moves.pop(sid, {}))
        self.grown.pop(sid, None)
        self.call("session_destroy", sid)


@pytest.fixture()
def pool(kv, tmp_path):
    """A pool runtime of the test's own: a copy of the library has its variables at their start."""
    return Pool(kv, shutil.copy(built(), tmp_path / "pool.so"))


A, B, G, H = 11, 22, 33, 44              # streams


def shared(pool, tokens=208):
    """A session and a fork that shares all of its blocks."""
    p = pool.create()
    pool.append(p, tokens, G)
    k, = pool.fork(p, 1, tokens, G)
    pool.synchronise()
    return p, k


@pytest.mark.parametrize("n,prefix", [(207, 0), (100, 0), (20, 187), (60, 70)])
def test_a_compaction_waits_for_a_former_holders_pause(pool, n, prefix):
    p, k = shared(pool)
    pool.pause(p, A)
    pool.compact(k, n, prefix, B)
    pool.append(k, 5, H)


@pytest.mark.parametrize("n,prefix", [(207, 0), (100, 0), (20, 187), (60, 70)])
def test_a_compaction_waits_for_a_former_holders_compaction(pool, n, prefix):
    p, k = shared(pool)
    pool.compact(p, 150, 10, A)
    pool.compact(k, n, prefix, B)
    pool.append(k, 5, H)


@pytest.mark.parametrize("grow", ["append", "reserve"])
@pytest.mark.parametrize("tokens", [200, 193, 100, 1])
@pytest.mark.parametrize("leave", ["pause", "compact", "truncate"])
def test_tokens_behind_a_cut_wait_for_a_former_holders_move(pool, leave, tokens, grow):
    p, k = shared(pool)
    if leave == "pause":
        pool.pause(p, A)
    elif leave == "compact":
        pool.compact(p, 150, 0, A)
    else:
        pool.truncate(p, tokens, A)
    pool.truncate(k, tokens, B)
    pool.append(k, 8, H) if grow == "append" else pool.reserve([k], 8, H)
    pool.append(k, 8, A)


@pytest.mark.parametrize("left", [1, 3])
def test_a_cut_that_gives_back_no_block_takes_no_fence(pool, left):
    """And the fence of who left stays on the block: who gets it after the session has ended waits for it."""
    p, k = shared(pool)
    pool.pause(p, A)
    made = pool.x.fake_events()
    for t in (206, 205, 204):
        pool.truncate(k, t, B)
        assert pool.waits > 0 and pool.launches == 0
    assert pool.x.fake_events() == made                  # (the ready event is the fork's)
    if left == 3:
        pool.truncate(k, 48, B)
    pool.destroy(k)
    o = pool.create(512)
    pool.append(o, 400, H)


def test_a_fork_of_a_block_that_was_shared(pool):
    """The fork reads a part of a block that a third session then writes."""
    p, k = shared(pool)
    f, = pool.fork(k, 1, 203, A)
    pool.pause(k, B)
    pool.truncate(p, 202, G)
    pool.append(p, 9, H)
    pool.append(f, 9, G)


def test_a_sessions_events_serve_the_next_one_of_its_id(pool):
    p = pool.create()
    pool.append(p, 100, G)

    def branches():
        for k in pool.fork(p, 3, 90, A):
            pool.append(k, 20, A)
            pool.destroy(k)
    branches()
    made = pool.x.fake_events()
    for _ in range(20):
        branches()
    assert pool.x.fake_events() == made
    assert pool.x.kv_pool_destroy(pool.h) == 0 and pool.x.fake_events() == 0


@pytest.mark.parametrize("call", ["fork", "truncate", "compact", "compact of shared blocks"])
def test_calls_that_cannot_have_an_event_launch_nothing(pool, call):
    p = pool.create()
    pool.append(p, 200, G)
    other = pool.create()
    pool.append(other, 200, G)
    if call != "compact":
        f, = pool.fork(other, 1, 200, G)
        g, = pool.fork(f, 1, 192, G)                     # 12 shared blocks; its events are made anew below
        pool.destroy(f)
        p = g if call != "fork" else p
    calls = {"fork": lambda: pool.call("session_fork", p, 150, 512, 2, (C.c_int32 * 2)(), A),
             "truncate": lambda: pool.call("session_truncate", p, 100, A)}
    f = calls.get(call, lambda: pool.call("session_compact", p, 256, 0, 0, 100, 20, A))
    failed = 0
    while True:
        before = [pool.info(s).tokens for s in (p, other)], pool.row(p), pool.row(other)
        pool.x.fake_fail_create(failed + 1)
        try:
            f()
            break
        except Refused as e:
            assert e.args[0] == pool.kv.KV_ERR_CUDA and b"EventCreate" in e.args[1]
            assert pool.launches == 0
            assert ([pool.info(s).tokens for s in (p, other)], pool.row(p), pool.row(other)) == before
        failed += 1
    pool.x.fake_fail_create(0)
    assert failed >= 1 and pool.launches >= 1


@pytest.mark.parametrize("call", ["select", "attend", "append"])
def test_a_failing_call_is_told_of_once(pool, call):
    """The runtime's last error is gone: a launch that asks for it finds its own."""
    p = pool.create()
    calls = {"select": lambda: pool.call("select_blocks", 0, 256, 0, 256, 256, 256, 1, 4, 1, 1, 2, 256, None, A),
             "attend": lambda: pool.call("sparse_attention", 0, 256, 0, None, None, 0, 256, 2, 256, 256, 1, 4, 1.0, 256, 0, A),
             "append": lambda: pool.append(p, 5, A)}
    no_resources = 101
    pool.x.fake_prepare_status(no_resources)
    pool.x.fake_fail_create(1)
    with pytest.raises(Refused) as e:
        calls[call]()
    assert e.value.args[0] == pool.kv.KV_ERR_CUDA and pool.launches == 0 and pool.x.fake_last_error() == 0
    pool.x.fake_prepare_status(0)
    pool.x.fake_fail_create(0)
    calls[call]()                                        # and it may go on
    assert pool.launches >= 1


def test_a_new_session_waits_for_nothing_of_its_ids_last_one(pool):
    p = pool.create()
    pool.append(p, 30, G)
    k, = pool.fork(p, 1, 20, A)
    pool.append(k, 5, A)
    pool.destroy(k)
    assert pool.create() == k
    ev = C.c_void_p(1)
    assert pool.x.session_ready_event(pool.h, k, C.byref(ev)) == 0 and ev.value is None
    pool.append(k, 5, B)
    assert pool.waits == 0


@pytest.mark.parametrize("seed", range(12))
def test_random_moves_on_several_streams(pool, seed):
    r = random.Random(seed)
    live, done = {}, {}                                  # session -> the stream that it grows on
    for step in range(700):
        st, op = r.choice([A, B, G, H]), r.choice(["create", "append", "append", "reserve", "pause", "resume", "fork", "fork",
                                                   "truncate", "truncate", "compact", "destroy"])
        sid = r.choice(list(live)) if live else None
        try:
            if op == "create" or sid is None:
                live[pool.create()] = r.choice([A, B, G, H])
            elif op == "append":
                pool.append(sid, r.choice([1, 7, 16, 60]), live[sid])
            elif op == "reserve":
                pool.reserve([s for s in live if live[s] == live[sid] and (s == sid or r.random() < 0.5)], r.choice([1, 20]), live[sid])
            elif op in ("pause", "resume"):
                getattr(pool, op)(sid, st)
            elif op == "fork":
                T = pool.info(sid).tokens
                for k in pool.fork(sid, r.choice([1, 2]), r.choice([T, T // BT * BT, r.randrange(T + 1)]), st):
                    live[k] = r.choice([A, B, G, H])
            elif op == "truncate":
                T = pool.info(sid).tokens
                pool.truncate(sid, max(0, T - r.choice([1, 5, 9, 30, 200])), st)
            elif op == "compact":
                T = pool.info(sid).tokens
                prefix = r.randrange(T + 1)
                pool.compact(sid, r.choice([T - prefix, max(0, T - prefix - 1), r.randrange(T - prefix + 1)]), prefix, st)
            elif r.random() < 0.5:
                pool.destroy(sid)
                del live[sid]
            done[op] = done.get(op, 0) + 1
        except Refused:                                  # full, or in another state
            pass
    assert all(done.get(x, 0) > 5 for x in ("append", "reserve", "pause", "resume", "fork", "truncate", "compact"))


# ---- residency mode -----------------------------------------------------------------------

class Resident(Pool):
    """A pool that evicts. Evictions and fetches of a call show in the sessions' tables; the model knows what each
    image holds. An allocating call is ordered by its caller behind reservations and what they write, as the header
    says."""

    def __init__(self, kv, path, **more):
        super().__init__(kv, path, flags=kv.KV_POOL_LRU_RESIDENCY, **more)
        self.image = {}                                  # session -> tokens of each block that its image holds
        self.appended = {}                               # session -> the clock of its last append

    def tokens_in(self, T, j):
        return max(0, min(BT, T - j * BT))

    def behind_reservations(self, st):
        for c in self.grown.values():
            self.merge(self.clock(st), c)

    def moved(self, st, f, skip=()):
        """Runs a call; notes its evictions and fetches."""
        old = {s: (self.row(s), self.info(s).tokens) for s in self.image}
        f()                                              # (evictions are its first launch)
        for s, (row, T) in old.items():
            now = self.row(s)
            for j, (a, b) in enumerate(zip(row, now)):
                if a >= 0 and b < 0:                     # out
                    n = self.tokens_in(T, j)
                    if n > self.image[s][j]:
                        at = (self.image[s][j], n)
                        self.touch(st, s, {0: a}, *at, False, f"eviction of {s}", self.first)
                        self.touch(st, s, {0: ("image", s, j)}, *at, True, f"eviction of {s}", self.first)
                        self.image[s][j] = n
        for s, (row, T) in old.items():
            now = self.row(s)
            for j, (a, b) in enumerate(zip(row, now)):
                if a < 0 and b >= 0 and s not in skip:   # back
                    n = self.tokens_in(T, j)
                    self.touch(st, s, {0: ("image", s, j)}, 0, n, False, f"fetch of {s}")
                    self.touch(st, s, {0: b}, 0, n, True, f"fetch of {s}")

    def shape(self, sid, T):
        im = self.image[sid]
        n = -(-T // BT)
        self.image[sid] = [min(x, self.tokens_in(T, j)) for j, x in enumerate(im[:n])] + [0] * (n - len(im))

    def create(self, n=512):
        sid = super().create(n)
        self.image[sid] = []
        return sid

    def append(self, sid, n, st):
        self.behind_reservations(st)
        T = self.info(sid).tokens
        self.moved(st, lambda: self.call("session_append", sid, 256, 256, n, st))
        self.touch(st, sid, self.row(sid), T, T + n, True, f"append({sid})")
        self.appended[sid] = dict(self.clock(st))
        self.shape(sid, T + n)

    def reserve(self, sids, n, st):
        self.behind_reservations(st)
        T = [self.info(s).tokens for s in sids]
        B = len(sids)
        self.moved(st, lambda: self.call("kv_pool_batch_reserve_tokens", (C.c_int32 * B)(*sids), (C.c_int32 * B)(*[n] * B), B, 256,
                                         64, 256, st))
        self.tick(st)
        for s, t in zip(sids, T):
            self.touch(st, s, self.row(s), t, t + n, True, f"reserved tokens({s})")
            self.grown[s] = dict(self.clock(st))
            self.shape(s, t + n)

    def pause(self, sid, st):
        self.call("session_pause", sid, st)

    def resume(self, sid, st):
        self.behind_reservations(st)
        self.moved(st, lambda: self.call("session_resume", sid, st))

    def prefetch(self, sids, st):
        self.behind_reservations(st)
        a = (C.c_int32 * len(sids))(*sids)
        self.moved(st, lambda: self.call("kv_pool_prefetch", a, len(sids), None, 0, st))

    def tables(self, sids, st):
        """A batch's tables and, behind them on the stream, a kernel that reads its tokens. (Appends are the caller's to
        come behind.)"""
        self.behind_reservations(st)
        for s in sids:
            self.merge(self.clock(st), self.appended.get(s, {}))
        a = (C.c_int32 * len(sids))(*sids)
        self.moved(st, lambda: self.call("kv_pool_batch_tables", a, len(sids), 256, 64, 256, st))
        self.tick(st)
        for s in sids:
            self.touch(st, s, self.row(s), 0, self.info(s).tokens, False, f"decode of {s}")
            self.grown[s] = dict(self.clock(st))

    def fork(self, sid, n, tokens, st):
        self.behind_reservations(st)
        out, row = (C.c_int32 * n)(), self.row(sid)
        self.moved(st, lambda: self.call("session_fork", sid, tokens, 512, n, out, st))
        for k in out:
            self.image[k] = [0] * -(-tokens // BT)
            for j in range(-(-tokens // BT)):
                rows = self.tokens_in(tokens, j)
                self.touch(st, sid, {0: row[j] if row[j] >= 0 else ("image", sid, j)}, 0, rows, False, f"fork of {sid}")
                self.touch(st, k, {0: self.row(k)[j]}, 0, rows, True, f"fork to {k}")
        return list(out)

    def truncate(self, sid, tokens, st):
        self.caller_orders(sid, st)
        self.call("session_truncate", sid, tokens, st)
        self.shape(sid, tokens)

    def compact(self, sid, n, prefix, st):
        self.behind_reservations(st)
        T = self.info(sid).tokens
        self.moved(st, lambda: self.call("session_compact", sid, 256, 0, 0, n, prefix, st))
        if n and prefix + n < T:
            self.touch(st, sid, self.row(sid), prefix, prefix + n, True, f"compaction of {sid}")
            self.shape(sid, prefix)
        self.shape(sid, prefix + n)

    def destroy(self, sid):
        self.truncate(sid, 0, B)                         # its blocks may be others' next, behind a fence
        super().destroy(sid)
        del self.image[sid]
        self.appended.pop(sid, None)
        self.past = {b: x for b, x in self.past.items() if not (isinstance(b, tuple) and b[1] == sid)}


@pytest.fixture()
def resident(kv, tmp_path):
    return Resident(kv, shutil.copy(built(), tmp_path / "pool.so"), nb=40)


@pytest.mark.parametrize("back", ["prefetch", "resume"])
def test_a_batchs_tables_wait_for_what_is_being_fetched(resident, back):
    pool = resident
    p, o = out_and_back(pool)
    pool.synchronise()
    pool.append(o, 16 * 17, G)                           # 9 of p's leave again
    assert pool.row(p)[:9] == [-1] * 9
    pool.truncate(o, 16, G)
    pool.synchronise()
    if back == "prefetch":
        pool.prefetch([p], A)
    else:
        pool.pause(p, A)
        pool.resume(p, A)
    pool.tables([p], B)


def out_and_back(pool):
    """A session whose first ten blocks had left and came back on stream A, and one of 20 blocks."""
    p, o = pool.create(), pool.create(1024)
    pool.append(p, 16 * 12, G)
    pool.append(o, 16 * 38, G)                           # 40 blocks: p's first ten leave
    pool.pause(p, G)
    pool.truncate(o, 16 * 20, G)
    pool.synchronise()
    pool.resume(p, A)
    return p, o


@pytest.mark.parametrize("then", ["compact", "fork", "append", "reserve", "evict"])
def test_a_second_resume_still_stands_for_the_first_ones_fetches(resident, then):
    pool = resident
    p, o = out_and_back(pool)
    pool.truncate(p, 16 * 11 + 9, B)
    pool.pause(p, B)
    pool.resume(p, B)                                    # nothing is missing: its event alone
    if then == "compact":
        pool.compact(p, 150, 5, H)
    elif then == "fork":
        pool.fork(p, 1, 100, H)
    elif then == "evict":
        pool.append(o, 16 * 18, H)
    elif then == "append":
        pool.truncate(p, 100, B)                         # into a block that was fetched
        pool.append(p, 7, H)
    else:
        pool.truncate(p, 100, B)
        pool.reserve([p], 7, H)


@pytest.mark.parametrize("seed", [*range(12), 126, 129])
def test_random_moves_on_several_streams_in_residency_mode(resident, seed):
    r, pool = random.Random(seed), resident
    live, done = {}, {}
    for step in range(700):
        st, op = r.choice([A, B, G, H]), r.choice(["create", "append", "append", "append", "reserve", "pause", "resume", "fork",
                                                   "truncate", "truncate", "compact", "compact", "prefetch", "tables", "destroy"])
        sid = r.choice(list(live)) if live else None
        try:
            if op == "create" or sid is None:
                live[pool.create()] = r.choice([A, B, G, H])
            elif op == "append":
                pool.append(sid, r.choice([1, 7, 16, 60, 100]), live[sid])
            elif op == "reserve":
                pool.reserve([sid], r.choice([1, 20]), live[sid])
            elif op in ("pause", "resume"):
                getattr(pool, op)(sid, st)
            elif op in ("prefetch", "tables"):
                getattr(pool, op)([sid], st)
            elif op == "fork":
                T = pool.info(sid).tokens
                for k in pool.fork(sid, r.choice([1, 2]), r.choice([T, T // BT * BT, r.randrange(T + 1)]), st):
                    live[k] = r.choice([A, B, G, H])
            elif op == "truncate":
                T = pool.info(sid).tokens
                pool.truncate(sid, max(0, T - r.choice([1, 5, 9, 30, 200])), st)
            elif op == "compact":
                T = pool.info(sid).tokens
                prefix = r.randrange(T + 1)
                pool.compact(sid, r.choice([T - prefix, max(0, T - prefix - 1), r.randrange(T - prefix + 1)]), prefix, st)
            elif r.random() < 0.5:
                pool.destroy(sid)
                del live[sid]
            done[op] = done.get(op, 0) + 1
        except Refused:                                  # full, or in another state
            pass
    assert all(done.get(x, 0) > 2 for x in ("append", "reserve", "pause", "resume", "fork", "truncate", "compact", "prefetch", "tables"))
