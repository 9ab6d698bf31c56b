// The pool's host state, and what the files that implement the C ABI share: pool.cpp (pools, sessions,
// migrations, decode, prompts), pages.cpp (forks, truncation, compaction) and sparse.cpp (block bounds,
// selection, attention over selected blocks).
#pragma once

#include <algorithm>
#include <cstring>
#include <map>
#include <set>
#include <string>
#include <utility>
#include <vector>

#include "../../include/kvtier.h"
#include "kvt_internal.h"

namespace kvt {

// Notes the message that kv_last_error() returns on this thread; returns `code`.
int fail(int code, const std::string &msg);

struct Session {
    int32_t state = KV_SESSION_FREE;
    int64_t T = 0, cap = 0, cold_valid = 0;
    int64_t img_off = -1, img_bytes = 0;
    uint64_t home = 0;                // its mark on blocks that it gave back (kv_pool::block_home), 0 = on none
    std::vector<int32_t> blocks;      // per logical block: hot slot, or -1 (residency mode)
    std::vector<int16_t> img_tok;     // residency mode: tokens of block j held by the image
    int64_t hot_count = 0;            // residency mode: blocks with a hot slot
    uint64_t last_use = 0;            // residency mode: recency stamp
    cudaEvent_t ready = nullptr;      // behind the last resume, fetch or move of its rows (pages.cpp); who records it
    bool ready_recorded = false;      // again waits for it first, so that it covers those before as well
    cudaEvent_t appended = nullptr;
    bool appended_recorded = false;
    cudaEvent_t packed = nullptr;     // residency mode: after the last eviction that wrote
    bool packed_recorded = false;     // the image (it covers every earlier one)
    int16_t pack_fence = -1;          // simple mode: fence slot and generation of the
    uint64_t pack_gen = 0;            // last pause's pack (it reads the table row)

    // Nobody's again. Its events stay, for the next session of this id.
    void reset() {
        Session fresh;
        fresh.ready = ready;
        fresh.appended = appended;
        fresh.packed = packed;
        *this = std::move(fresh);
    }
};

// A planned eviction: block j of session sid leaves hot slot `slot`; tokens
// [t0, t1) are written to the image first (t0 == t1: the image has them).
struct Victim {
    int32_t sid, j, slot, t0, t1;
};

constexpr int kFenceSlots = 64;
struct Fence {
    cudaEvent_t ev = nullptr;
    uint64_t gen = 0;
};

class DeviceGuard {
  public:
    DeviceGuard(int dev, bool active) : active_(active) {
        if (active_ && cudaGetDevice(&prev_) == cudaSuccess && prev_ != dev) cudaSetDevice(dev);
        else prev_ = -1;
    }
    ~DeviceGuard() {
        if (active_ && prev_ >= 0) cudaSetDevice(prev_);
    }

  private:
    bool active_;
    int prev_ = -1;
};

}  // namespace kvt

struct kv_pool {
    kv_pool_config cfg{};
    bool host_only = false;
    int64_t block_bytes = 0, token_bytes = 0;
    int64_t image_token_bytes = 0;       // of a token in a cold image
    bool int8 = false;                   // KV_POOL_COLD_INT8
    int32_t table_stride = 0;            // max blocks per session
    int32_t max_splits = 0;              // split bound for max_context
    int64_t part_rows = 0;               // decode workspace capacity (partial rows)
    int64_t part_alloc = 0;              // partial rows allocated (at least part_rows)
    int num_sms = 1;
    int mig_ctas = 0;                    // cap on migration-kernel CTAs, 0 = none
    // Stream of the last decode call: moves on another one may run beside
    // decode. Compared only, and only to size a grid.
    bool decoded = false;
    cudaStream_t decode_stream = nullptr;
    kvt::Shape shape{};

    std::vector<int32_t> free_list;      // top = back
    std::vector<int16_t> block_fence;    // fence slot of the pack that freed it, or -1
    std::vector<uint64_t> block_fence_gen;
    // Simple mode: sessions that hold a block beside its first one. Forks share full blocks; a shared block
    // is only read, and goes back to the free list with its last session. The session that stays with it may write
    // it again behind the moves of those that left (live_fence).
    std::vector<int32_t> block_extra;
    bool forked = false;                 // some block has been shared
    std::vector<uint64_t> block_home;    // of a free block: Session::home of who gave it back, 0 = nobody's
    uint64_t homes = 0;                  // the last one of these marks
    std::vector<kvt::Session> sessions;
    std::map<int64_t, int64_t> cold_free;  // offset -> bytes
    int64_t cold_used = 0;

    void *d_slab = nullptr;              // the allocation behind the pointers below
    int32_t *d_tables = nullptr;
    float *d_part_o = nullptr;
    float *d_part_ml = nullptr;
    int32_t *d_counters = nullptr;       // split arrivals per (layer-batch row, kv-head)
    int64_t counter_count = 0;
    int32_t *d_err = nullptr;
    CUtensorMap tmap{};
    bool select_ready = false;           // the kernels of select_blocks
    bool sparse_ready = false;           // and of sparse_attention
    kvt::SelectFit select_fit{};
    kvt::SparseFit sparse_fit{};
    // prefill_attention and tree_attention (turn_setup)
    bool turn_ready = false;             // the kernel and the maps
    CUtensorMap turn_maps[2]{};
    float *d_turn_part = nullptr;        // partial results

    kvt::Fence fences[kvt::kFenceSlots];
    int next_fence = 0;
    uint64_t fence_gen = 0;

    kv_pool_stats stats{};
    int32_t inject_countdown = 0;
    bool inject_timeout = false;   // kv_pool_inject_decode_timeout, next attention call only

    // Residency mode (KV_POOL_LRU_RESIDENCY): sessions holding hot blocks,
    // ordered by (last use, sid); the first one is the least recently used.
    bool lru = false;
    uint64_t clock = 0;
    std::set<std::pair<uint64_t, int32_t>> lru_set;

    // Every CUDA call of the pool goes through here: the failure-injection
    // hook fires first, then (unless the pool is host-logic only) the call. A failing call is
    // told of once, here.
    template <typename F>
    int cuda(const char *what, F &&fn) {
        if (inject_countdown > 0 && --inject_countdown == 0)
            return kvt::fail(KV_ERR_CUDA, std::string(what) + ": injected CUDA failure");
        if (host_only) return KV_OK;
        cudaError_t e = fn();
        if (e != cudaSuccess) {
            cudaGetLastError();   // a later launch asks for its own
            return kvt::fail(KV_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
        }
        return KV_OK;
    }

    bool beside_decode(cudaStream_t st) const { return decoded && st != decode_stream; }
    int move_ctas(cudaStream_t st) const {
        return kvt::migration_ctas(mig_ctas, beside_decode(st), num_sms);
    }

    kvt::Session *session(int32_t sid) {
        if (sid < 0 || sid >= static_cast<int32_t>(sessions.size())) return nullptr;
        kvt::Session &s = sessions[sid];
        return s.state == KV_SESSION_FREE ? nullptr : &s;
    }

    int64_t image_bytes(int64_t cap) const {
        return (cap * image_token_bytes + 255) / 256 * 256;
    }

    bool cold_alloc(int64_t bytes, int64_t *off) {
        for (auto it = cold_free.begin(); it != cold_free.end(); ++it) {
            if (it->second >= bytes) {
                *off = it->first;
                const int64_t rest = it->second - bytes;
                const int64_t at = it->first + bytes;
                cold_free.erase(it);
                if (rest > 0) cold_free[at] = rest;
                cold_used += bytes;
                return true;
            }
        }
        return false;
    }

    void cold_release(int64_t off, int64_t bytes) {
        cold_used -= bytes;
        auto it = cold_free.emplace(off, bytes).first;
        auto nx = std::next(it);
        if (nx != cold_free.end() && it->first + it->second == nx->first) {
            it->second += nx->second;
            cold_free.erase(nx);
        }
        if (it != cold_free.begin()) {
            auto pv = std::prev(it);
            if (pv->first + pv->second == it->first) {
                pv->second += it->second;
                cold_free.erase(it);
            }
        }
    }

    // Whether a move of a session that left the block may still be running.
    bool live_fence(int32_t block) const {
        const int f = block_fence[block];
        return f >= 0 && fences[f].gen == block_fence_gen[block];
    }

    // Blocks popped for a session, or that it alone holds now and is about to write: make `st` wait for the moves of
    // the sessions that left them, if those may still be running.
    int wait_fences(const int32_t *blocks, size_t n, cudaStream_t st) {
        bool need[kvt::kFenceSlots] = {};
        for (size_t i = 0; i < n; ++i) {
            if (live_fence(blocks[i])) need[block_fence[blocks[i]]] = true;
        }
        for (int f = 0; f < kvt::kFenceSlots; ++f) {
            if (!need[f]) continue;
            int rc = cuda("cudaStreamWaitEvent", [&] { return cudaStreamWaitEvent(st, fences[f].ev, 0); });
            if (rc) return rc;
        }
        return KV_OK;
    }

    // A session gives up its hold on a block; true: nobody holds it any more.
    bool release(int32_t block) {
        if (block_extra[block] == 0) return true;
        --block_extra[block];
        return false;
    }

    // The fence slot for work that is about to be enqueued on blocks which leave a session. What the slot
    // marked before has to be complete; `st` waits for other sessions' moves of the same blocks, so that the
    // fence covers them too.
    int open_fence(const int32_t *blocks, size_t n, cudaStream_t st, int *slot) {
        const int f = *slot = next_fence;
        int rc = KV_OK;
        if (!fences[f].ev && !host_only)
            rc = cuda("cudaEventCreate",
                      [&] { return cudaEventCreateWithFlags(&fences[f].ev, cudaEventDisableTiming); });
        if (!rc && fences[f].gen != 0)
            rc = cuda("cudaEventSynchronize", [&] { return cudaEventSynchronize(fences[f].ev); });
        if (!rc && forked) rc = wait_fences(blocks, n, st);
        return rc;
    }

    int record_fence(int slot, cudaStream_t st) {
        return cuda("cudaEventRecord", [&] { return cudaEventRecord(fences[slot].ev, st); });
    }

    // Host side of a fence that has been recorded: its generation.
    uint64_t commit_fence(int slot) {
        next_fence = (slot + 1) % kvt::kFenceSlots;
        fences[slot].gen = ++fence_gen;
        return fence_gen;
    }

    // A block leaves a session behind the fence; true: it went back to the free list.
    bool give_back(int32_t block, int slot, uint64_t gen) {
        block_fence[block] = static_cast<int16_t>(slot);
        block_fence_gen[block] = gen;
        if (!release(block)) return false;
        free_list.push_back(block);
        stats.free_blocks += 1;
        stats.used_blocks -= 1;
        return true;
    }

    // Blocks have been popped: what the free list knew of them is over.
    void clear_fences(const int32_t *blocks, size_t n) {
        for (size_t i = 0; i < n; ++i) {
            block_fence[blocks[i]] = -1;
            block_home[blocks[i]] = 0;
        }
    }

    // Write entries [from, from+n) of a session's device table row.
    int write_table(int32_t sid, const int32_t *vals, int64_t from, int64_t n, cudaStream_t st) {
        for (int64_t i = 0; i < n; i += kvt::kTableWriteMax) {
            kvt::TableWriteArgs a;
            a.dst = d_tables + static_cast<int64_t>(sid) * table_stride + from + i;
            a.n = static_cast<int32_t>(std::min<int64_t>(kvt::kTableWriteMax, n - i));
            std::memcpy(a.vals, vals + i, sizeof(int32_t) * a.n);
            int rc = cuda("table write launch", [&] { return kvt::launch_table_write(a, st); });
            if (rc) return rc;
        }
        return KV_OK;
    }

    // Write n tokens at position s.T; the row gains blocks vals[0 .. fresh_n)
    // at entry `from`, in the same launch where they fit its parameters.
    int append_device(int32_t sid, const kvt::Session &s, const void *k, const void *v, int32_t n,
                      const int32_t *vals, int64_t from, int64_t fresh_n, cudaStream_t st) {
        kvt::AppendInlineArgs r;
        kvt::AppendArgs &a = r.m;
        a.k = static_cast<const uint8_t *>(k);
        a.v = static_cast<const uint8_t *>(v);
        a.table = d_tables + static_cast<int64_t>(sid) * table_stride;
        a.hot = static_cast<uint8_t *>(cfg.hot_base);
        a.pos0 = static_cast<int32_t>(s.T);
        a.n = n;
        a.err = d_err;
        a.s = shape;
        // the caller's bound is for migrations alone
        const int ctas = kvt::migration_ctas(0, beside_decode(st), num_sms);
        if (fresh_n > 0 && fresh_n <= kvt::kResumeInlineMax) {
            r.from = static_cast<int32_t>(from);
            r.n = static_cast<int32_t>(fresh_n);
            std::memcpy(r.blocks, vals, sizeof(int32_t) * fresh_n);
            return cuda("append launch", [&] { return kvt::launch_append_inline(r, ctas, st); });
        }
        int rc = fresh_n > 0 ? write_table(sid, vals, from, fresh_n, st) : KV_OK;
        if (!rc) rc = cuda("append launch", [&] { return kvt::launch_append(a, ctas, st); });
        return rc;
    }

    // ---- residency mode -------------------------------------------------
    int32_t tokens_in_block(const kvt::Session &s, int64_t j) const {
        const int64_t n = s.T - j * cfg.block_tokens;
        return static_cast<int32_t>(n < cfg.block_tokens ? n : cfg.block_tokens);
    }

    void lru_out(int32_t sid) {
        kvt::Session &s = sessions[sid];
        if (s.hot_count > 0) lru_set.erase({s.last_use, sid});
    }
    void lru_in(int32_t sid) {
        kvt::Session &s = sessions[sid];
        if (s.hot_count > 0) lru_set.insert({s.last_use, sid});
    }

    // Least recently used hot blocks, outside `protect`, until `need` blocks
    // would be free. Sessions in recency order; within one, ascending j.
    bool plan_evict(int64_t need, const std::vector<int32_t> &protect, std::vector<kvt::Victim> &out) {
        int64_t have = static_cast<int64_t>(free_list.size());
        for (const auto &e : lru_set) {
            if (have >= need) break;
            const int32_t sid = e.second;
            if (std::find(protect.begin(), protect.end(), sid) != protect.end()) continue;
            const kvt::Session &s = sessions[sid];
            for (size_t j = 0; j < s.blocks.size() && have < need; ++j) {
                if (s.blocks[j] < 0) continue;
                out.push_back({sid, static_cast<int32_t>(j), s.blocks[j], s.img_tok[j],
                               tokens_in_block(s, static_cast<int64_t>(j))});
                ++have;
            }
        }
        return have >= need;
    }

    // The `need` slots the call will pop once the victims are pushed back:
    // the free list grows by the victims (in order), pops come off its end.
    std::vector<int32_t> peek_alloc(int64_t need, const std::vector<kvt::Victim> &v) const {
        std::vector<int32_t> all(free_list);
        for (const kvt::Victim &x : v) all.push_back(x.slot);
        std::vector<int32_t> out(need);
        for (int64_t i = 0; i < need; ++i) out[i] = all[all.size() - 1 - i];
        return out;
    }

    // Device side of the victims: wait for their last writes, then write the
    // tokens each image lacks. A session whose image this writes records its
    // `packed` event after the writes; the stream first waits for the previous
    // recording, so the event covers every eviction of the session so far.
    // Whatever later fetches the session's blocks back waits on it
    // (wait_packed), on whichever stream it runs.
    int evict_device(const std::vector<kvt::Victim> &v, cudaStream_t st) {
        std::vector<int32_t> seen, writes;
        for (const kvt::Victim &x : v) {
            if (x.t1 > x.t0 && std::find(writes.begin(), writes.end(), x.sid) == writes.end())
                writes.push_back(x.sid);
            if (std::find(seen.begin(), seen.end(), x.sid) != seen.end()) continue;
            seen.push_back(x.sid);
            kvt::Session &s = sessions[x.sid];
            int rc = KV_OK;
            if (s.appended_recorded)
                rc = cuda("cudaStreamWaitEvent", [&] { return cudaStreamWaitEvent(st, s.appended, 0); });
            if (!rc && s.ready_recorded)
                rc = cuda("cudaStreamWaitEvent", [&] { return cudaStreamWaitEvent(st, s.ready, 0); });
            if (!rc) rc = wait_packed(x.sid, st);
            if (rc) return rc;
        }
        std::vector<kvt::BlockJob> jobs;
        for (const kvt::Victim &x : v)
            if (x.t1 > x.t0) jobs.push_back(job_for(x.sid, x.j, x.slot, x.t0, x.t1));
        int rc = run_jobs(jobs, true, st);
        for (size_t i = 0; !rc && !host_only && i < writes.size(); ++i) {
            kvt::Session &s = sessions[writes[i]];
            if (!s.packed)
                rc = cuda("cudaEventCreate",
                          [&] { return cudaEventCreateWithFlags(&s.packed, cudaEventDisableTiming); });
            if (!rc) rc = cuda("cudaEventRecord", [&] { return cudaEventRecord(s.packed, st); });
        }
        if (rc) return rc;
        for (int32_t sid : writes) sessions[sid].packed_recorded = !host_only;
        return KV_OK;
    }

    // Before blocks of `sid` are fetched from its image on `st`: the image
    // writes of its evictions (possibly on another stream) must be complete.
    int wait_packed(int32_t sid, cudaStream_t st) {
        const kvt::Session &s = sessions[sid];
        if (!s.packed_recorded) return KV_OK;
        return cuda("cudaStreamWaitEvent", [&] { return cudaStreamWaitEvent(st, s.packed, 0); });
    }

    void evict_commit(const std::vector<kvt::Victim> &v) {
        for (const kvt::Victim &x : v) {
            kvt::Session &s = sessions[x.sid];
            lru_out(x.sid);
            if (x.t1 > x.t0) stats.bytes_packed += static_cast<int64_t>(x.t1 - x.t0) * image_token_bytes;
            s.img_tok[x.j] = static_cast<int16_t>(x.t1);
            s.blocks[x.j] = -1;
            s.hot_count -= 1;
            lru_in(x.sid);
            free_list.push_back(x.slot);
            stats.blocks_evicted += 1;
            stats.free_blocks += 1;
            stats.used_blocks -= 1;
        }
    }

    kvt::BlockJob job_for(int32_t sid, int32_t j, int32_t slot, int32_t t0, int32_t t1) const {
        const kvt::Session &s = sessions[sid];
        kvt::BlockJob b;
        b.img = static_cast<uint8_t *>(cfg.cold_base) + s.img_off;
        b.T_cap = static_cast<int32_t>(s.cap);
        b.sid = -1;
        b.slot = slot;
        b.j = j;
        b.t0 = t0;
        b.t1 = t1;
        return b;
    }

    // A fetch of block j into `slot`: the copy also writes the session's
    // device table entry j.
    kvt::BlockJob fetch_job(int32_t sid, int32_t j, int32_t slot, int32_t t0, int32_t t1) const {
        kvt::BlockJob b = job_for(sid, j, slot, t0, t1);
        b.sid = sid;
        return b;
    }

    int run_jobs(const std::vector<kvt::BlockJob> &jobs, bool pack, cudaStream_t st) {
        for (size_t i = 0; i < jobs.size(); i += kvt::kBlockJobsMax) {
            kvt::BlockJobs a;
            a.hot = static_cast<uint8_t *>(cfg.hot_base);
            a.err = d_err;
            a.tables = d_tables;
            a.table_stride = table_stride;
            a.s = shape;
            a.n = static_cast<int32_t>(std::min<size_t>(kvt::kBlockJobsMax, jobs.size() - i));
            a.once = 0;
            a.int8 = int8;
            std::copy(jobs.begin() + i, jobs.begin() + i + a.n, a.job);
            int rc = cuda(pack ? "pack launch" : "unpack launch",
                          [&] { return kvt::launch_block_jobs(a, pack, move_ctas(st), st); });
            if (rc) return rc;
        }
        return KV_OK;
    }

    kvt::MigArgs mig_args(int32_t sid, const kvt::Session &s) const {
        kvt::MigArgs m;
        m.table = d_tables + static_cast<int64_t>(sid) * table_stride;
        m.hot = static_cast<uint8_t *>(cfg.hot_base);
        m.img = static_cast<uint8_t *>(cfg.cold_base) + s.img_off;
        m.T_cap = s.cap;
        m.t_begin = 0;
        m.t_end = 0;
        m.once = 0;
        m.int8 = int8;
        m.err = d_err;
        m.s = shape;
        return m;
    }
};

// Shared by the files of the C ABI (pool.cpp).
namespace kvt {
int create_session(kv_pool *p, int64_t max_tokens, int64_t tokens, int32_t state, int32_t *sid_out);
int ensure_event(kv_pool *p, cudaEvent_t *ev);
int wait_event(kv_pool *p, cudaStream_t st, cudaEvent_t ev);
// Residency mode: every evicted block of the sessions `uniq` comes back.
int lru_fetch(kv_pool *p, const std::vector<int32_t> &uniq, const std::vector<int32_t> &protect,
              bool record_ready, cudaStream_t st, int64_t *blocks);
}  // namespace kvt
