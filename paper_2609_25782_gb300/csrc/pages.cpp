// Forks, truncation and compaction of sessions (include/kvtier.h), over the state in pool_state.h. Device
// work goes to page_kernels.cu, and to copy_kernels.cu where a fork reads its parent's image.
#include "cache_ops.h"
#include "pool_state.h"

static_assert(KV_DEVICE_BAD_INDEX == kvt::kErrBadIndex, "public device flag bits must match the kernels'");

using kvt::DeviceGuard;
using kvt::ensure_event;
using kvt::fail;
using kvt::Session;
using kvt::Victim;
using kvt::wait_event;

namespace {

int64_t blocks_of(int64_t tokens, int bt) { return (tokens + bt - 1) / bt; }

// Before work that reads or moves a session's rows.
int wait_written(kv_pool *p, const Session &s, cudaStream_t st) {
    int rc = KV_OK;
    if (s.appended_recorded) rc = wait_event(p, st, s.appended);
    if (!rc && s.ready_recorded) rc = wait_event(p, st, s.ready);
    return rc;
}

// Behind work that reads or moves a session's rows: whatever the pool does with the session next, on any
// stream, waits for it. The stream has waited for what the event marked before (wait_written); the event is made
// before the work is launched, so that a call which cannot have one moves nothing.
int mark_moved(kv_pool *p, Session &s, cudaStream_t st) {
    return p->cuda("cudaEventRecord", [&] { return cudaEventRecord(s.ready, st); });
}

// Copies of blocks and the children's first table entries, as many launches as their parameters take.
template <int kMost>
int run_copies_by(kv_pool *p, const std::vector<kvt::CopyJob> &jobs, int32_t parent, int32_t shared,
                  const std::vector<int32_t> &children, cudaStream_t st) {
    size_t j = 0, c = 0;
    const size_t nc = shared > 0 ? children.size() : 0;
    while (j < jobs.size() || c < nc) {
        kvt::CopyJobs<kMost> a;
        a.hot = static_cast<uint8_t *>(p->cfg.hot_base);
        a.err = p->d_err;
        a.tables = p->d_tables;
        a.table_stride = p->table_stride;
        a.s = p->shape;
        a.parent = parent;
        a.shared = shared;
        a.n = static_cast<int32_t>(std::min<size_t>(kMost, jobs.size() - j));
        a.children = static_cast<int32_t>(std::min<size_t>(kMost, nc - c));
        std::copy(jobs.begin() + j, jobs.begin() + j + a.n, a.job);
        std::copy(children.begin() + c, children.begin() + c + a.children, a.child);
        int rc = p->cuda("block copy launch", [&] { return kvt::launch_copy_jobs(a, p->move_ctas(st), st); });
        if (rc) return rc;
        j += a.n;
        c += a.children;
    }
    return KV_OK;
}
int run_copies(kv_pool *p, const std::vector<kvt::CopyJob> &jobs, int32_t parent, int32_t shared,
               const std::vector<int32_t> &children, cudaStream_t st) {
    return std::max(jobs.size(), children.size()) <= kvt::kCopyJobsFew
               ? run_copies_by<kvt::kCopyJobsFew>(p, jobs, parent, shared, children, st)
               : run_copies_by<kvt::kCopyJobsMax>(p, jobs, parent, shared, children, st);
}

// `need` blocks that a simple pool's free list gives, in the order of their pops.
std::vector<int32_t> next_free(const kv_pool *p, int64_t need) {
    std::vector<int32_t> v(need);
    for (int64_t i = 0; i < need; ++i) v[i] = p->free_list[p->free_list.size() - 1 - i];
    return v;
}

void take(kv_pool *p, const std::vector<int32_t> &v) {
    p->free_list.resize(p->free_list.size() - v.size());
    p->clear_fences(v.data(), v.size());
    p->stats.free_blocks -= static_cast<int64_t>(v.size());
    p->stats.used_blocks += static_cast<int64_t>(v.size());
}

// A session's blocks from logical block `from` on leave it, the last one first, behind the fence; those that are
// free then keep its mark.
void drop_tail(kv_pool *p, Session &s, int64_t from, int slot, uint64_t gen) {
    if (s.home == 0) s.home = ++p->homes;
    for (int64_t j = static_cast<int64_t>(s.blocks.size()); j-- > from;)
        if (s.blocks[j] >= 0) {
            if (p->give_back(s.blocks[j], slot, gen)) p->block_home[s.blocks[j]] = s.home;
            if (p->lru) s.hot_count -= 1;
        }
    s.blocks.resize(from);
    if (p->lru) s.img_tok.resize(from);
}

// What the image still holds once tokens from `valid` on have changed or gone.
void forget_image(kv_pool *p, Session &s, int64_t valid) {
    s.cold_valid = std::min(s.cold_valid, valid);
    const int64_t bt = p->cfg.block_tokens;
    for (size_t j = 0; j < s.img_tok.size(); ++j) {
        const int64_t most = std::max<int64_t>(0, valid - static_cast<int64_t>(j) * bt);
        if (s.img_tok[j] > most) s.img_tok[j] = static_cast<int16_t>(most);
    }
}

// A session that a failed fork had made.
void unmake(kv_pool *p, int32_t sid) {
    Session &s = p->sessions[sid];
    p->cold_release(s.img_off, s.img_bytes);
    p->stats.cold_bytes_used = p->cold_used;
    s.reset();
}

}  // namespace

extern "C" {

int session_fork(kv_pool *p, int32_t sid, int64_t tokens, int64_t max_tokens, int32_t n,
                 int32_t *sids_out, kv_stream_t stream_) {
    if (!p || !sids_out) return fail(KV_ERR_INVALID_ARG, "null argument");
    Session *parent = p->session(sid);
    if (!parent) return fail(KV_ERR_INVALID_ARG, "no such session");
    if (parent->state != KV_SESSION_ACTIVE) return fail(KV_ERR_BAD_STATE, "fork of a paused session");
    if (n < 1) return fail(KV_ERR_INVALID_ARG, "n must be >= 1");
    if (tokens < 0 || tokens > parent->T) return fail(KV_ERR_INVALID_ARG, "tokens past the session's end");
    if (max_tokens < tokens) return fail(KV_ERR_INVALID_ARG, "max_tokens below tokens");
    const int bt = p->cfg.block_tokens;
    const int64_t nb = blocks_of(tokens, bt);
    const int64_t shared = p->lru ? 0 : tokens / bt;
    const int64_t each = nb - shared;             // blocks of a new session's own
    const int64_t need = each * n;
    std::vector<Victim> vic;
    if (p->lru ? !p->plan_evict(need, {sid}, vic) : need > static_cast<int64_t>(p->free_list.size()))
        return fail(KV_ERR_NO_HOT_BLOCKS, "hot pool has too few blocks for the fork");
    std::vector<int32_t> kids;
    int64_t fetched = 0;                          // tokens out of the parent's image
    int rc = KV_OK;
    while (!rc && static_cast<int32_t>(kids.size()) < n) {
        int32_t id = -1;
        rc = kvt::create_session(p, max_tokens, 0, KV_SESSION_ACTIVE, &id);
        if (!rc) kids.push_back(id);
    }
    const std::vector<int32_t> got = rc ? std::vector<int32_t>{} : p->peek_alloc(need, vic);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream_);
    DeviceGuard dg(p->cfg.device, !p->host_only);
    if (!rc) {
        std::vector<kvt::CopyJob> copies;
        std::vector<kvt::BlockJob> fetches;
        // A block's copies one after the other: they read it from the L2.
        for (int64_t j = shared; j < nb; ++j)
            for (int32_t c = 0; c < n; ++c) {
                const int32_t to = got[c * each + j - shared], from = parent->blocks[j];
                const int32_t rows = static_cast<int32_t>(std::min<int64_t>(bt, tokens - j * bt));
                const int32_t jj = static_cast<int32_t>(j);
                if (from >= 0) {
                    copies.push_back({from, to, kids[c], jj, rows});
                } else {
                    kvt::BlockJob b = p->job_for(sid, jj, to, 0, rows);   // out of the parent's image
                    b.sid = kids[c];
                    fetches.push_back(b);
                    fetched += rows;
                }
            }
        for (size_t c = 0; !rc && c < kids.size(); ++c) rc = ensure_event(p, &p->sessions[kids[c]].ready);
        if (!rc) rc = ensure_event(p, &parent->ready);
        if (!rc) rc = wait_written(p, *parent, st);
        if (!rc) rc = p->wait_fences(got.data(), got.size(), st);
        if (!rc) rc = p->evict_device(vic, st);
        if (!rc && !fetches.empty()) rc = p->wait_packed(sid, st);
        if (!rc) rc = run_copies(p, copies, sid, static_cast<int32_t>(shared), kids, st);
        if (!rc) rc = p->run_jobs(fetches, false, st);
        if (!rc) rc = mark_moved(p, *parent, st);   // the parent's blocks stay until they have been read
        for (size_t c = 0; !rc && c < kids.size(); ++c) {
            const cudaEvent_t ev = p->sessions[kids[c]].ready;
            rc = p->cuda("cudaEventRecord", [&] { return cudaEventRecord(ev, st); });
        }
    }
    if (rc) {
        for (int32_t id : kids) unmake(p, id);
        return rc;
    }

    p->evict_commit(vic);
    take(p, got);
    p->stats.bytes_unpacked += fetched * p->image_token_bytes;
    parent->ready_recorded = !p->host_only;
    for (int64_t j = 0; j < shared; ++j) p->block_extra[parent->blocks[j]] += n;
    p->forked = p->forked || shared > 0;
    const uint64_t stamp = p->lru ? ++p->clock : 0;
    for (int32_t c = 0; c < n; ++c) {
        Session &s = p->sessions[kids[c]];
        s.T = tokens;
        s.blocks.assign(parent->blocks.begin(), parent->blocks.begin() + shared);
        s.blocks.insert(s.blocks.end(), got.begin() + c * each, got.begin() + (c + 1) * each);
        s.ready_recorded = !p->host_only;
        if (p->lru) {
            s.img_tok.assign(nb, 0);
            s.hot_count = nb;
            s.last_use = stamp;
            p->lru_in(kids[c]);
        }
        sids_out[c] = kids[c];
    }
    return KV_OK;
}

int session_truncate(kv_pool *p, int32_t sid, int64_t tokens, kv_stream_t stream_) {
    if (!p) return fail(KV_ERR_INVALID_ARG, "null pool");
    Session *s = p->session(sid);
    if (!s) return fail(KV_ERR_INVALID_ARG, "no such session");
    if (tokens < 0 || tokens > s->T) return fail(KV_ERR_INVALID_ARG, "tokens past the session's end");
    if (tokens == s->T) return KV_OK;
    const int bt = p->cfg.block_tokens;
    const int64_t nb = std::min<int64_t>(blocks_of(tokens, bt), static_cast<int64_t>(s->blocks.size()));
    // A shared block that will be written again becomes the session's own. (A paused session's blocks are
    // its image's: none.)
    const bool own = !p->lru && nb > 0 && tokens % bt != 0 && p->block_extra[s->blocks[nb - 1]] > 0;
    if (own && p->free_list.empty()) return fail(KV_ERR_NO_HOT_BLOCKS, "no free block for a shared block's part");
    const std::vector<int32_t> got = own ? next_free(p, 1) : std::vector<int32_t>{};
    // One that was shared, and whose other holder may still be reading behind the cut: what comes there next waits.
    const bool left = !p->lru && nb > 0 && tokens % bt != 0 && !own && p->live_fence(s->blocks[nb - 1]);
    std::vector<int32_t> gone(s->blocks.begin() + nb - (own ? 1 : 0), s->blocks.end());
    gone.erase(std::remove(gone.begin(), gone.end(), -1), gone.end());
    if (left || !gone.empty()) {
        cudaStream_t st = reinterpret_cast<cudaStream_t>(stream_);
        DeviceGuard dg(p->cfg.device, !p->host_only);
        const bool fence = !gone.empty();
        int f = 0;
        int rc = own || left ? ensure_event(p, &s->ready) : KV_OK;
        if (!rc && fence) rc = p->open_fence(gone.data(), gone.size(), st, &f);
        if (!rc) rc = wait_written(p, *s, st);
        if (!rc && own) {
            rc = p->wait_fences(got.data(), got.size(), st);
            if (!rc)
                rc = run_copies(p, {{s->blocks[nb - 1], got[0], sid, static_cast<int32_t>(nb - 1),
                                     static_cast<int32_t>(tokens % bt)}}, sid, 0, {}, st);
        }
        if (!rc && left) rc = p->wait_fences(&s->blocks[nb - 1], 1, st);
        if (!rc && (own || left)) rc = mark_moved(p, *s, st);
        if (!rc && fence) rc = p->record_fence(f, st);
        if (rc) return rc;

        const uint64_t gen = fence ? p->commit_fence(f) : 0;
        if (p->lru) p->lru_out(sid);
        take(p, got);
        drop_tail(p, *s, nb, f, gen);
        if (own) {
            p->give_back(s->blocks[nb - 1], f, gen);
            s->blocks[nb - 1] = got[0];
        }
        if (own || left) s->ready_recorded = !p->host_only;
        if (p->lru) p->lru_in(sid);
    } else {
        s->blocks.resize(nb);                     // evicted ones, if any
        if (p->lru) s->img_tok.resize(blocks_of(tokens, bt));
    }
    s->T = tokens;
    forget_image(p, *s, tokens);
    return KV_OK;
}

int session_compact(kv_pool *p, int32_t sid, const int32_t *keep, int64_t layer_stride,
                    int64_t head_stride, int32_t n, int64_t prefix, kv_stream_t stream_) {
    if (!p) return fail(KV_ERR_INVALID_ARG, "null pool");
    Session *s = p->session(sid);
    if (!s) return fail(KV_ERR_INVALID_ARG, "no such session");
    if (s->state != KV_SESSION_ACTIVE) return fail(KV_ERR_BAD_STATE, "compaction of a paused session");
    if (n < 0 || prefix < 0 || prefix > s->T || n > s->T - prefix)
        return fail(KV_ERR_INVALID_ARG, "prefix and kept tokens exceed the session's");
    if (layer_stride < 0 || head_stride < 0 || layer_stride > (int64_t(1) << 40) || head_stride > (int64_t(1) << 40))
        return fail(KV_ERR_INVALID_ARG, "strides of the lists out of range");
    if (n > 0 && !p->host_only && !keep) return fail(KV_ERR_INVALID_ARG, "null lists");
    if (reinterpret_cast<uintptr_t>(keep) & 3) return fail(KV_ERR_INVALID_ARG, "lists must be 4-byte aligned");
    if (n == 0) return session_truncate(p, sid, prefix, stream_);
    if (prefix + n == s->T) return KV_OK;
    const int bt = p->cfg.block_tokens;
    const int64_t end = prefix + n;
    const int64_t j0 = prefix / bt, j1 = blocks_of(end, bt);
    std::vector<int32_t> slot(j1 - j0, -1);       // new places of shared blocks
    int64_t need = 0;
    for (int64_t j = j0; !p->lru && j < j1; ++j)
        if (p->block_extra[s->blocks[j]] > 0) ++need;
    if (need > static_cast<int64_t>(p->free_list.size()))
        return fail(KV_ERR_NO_HOT_BLOCKS, "hot pool has too few free blocks for the compaction of shared ones");

    DeviceGuard dg(p->cfg.device, !p->host_only);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream_);
    if (p->lru) {
        int64_t fetched = 0;
        int rc = kvt::lru_fetch(p, {sid}, {sid}, true, st, &fetched);
        if (rc) return rc;
        s = p->session(sid);
    }
    const std::vector<int32_t> got = next_free(p, need);
    for (int64_t j = j0, k = 0; need > 0 && j < j1; ++j)
        if (p->block_extra[s->blocks[j]] > 0) slot[j - j0] = got[k++];
    std::vector<int32_t> gone(s->blocks.begin() + j1, s->blocks.end()), kept;
    for (int64_t j = j0; j < j1; ++j) (slot[j - j0] >= 0 ? gone : kept).push_back(s->blocks[j]);

    int f = 0;
    int rc = ensure_event(p, &s->ready);
    if (!rc) rc = p->open_fence(gone.data(), gone.size(), st, &f);
    if (!rc) rc = wait_written(p, *s, st);
    if (!rc) rc = p->wait_fences(got.data(), got.size(), st);
    if (!rc && p->forked) rc = p->wait_fences(kept.data(), kept.size(), st);   // written in place
    const int64_t step = need > 0 ? kvt::kCompactFresh : j1 - j0;
    for (int64_t j = j0; !rc && j < j1; j += step) {
        kvt::CompactArgs a;
        a.hot = static_cast<uint8_t *>(p->cfg.hot_base);
        a.err = p->d_err;
        a.table = p->d_tables + static_cast<int64_t>(sid) * p->table_stride;
        a.keep = keep;
        a.layer_stride = layer_stride;
        a.head_stride = head_stride;
        const int64_t to = std::min(j1, j + step);
        // In a block that is new the tokens before `prefix` move as well.
        a.t_begin = static_cast<int32_t>(std::max(j * bt, j == j0 && slot[0] < 0 ? prefix : 0));
        a.t_end = static_cast<int32_t>(std::min(end, to * bt));
        a.prefix = static_cast<int32_t>(prefix);
        a.T = static_cast<int32_t>(s->T);
        a.fresh = need > 0;
        a.fresh_at = static_cast<int32_t>(j);
        if (need > 0) std::copy(slot.begin() + (j - j0), slot.begin() + (to - j0), a.slot);
        a.s = p->shape;
        rc = p->cuda("compaction launch", [&] { return kvt::launch_compact(a, p->num_sms, st); });
    }
    std::vector<int32_t> row(s->blocks.begin() + j0, s->blocks.begin() + j1);
    for (int64_t j = 0; j < j1 - j0; ++j)
        if (slot[j] >= 0) row[j] = slot[j];
    if (!rc && need > 0) rc = p->write_table(sid, row.data(), j0, j1 - j0, st);
    if (!rc) rc = mark_moved(p, *s, st);
    if (!rc) rc = p->record_fence(f, st);
    if (rc) return rc;

    const uint64_t gen = p->commit_fence(f);
    if (p->lru) p->lru_out(sid);
    take(p, got);
    drop_tail(p, *s, j1, f, gen);
    for (int64_t j = j1; j-- > j0;)
        if (slot[j - j0] >= 0) {
            p->give_back(s->blocks[j], f, gen);
            s->blocks[j] = slot[j - j0];
        }
    if (p->lru) p->lru_in(sid);
    s->T = end;
    s->ready_recorded = !p->host_only;
    forget_image(p, *s, prefix);
    return KV_OK;
}

}  // extern "C"
