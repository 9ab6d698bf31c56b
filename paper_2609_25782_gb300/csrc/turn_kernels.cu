// Attention of several new tokens per session over the paged cache, for sm_103a:
// a turn's context or a whole prompt (causal, its K and V written into the hot
// pool), and drafted tokens (a bit mask per draft, nothing written).
//
// One persistent CTA per SM works through its piece of the line of items that
// turn_plan.h lays out. The query heads that share a kv-head are packed into the
// 128 rows of a row tile, so K and V are read once for all of them. A CTA has two
// streams, each with a row tile's scores and output in tensor memory: two row
// tiles of a pair against the same key tile, or (narrow items) every other key
// tile against one row tile. Roles, by warp:
//   0-3, 4-7  softmax of stream 0 and 1, a thread per row: scores from tensor
//             memory, running maximum and sum in 32 bits, weights back to tensor
//             memory in bf16; at the end the output
//   8         copies: q tiles and key tiles (TMA, 128-byte swizzle)
//   9         matrix products (tcgen05): S = Q K^T from shared memory, O += P V
//             with P from tensor memory
// The tensor cores work on one stream while the other's softmax runs.
#include <cuda_bf16.h>

#include "kvt_internal.h"
#include "turn_plan.h"

namespace kvt {
namespace {

constexpr int kTileBytes = kTurnKeys * kRowBytes;   // a key or row tile, 32 KB
constexpr int kHalfBytes = kTileBytes / 2;          // its columns 0-63, then 64-127: 128 rows of 128 B
constexpr int kBoxRows = 16;                        // rows of one copy
constexpr int kStages = 5;                          // K or V tiles in flight
constexpr int kThreads = 384;
constexpr int kCopyWarp = 8, kMmaWarp = 9;          // 10 and 11 only make up a warpgroup
// Registers per thread: at launch, then of the softmax warps and of the others. A softmax thread
// keeps its row's 128 scores; the shares add up to what the CTA was launched with.
constexpr int kRegsLaunch = 168, kRegsSoftmax = 200, kRegsOther = 104;
static_assert(256 * kRegsSoftmax + 128 * kRegsOther <= kThreads * kRegsLaunch, "a larger share would wait forever");
constexpr unsigned long long kWaitLimitNs = 2000000000ull;   // 2 s

// Tensor memory: 128 columns of 32 bits each for S (and P in its lower half) and O of both streams.
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256, kColStream = 128;

struct Plan {
    int64_t W;
    int64_t begin_at, end_at;   // cost at which the first and the last item begin
    TurnPos begin, end;
    int32_t pieces;
};

struct alignas(1024) Smem {
    uint8_t q[2][kTileBytes];
    uint8_t kv[kStages][kTileBytes];
    uint64_t kv_full[kStages], kv_empty[kStages];
    uint64_t q_full[2], q_empty, s_full[2], p_full[2], o_full[2], drained;
    Plan plan;
    float other_m[kTurnRows], other_l[kTurnRows];   // narrow items: stream 1's statistics
    uint32_t tmem;
    int32_t abort;
    int32_t last[2];
};
constexpr int kSmemBytes = sizeof(Smem) + 1024;     // and the way to a 1 024-byte boundary
static_assert(kSmemBytes <= 227 * 1024, "shared memory of a CTA");

struct Maps {
    CUtensorMap q, k, v, hot;
};

// ---- instructions ------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void *p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ unsigned long long global_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void mbar_init(uint64_t *bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t *bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint64_t *bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes)
                 : "memory");
}
__device__ __forceinline__ bool mbar_try(uint64_t *bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// A wait with a limit. false: it ran out here or in another role, and the caller stops.
__device__ __forceinline__ bool mbar_wait(Smem &sm, uint64_t *bar, uint32_t parity) {
    if (mbar_try(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    while (!mbar_try(bar, parity)) {
        if (*reinterpret_cast<volatile int32_t *>(&sm.abort)) return false;
        if (global_ns() - t0 > kWaitLimitNs) {
            *reinterpret_cast<volatile int32_t *>(&sm.abort) = 1;
            return false;
        }
    }
    return true;
}

__device__ __forceinline__ void copy_box3(void *dst, const CUtensorMap *map, int row, int half, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(half), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void copy_box4(void *dst, const CUtensorMap *map, int head, int token, int half,
                                          uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(head), "r"(token), "r"(half), "r"(smem_u32(bar))
        : "memory");
}

// Shared-memory operand, 128-byte swizzle. Q and K have their inner (summed) dimension contiguous:
// groups of 8 rows are 1 024 bytes apart. V is summed over its rows: 8 keys are 1 024 bytes
// apart, its two column halves kHalfBytes.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t leading) {
    return static_cast<uint64_t>(addr >> 4 & 0x3FFF) | static_cast<uint64_t>(leading >> 4) << 16 |
           static_cast<uint64_t>(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// bf16 x bf16 -> fp32, 128 rows; n columns, the right operand transposed for V, the left negated.
__device__ __forceinline__ uint32_t mma_form(int n, bool v, bool negate) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (negate ? 1u << 13 : 0u) | (v ? 1u << 16 : 0u) |
           static_cast<uint32_t>(n >> 3) << 17 | static_cast<uint32_t>(kTurnRows >> 4) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t form, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(form), "r"(static_cast<uint32_t>(add))
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t form, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(form), "r"(static_cast<uint32_t>(add))
        : "memory");
}
// Arrives at bar once everything this thread has issued to the tensor cores is done.
__device__ __forceinline__ void mma_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

#define KVT_R8(x, o) "=r"(x[o]), "=r"(x[o + 1]), "=r"(x[o + 2]), "=r"(x[o + 3]), "=r"(x[o + 4]), "=r"(x[o + 5]), \
        "=r"(x[o + 6]), "=r"(x[o + 7])
#define KVT_U8(x, o) "r"(x[o]), "r"(x[o + 1]), "r"(x[o + 2]), "r"(x[o + 3]), "r"(x[o + 4]), "r"(x[o + 5]), \
        "r"(x[o + 6]), "r"(x[o + 7])
#define KVT_RW8(x, o) "+r"(x[o]), "+r"(x[o + 1]), "+r"(x[o + 2]), "+r"(x[o + 3]), "+r"(x[o + 4]), "+r"(x[o + 5]), \
        "+r"(x[o + 6]), "+r"(x[o + 7])

// 32 columns of this thread's row. The values are there after tmem_wait on them.
__device__ __forceinline__ void tmem_load(uint32_t (&x)[32], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,"
        "%28,%29,%30,%31}, [%32];"
        : KVT_R8(x, 0), KVT_R8(x, 8), KVT_R8(x, 16), KVT_R8(x, 24)
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&x)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : KVT_RW8(x, 0), KVT_RW8(x, 8), KVT_RW8(x, 16), KVT_RW8(x, 24)::"memory");
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&x)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,"
        "%28,%29,%30,%31};" ::KVT_U8(x, 0),
        KVT_U8(x, 8), KVT_U8(x, 16), KVT_U8(x, 24), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t (&x)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::KVT_U8(x, 0),
        KVT_U8(x, 8), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t y;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
    return y;
}
__device__ __forceinline__ void sync_threads(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ int arrive(int32_t *counter) {
    int prev;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(prev) : "l"(counter) : "memory");
    return prev;
}

// ---- the work ----------------------------------------------------------------------------

__device__ __forceinline__ TurnShape turn_shape(const TurnArgs &a) {
    return {kTurnRows / (a.s.Hq / a.s.Hkv), a.s.Hkv, a.masks == nullptr};
}

// Session b as the call describes it; n = 0 for one whose data is out of range.
__device__ __forceinline__ TurnSession session_of(const TurnArgs &a, int b, bool *bad = nullptr) {
    const int lo = a.cu[b], hi = a.cu[b + 1], T = a.seq_lens[b];
    const bool drafts = a.masks != nullptr;
    const int64_t n = static_cast<int64_t>(hi) - lo;
    const bool ok = lo >= 0 && n >= 0 && hi <= a.total && T >= (drafts ? 0 : n) &&
                    T <= static_cast<int64_t>(a.max_blocks) * a.s.bt && !(drafts && n > kMaxDrafts);
    if (bad) *bad = !ok;
    TurnSession x;
    x.n = ok ? static_cast<int>(n) : 0;
    x.P = ok ? (drafts ? T : T - x.n) : 0;
    x.lo = lo;
    return x;
}

// Sum of x over the lanes before this one, and over all.
__device__ __forceinline__ int64_t scan(int64_t x, int lane, int64_t *all) {
    int64_t y = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t z = __shfl_up_sync(~0u, y, d);
        if (lane >= d) y += z;
    }
    *all = __shfl_sync(~0u, y, 31);
    return y - x;
}

// This CTA's piece, by one warp.
__device__ void make_plan(const TurnArgs &a, Plan &plan, int lane) {
    const TurnShape s = turn_shape(a);
    int64_t W = 0, mine = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int b = b0 + lane;
        int64_t cost = 0, all;
        if (b < a.B) {
            bool bad;
            cost = s.Hkv * turn_head_cost(s, session_of(a, b, &bad));
            if (bad && blockIdx.x == 0) atomicOr(a.err, kErrBadLength);
        }
        mine = cost;   // kept for the second pass where one round has all sessions
        scan(cost, lane, &all);
        W += all;
    }
    const int pieces = W == 0 ? 0 : turn_pieces(W, gridDim.x);
    if (lane == 0) {
        plan.W = W;
        plan.pieces = pieces;
        plan.begin = plan.end = {a.B, 0, 0, 0};
        plan.begin_at = plan.end_at = 0;
    }
    __syncwarp();
    const int c = blockIdx.x;
    if (c >= pieces) return;
    const int64_t u[2] = {turn_cut(W, pieces, c), turn_cut(W, pieces, c + 1)};   // the second is W at the end
    int64_t before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int b = b0 + lane;
        int64_t cost = 0, all;
        TurnSession x = {0, 0, 0};
        if (a.B <= 32) cost = mine;
        if (b < a.B) {
            x = session_of(a, b);
            if (a.B > 32) cost = s.Hkv * turn_head_cost(s, x);
        }
        const int64_t at = before + scan(cost, lane, &all);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (u[e] < at || u[e] >= at + cost) continue;
            int64_t item;
            TurnPos p = turn_locate(s, x, b, u[e] - at, &item);
            if (p.t >= turn_tiles(s, x, p.pair)) {   // the item's end: the next one's start
                p.t = 0;
                if (++p.pair >= turn_pairs(s, x)) {
                    p.pair = 0;
                    if (++p.g >= s.Hkv) {
                        p.g = 0;
                        ++p.b;   // an empty session here is passed over by the walk
                    }
                }
            }
            (e ? plan.end : plan.begin) = p;
            (e ? plan.end_at : plan.begin_at) = at + item;
        }
        before += all;
    }
    __syncwarp();
}

// A run of key tiles t0 .. t1 - 1 of one item.
struct Run {
    TurnSession x;
    int b, g, pair, t0, t1, tiles, cached_tiles, own_keys;
    bool narrow;
};

// The runs of a piece, in order; every role walks them by itself.
struct Walk {
    TurnPos at;
    __device__ explicit Walk(const Plan &plan) : at(plan.begin) {}
    __device__ bool next(const TurnArgs &a, const Plan &plan, Run &r) {
        const TurnShape s = turn_shape(a);
        while (at.b < a.B) {
            const TurnPos &end = plan.end;
            const bool to_end = at.b == end.b && at.g == end.g && at.pair == end.pair;
            if (to_end && at.t >= end.t) return false;
            r.x = session_of(a, at.b);
            if (r.x.n == 0) {   // nothing of this session; the end may be its start
                if (at.b == end.b) return false;
                at = {at.b + 1, 0, 0, 0};
                continue;
            }
            r.b = at.b;
            r.g = at.g;
            r.pair = at.pair;
            r.tiles = turn_tiles(s, r.x, at.pair);
            r.cached_tiles = turn_cached_tiles(r.x);
            r.own_keys = turn_own_keys(s, r.x, at.pair);
            r.narrow = turn_narrow(s, r.x, at.pair);
            r.t0 = at.t;
            r.t1 = to_end ? end.t : r.tiles;
            if (to_end) {
                at.t = end.t;
                return true;
            }
            at.t = 0;
            if (++at.pair >= turn_pairs(s, r.x)) {
                at.pair = 0;
                if (++at.g >= s.Hkv) {
                    at.g = 0;
                    ++at.b;
                }
            }
            return true;
        }
        return false;
    }
};

// Keys of key tile t of an item.
__device__ __forceinline__ int keys_of(const Run &r, int t) {
    const int left = t < r.cached_tiles ? r.x.P - t * kTurnKeys : r.own_keys - (t - r.cached_tiles) * kTurnKeys;
    return min(left, kTurnKeys);
}

// ---- copies ------------------------------------------------------------------------------

// One K (kv = 0) or V tile into a stage, by the copy warp: groups of 16 keys by TMA, two boxes each
// (the column halves, kHalfBytes apart). Keys past the last full group come by plain loads, rows up
// to the group's end are cleared: what they hold in memory may be anything, and a weight of 0 does not
// make a NaN go away in the product with V.
__device__ __forceinline__ void copy_key_tile(const TurnArgs &a, const Maps &maps, const Run &r, int t, int kv,
                                              uint8_t *stage, uint64_t *full, int lane) {
    const Shape &sh = a.s;
    const int keys = keys_of(r, t), groups = keys / kBoxRows, rest = keys % kBoxRows;
    const bool cached = t < r.cached_tiles;
    const int k0 = (cached ? t : t - r.cached_tiles) * kTurnKeys;
    // Lane l has group l / 2, column half l % 2.
    const int group = lane >> 1, half = lane & 1;
    int row = 0;   // of the pool: below 2^31
    if (cached && group * kBoxRows < keys) {
        const int pos = k0 + group * kBoxRows, j = pos / sh.bt;
        int blk = a.tables[static_cast<int64_t>(r.b) * a.max_blocks + j];
        if (blk < 0 || blk >= sh.num_blocks) {
            atomicOr(a.err, kErrBadBlock);
            blk = 0;   // the result is wrong, the access is not
        }
        row = (((blk * sh.L + a.layer) * 2 + kv) * sh.Hkv + r.g) * sh.bt + pos - j * sh.bt;
    }
    if (rest) {
        const int first = __shfl_sync(~0u, row, 2 * groups);
        const uint16_t *src;
        int64_t step;
        if (cached) {
            src = a.hot + static_cast<int64_t>(first) * kHeadDim;
            step = kHeadDim;
        } else {
            src = (kv ? a.v_new : a.k_new) + (r.x.lo + k0 + groups * kBoxRows) * a.kv_stride + r.g * kHeadDim;
            step = a.kv_stride;
        }
#pragma unroll
        for (int i = 0; i < kBoxRows * 16 / 32; ++i) {
            const int rr = i * 2 + (lane >> 4), u = lane & 15;   // row of the group, 16-byte unit of the row
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (rr < rest) x = *reinterpret_cast<const uint4 *>(src + rr * step + u * 8);
            *reinterpret_cast<uint4 *>(stage + (u >> 3) * kHalfBytes + (groups * kBoxRows + rr) * 128 +
                                       (((u & 7) ^ (rr & 7)) << 4)) = x;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
    }
    if (lane == 0) mbar_expect(full, groups * kBoxRows * kRowBytes);
    __syncwarp();
    if (group < groups) {
        uint8_t *dst = stage + half * kHalfBytes + group * kBoxRows * 128;
        if (cached) copy_box3(dst, &maps.hot, row, half, full);
        else copy_box4(dst, kv ? &maps.v : &maps.k, r.g, r.x.lo + k0 + group * kBoxRows, half, full);
    }
    __syncwarp();
}

__device__ void copy_role(const TurnArgs &a, const Maps &maps, Smem &sm, int lane) {
    const TurnShape s = turn_shape(a);
    const int G = a.s.Hq / a.s.Hkv;
    int stage = 0, round = 0, items = 0, pairs = 0;
    uint32_t filled = 0;   // copies issued so far, saturating at kStages
    bool ok = true;   // the same in all lanes until the last copy is out
    Walk walk(sm.plan);
    Run r;
    while (ok && walk.next(a, sm.plan, r)) {
        if (items > 0) ok = __all_sync(~0u, mbar_wait(sm, &sm.q_empty, (items - 1) & 1));
        if (!ok) break;
        ++items;
        const int tiles = r.narrow ? 1 : 2;
        pairs += tiles - 1;
        if (lane < tiles) mbar_expect(&sm.q_full[lane], kTileBytes);
        __syncwarp();
        if (lane < 2 * tiles)
            copy_box4(sm.q[lane >> 1] + (lane & 1) * kHalfBytes, &maps.q, r.g * G,
                      r.x.lo + (2 * r.pair + (lane >> 1)) * s.tokens, lane & 1, &sm.q_full[lane >> 1]);
        __syncwarp();
        for (int t = r.t0; ok && t < r.t1; ++t)
            for (int kv = 0; kv < 2; ++kv) {
                if (round > 0) ok = __all_sync(~0u, mbar_wait(sm, &sm.kv_empty[stage], (round - 1) & 1));
                if (!ok) break;
                copy_key_tile(a, maps, r, t, kv, sm.kv[stage], &sm.kv_full[stage], lane);
                if (filled < kStages) ++filled;
                if (++stage == kStages) {
                    stage = 0;
                    ++round;
                }
            }
    }
    // Every copy lands before the CTA ends, whatever became of the other roles; with all well,
    // every stage has been given back as well.
    for (uint32_t i = 0; i < filled; ++i) {
        const bool now = static_cast<int>(i) < stage;   // filled in this round, or in the one before
        const uint32_t parity = (now ? round : round - 1) & 1;
        if (ok) ok = mbar_wait(sm, &sm.kv_empty[i], parity);
        const unsigned long long t0 = global_ns();
        while (!mbar_try(&sm.kv_full[i], parity) && global_ns() - t0 < kWaitLimitNs) {}
    }
    if (ok && items > 0) ok = mbar_wait(sm, &sm.q_empty, (items - 1) & 1);
    for (int i = 0; !ok && i < 2; ++i) {   // and the last q tiles
        const int loads = i ? pairs : items;
        const unsigned long long t0 = global_ns();
        while (loads > 0 && !mbar_try(&sm.q_full[i], (loads - 1) & 1) && global_ns() - t0 < kWaitLimitNs) {}
    }
}

// ---- matrix products -----------------------------------------------------------------------

// S = Q K^T. The steps' operands lie a constant apart: one addition per step and operand, so that the
// issuing thread keeps up with the tensor cores (64 cycles a step).
__device__ __forceinline__ void product_qk(uint32_t d, uint32_t q, uint32_t k, uint32_t form) {
    const uint64_t a = operand(q, 16), b = operand(k, 16);
#pragma unroll
    for (int i = 0; i < kHeadDim / 16; ++i) {
        const int off = ((i >> 2) * kHalfBytes + (i & 3) * 32) >> 4;
        mma_ss(d, a + off, b + off, form, i > 0);
    }
}
// O += P V over 16 * steps keys, or O = P V.
__device__ __forceinline__ void product_pv(uint32_t d, uint32_t p, uint32_t v, int steps, bool add) {
    const uint64_t b = operand(v, kHalfBytes);
    const uint32_t form = mma_form(kHeadDim, true, false);
    if (steps == kTurnKeys / 16) {
#pragma unroll
        for (int i = 0; i < kTurnKeys / 16; ++i) mma_ts(d, p + i * 8, b + i * (16 * 128 >> 4), form, i > 0 || add);
    } else {
        for (int i = 0; i < steps; ++i) mma_ts(d, p + i * 8, b + i * (16 * 128 >> 4), form, i > 0 || add);
    }
}

// A stage of the ring and the parity of its present round, two stages further at each step: K tiles
// have the even places, V tiles the odd ones.
struct Cursor {
    int stage;
    uint32_t parity;
    __device__ __forceinline__ void next() {
        stage += 2;
        if (stage >= kStages) {
            stage -= kStages;
            parity ^= 1;
        }
    }
};

// One lane of the warp.
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(~0u, x, 0); }

// The whole warp walks and waits, one lane issues: control flow and operands are the same in all lanes,
// which the compiler has to see (votes, shuffles) to keep them in uniform registers. With one lane
// doing everything each step moved its operands there first: 90 cycles a step, 64 of the tensor cores'.
__device__ void mma_role(const TurnArgs &a, Smem &sm) {
    const uint32_t tmem = uniform(sm.tmem);
    const bool negate = a.negate != 0;
    uint32_t q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
    Cursor at_k = {0, 0}, at_v = {1, 0};
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t parity) { ok = __all_sync(~0u, mbar_wait(sm, bar, parity)); };
    Walk walk(sm.plan);
    Run r;
    while (ok && __all_sync(~0u, walk.next(a, sm.plan, r))) {
        const int tiles = uniform(r.t1 - r.t0), t0 = uniform(r.t0), cached_tiles = uniform(r.cached_tiles);
        const int cached_keys = uniform(r.x.P), own_keys = uniform(r.own_keys);
        const bool narrow = uniform(r.narrow);
        const int jobs = narrow ? tiles : 2 * tiles;
        auto steps_of = [&](int i) {   // of 16 keys, of the run's tile i
            const int t = t0 + i;
            const int left = t < cached_tiles ? cached_keys - t * kTurnKeys : own_keys - (t - cached_tiles) * kTurnKeys;
            return left >= kTurnKeys ? kTurnKeys / 16 : (left + 15) / 16;
        };
        for (int s = 0; ok && s < (narrow ? 1 : 2); ++s) {
            wait(&sm.q_full[s], q_phase[s]);
            q_phase[s] ^= 1;
        }
        // O_s += P_s V of job j
        auto pv = [&](int j) {
            const int s = j & 1;
            if (narrow || s == 0) wait(&sm.kv_full[at_v.stage], at_v.parity);
            if (ok) wait(&sm.p_full[s], p_phase[s]);
            if (!ok) return;
            p_phase[s] ^= 1;
            fence_after();
            const int steps = steps_of(narrow ? j : j >> 1);
            if (elected()) {
                product_pv(tmem + kColO + s * kColStream, tmem + kColS + s * kColStream,
                           smem_u32(sm.kv[at_v.stage]), steps, j >= 2);
                if (narrow || s == 1) mma_commit(&sm.kv_empty[at_v.stage]);
                if (j + 2 >= jobs) mma_commit(&sm.o_full[s]);
            }
            __syncwarp();
            if (narrow || s == 1) at_v.next();
        };
        for (int j = 0; ok && j < jobs; ++j) {
            const int s = j & 1;
            if (j >= 2) pv(j - 2);
            if (ok && (narrow || s == 0)) wait(&sm.kv_full[at_k.stage], at_k.parity);
            if (!ok) break;
            fence_after();
            const int steps = steps_of(narrow ? j : j >> 1);
            if (elected()) {
                product_qk(tmem + kColS + s * kColStream, smem_u32(sm.q[narrow ? 0 : s]),
                           smem_u32(sm.kv[at_k.stage]), mma_form(16 * steps, false, negate));
                mma_commit(&sm.s_full[s]);
                if (narrow || s == 1) mma_commit(&sm.kv_empty[at_k.stage]);
                if (j == jobs - 1) mma_commit(&sm.q_empty);
            }
            __syncwarp();
            if (narrow || s == 1) at_k.next();
        }
        for (int j = jobs < 2 ? 0 : jobs - 2; ok && j < jobs; ++j) pv(j);
    }
    // Nothing of the tensor cores' is left behind.
    if (elected()) mma_commit(&sm.drained);
    __syncwarp();
    const unsigned long long t0 = global_ns();
    while (!mbar_try(&sm.drained, 0) && global_ns() - t0 < kWaitLimitNs) {}
}

// ---- softmax -------------------------------------------------------------------------------

// The running maximum moves only when a score exceeds it by more than this many powers of two, so that
// O is rescaled rarely; weights then stay below 2^8, which their sums in 32 bits and bf16 hold as well.
constexpr float kLazyLog2 = 8.f;

struct Stats {
    float m, l;   // running maximum of the scaled scores (base 2), sum of the weights
};

// Two values at a time.
__device__ __forceinline__ uint64_t pair_of(uint32_t lo, uint32_t hi) {
    uint64_t y;
    asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "r"(lo), "r"(hi));
    return y;
}
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) {
    uint64_t w;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(w) : "l"(x), "l"(y), "l"(z));
    return w;
}
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) {
    uint64_t w;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(w) : "l"(x), "l"(y));
    return w;
}
__device__ __forceinline__ float2 halves(uint64_t x) {
    float2 y;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(y.x), "=f"(y.y) : "l"(x));
    return y;
}

// Four running maxima, so that no instruction waits for the one before it.
struct Tops {
    float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    __device__ __forceinline__ void add(const uint32_t (&x)[32]) {
#pragma unroll
        for (int i = 0; i < 32; i += 2)
            t[i / 2 % 4] = fmaxf(t[i / 2 % 4], fmaxf(__uint_as_float(x[i]), __uint_as_float(x[i + 1])));
    }
    __device__ __forceinline__ float all() const { return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])); }
};

// The running maximum after a tile whose largest scaled score is `top`; O follows where it moves.
// A row that sees nothing yet keeps m = -infinity.
__device__ __forceinline__ void move_top(float top, uint32_t o_addr, bool first, Stats &st) {
    if (!__any_sync(~0u, top > st.m + kLazyLog2)) return;
    const float m = fmaxf(st.m, top);
    const float c = m == -INFINITY ? 1.f : ex2(st.m - m);
    st.m = m;
    st.l *= c;
    if (first) return;
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
        uint32_t o[32];
        tmem_load(o, o_addr + i * 32);
        tmem_wait(o);
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * c);
        tmem_store(o_addr + i * 32, o);
    }
}

// Weights ex2(x * scale - ref) of 32 scores, in bf16 to tensor memory; their sum (of the unrounded
// ones) is added to `sum`.
__device__ __forceinline__ void put_weights(const uint32_t (&x)[32], uint64_t scale, uint64_t ref, uint32_t p_addr,
                                            uint64_t (&sum)[4]) {
    uint32_t p[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float2 e = halves(fma2(pair_of(x[2 * i], x[2 * i + 1]), scale, ref));
        const float y0 = ex2(e.x), y1 = ex2(e.y);
        sum[i % 4] = add2(sum[i % 4], pair_of(__float_as_uint(y0), __float_as_uint(y1)));
        p[i] = pack_bf16(y0, y1);
    }
    tmem_store16(p_addr, p);
}

// Scores of which the row sees those in `sees`; the others become -infinity, weight 0.
__device__ __forceinline__ void hide(uint32_t (&x)[32], uint32_t sees) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (!(sees >> i & 1)) x[i] = 0xFF800000u;
}

// A key tile's weights of this thread's row: S from tensor memory, P back over it (16 columns
// of P for 32 of S, so a chunk's weights never reach scores that are still to be read).
__device__ __forceinline__ void softmax_tile(const TurnArgs &a, const Run &r, int t, int token, uint64_t mask,
                                             uint32_t s_addr, uint32_t o_addr, bool first, Stats &st) {
    const int keys = keys_of(r, t);
    const bool own = t >= r.cached_tiles;
    // Keys of the tile that the row sees: the first `seen` of them, of drafts those in its mask.
    int seen = keys;
    if (own && !a.masks) seen = min(keys, token + 1 - (t - r.cached_tiles) * kTurnKeys);
    const uint64_t scale = pair_of(__float_as_uint(a.scale_log2), __float_as_uint(a.scale_log2));
    uint64_t sum[4] = {0, 0, 0, 0};
    Tops top;
    if (__all_sync(~0u, seen == kTurnKeys) && !(own && a.masks)) {
        uint32_t x[4][32];
        tmem_load(x[0], s_addr);
        tmem_load(x[1], s_addr + 32);
        tmem_wait(x[0]);
        tmem_wait(x[1]);
        tmem_load(x[2], s_addr + 64);
        tmem_load(x[3], s_addr + 96);
        top.add(x[0]);
        top.add(x[1]);
        tmem_wait(x[2]);
        tmem_wait(x[3]);
        top.add(x[2]);
        top.add(x[3]);
        move_top(top.all() * a.scale_log2, o_addr, first, st);
        const uint32_t minus = __float_as_uint(st.m == -INFINITY ? 0.f : -st.m);
        const uint64_t ref = pair_of(minus, minus);
#pragma unroll
        for (int c = 0; c < 4; ++c) put_weights(x[c], scale, ref, s_addr + c * 16, sum);
    } else {
        const uint64_t bits = own && a.masks ? mask : ~0ull;   // drafts are at most 64 keys
        const int chunks = (keys + 31) / 32;
        auto sees = [&](int c) {
            const int n = seen - c * 32;
            return (n >= 32 ? ~0u : n > 0 ? (1u << n) - 1 : 0u) & (c < 2 ? static_cast<uint32_t>(bits >> (c * 32)) : ~0u);
        };
#pragma unroll 1
        for (int c = 0; c < chunks; ++c) {
            uint32_t x[32];
            tmem_load(x, s_addr + c * 32);
            tmem_wait(x);
            hide(x, sees(c));
            top.add(x);
        }
        move_top(top.all() * a.scale_log2, o_addr, first, st);
        const uint32_t minus = __float_as_uint(st.m == -INFINITY ? 0.f : -st.m);
        const uint64_t ref = pair_of(minus, minus);
#pragma unroll 1
        for (int c = 0; c < chunks; ++c) {
            uint32_t x[32];
            tmem_load(x, s_addr + c * 32);
            tmem_wait(x);
            hide(x, sees(c));
            put_weights(x, scale, ref, s_addr + c * 16, sum);
        }
    }
    const float2 y = halves(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
    st.l += y.x + y.y;
    tmem_stored();
}

// 32 values of an output row from column d0.
__device__ __forceinline__ void store_out(const TurnArgs &a, int64_t row, int d0, const float (&y)[32]) {
    if (a.out_bf16) {
        uint4 *to = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.out) + row * kHeadDim + d0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            to[i] = make_uint4(pack_bf16(y[8 * i], y[8 * i + 1]), pack_bf16(y[8 * i + 2], y[8 * i + 3]),
                               pack_bf16(y[8 * i + 4], y[8 * i + 5]), pack_bf16(y[8 * i + 6], y[8 * i + 7]));
    } else {
        float4 *to = reinterpret_cast<float4 *>(static_cast<float *>(a.out) + row * kHeadDim + d0);
#pragma unroll
        for (int i = 0; i < 8; ++i) to[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
    }
}

// A slot of partial results: 256 rows of 128 values, four values of all rows together (so that a warp's
// rows are next to each other), then (m, l) of the rows.
__device__ __forceinline__ float4 *part_o(const TurnArgs &a, int slot, int stream) {
    return reinterpret_cast<float4 *>(a.part) + (static_cast<int64_t>(slot) * 2 + stream) * kTurnRows * (kHeadDim / 4);
}
__device__ __forceinline__ float2 *part_ml(const TurnArgs &a, int slot, int stream) {
    return reinterpret_cast<float2 *>(a.part + static_cast<int64_t>(a.part_slots) * 2 * kTurnRows * kHeadDim) +
           (static_cast<int64_t>(slot) * 2 + stream) * kTurnRows;
}

// The item's output row of this thread, from tensor memory, 32 columns at a time: O times `w`, and
// (kTwo) the other stream's, at `other`, times `w_other`.
template <bool kTwo, typename Put>
__device__ __forceinline__ void read_o(uint32_t o_addr, float w, uint32_t other, float w_other, Put put) {
#pragma unroll 1
    for (int d = 0; d < kHeadDim; d += 32) {
        uint32_t o[32];
        float y[32];
        tmem_load(o, o_addr + d);
        tmem_wait(o);
#pragma unroll
        for (int i = 0; i < 32; ++i) y[i] = __uint_as_float(o[i]) * w;
        if constexpr (kTwo) {
            tmem_load(o, other + d);
            tmem_wait(o);
#pragma unroll
            for (int i = 0; i < 32; ++i) y[i] = __fmaf_rn(__uint_as_float(o[i]), w_other, y[i]);
        }
        put(d, y);
    }
}

// The item's new tokens' K and V of its kv-head into their slots of the pool; thread `tid` of `threads`.
__device__ __forceinline__ void store_new_kv(const TurnArgs &a, const TurnShape &s, const Run &r, int tid,
                                             int threads) {
    const Shape &sh = a.s;
    const int i0 = r.pair * 2 * s.tokens, n = min(2 * s.tokens, r.x.n - i0);
    for (int u = tid; u < n * 32; u += threads) {   // 16-byte units: token, K or V, unit
        const int i = i0 + (u >> 5), kv = u >> 4 & 1, c = u & 15;
        const int pos = r.x.P + i, j = pos / sh.bt;
        const int blk = a.tables[static_cast<int64_t>(r.b) * a.max_blocks + j];
        if (blk < 0 || blk >= sh.num_blocks) {
            atomicOr(a.err, kErrBadBlock);
            continue;
        }
        const int row = (((blk * sh.L + a.layer) * 2 + kv) * sh.Hkv + r.g) * sh.bt + pos - j * sh.bt;
        const uint16_t *src = (kv ? a.v_new : a.k_new) + (r.x.lo + i) * a.kv_stride + r.g * kHeadDim;
        reinterpret_cast<uint4 *>(a.hot + static_cast<int64_t>(row) * kHeadDim)[c] =
            reinterpret_cast<const uint4 *>(src)[c];
    }
}

__device__ void softmax_role(const TurnArgs &a, Smem &sm, int stream) {
    const TurnShape s = turn_shape(a);
    const int G = a.s.Hq / a.s.Hkv;
    const int row = threadIdx.x & (kTurnRows - 1);
    const uint32_t lanes = static_cast<uint32_t>(row & ~31) << 16;   // a warp has 32 lanes of tensor memory
    const uint32_t tmem = sm.tmem + lanes;
    const uint32_t s_addr = tmem + kColS + stream * kColStream, o_addr = tmem + kColO + stream * kColStream;
    uint32_t s_phase = 0, o_phase = 0;
    // A wait that ran out ends this warp's work, but not its walk: the barriers below count on every warp.
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t &phase) {
        ok = __all_sync(~0u, ok && mbar_wait(sm, bar, phase));
        phase ^= 1;
        fence_after();
    };
    Walk walk(sm.plan);
    Run r;
    while (walk.next(a, sm.plan, r)) {
        const int tile = r.narrow ? 2 * r.pair : 2 * r.pair + stream;
        const int token = tile * s.tokens + row / G;          // of the session's new ones
        const bool live = token < r.x.n;
        const int64_t out_row = (static_cast<int64_t>(r.x.lo) + token) * a.s.Hq + r.g * G + row % G;
        uint64_t mask = 0;
        if (a.masks && live) mask = a.masks[r.x.lo + token];
        Stats st = {-INFINITY, 0.f};
        const int step = r.narrow ? 2 : 1;
        const int t_first = r.narrow ? r.t0 + stream : r.t0;
        for (int t = t_first; ok && t < r.t1; t += step) {
            wait(&sm.s_full[stream], s_phase);
            if (!ok) break;
            softmax_tile(a, r, t, token, mask, s_addr, o_addr, t == t_first, st);
            fence_before();
            mbar_arrive(&sm.p_full[stream]);
        }
        if (ok && t_first < r.t1) wait(&sm.o_full[stream], o_phase);
        // A narrow item: stream 0 takes both streams' results together.
        float w = 1.f, w_other = 0.f;
        uint32_t other = 0;
        if (r.narrow) {
            if (stream == 1) {
                sm.other_m[row] = st.m;
                sm.other_l[row] = st.l;
            }
            sync_threads(3, 2 * kTurnRows);
            if (stream == 0 && r.t1 - r.t0 > 1) {
                const float m1 = sm.other_m[row], l1 = sm.other_l[row], m = fmaxf(st.m, m1);
                const float ref = m == -INFINITY ? 0.f : m;
                w = ex2(st.m - ref);
                w_other = ex2(m1 - ref);
                st.l = st.l * w + l1 * w_other;
                st.m = m;
                other = tmem + kColO + kColStream;
            }
        }
        const bool whole = r.t0 == 0 && r.t1 == r.tiles;
        if (!(r.narrow && stream == 1)) {
            if (whole) {
                const float inv = st.l > 0.f || st.l != st.l ? __frcp_rn(st.l) : 0.f;   // nothing seen: zeros
                const auto put = [&](int d, const float (&y)[32]) {
                    if (live) store_out(a, out_row, d, y);
                };
                if (ok && other) read_o<true>(o_addr, w * inv, other, w_other * inv, put);
                else if (ok) read_o<false>(o_addr, w * inv, 0, 0.f, put);
            } else {
                int c0, c1;
                turn_item_pieces(sm.plan.W, sm.plan.pieces, r.t0 > 0 ? sm.plan.begin_at : sm.plan.end_at, r.tiles,
                                 turn_tile_cost(s, r.x, r.pair), &c0, &c1);
                const int slot = r.t0 > 0 ? 2 * blockIdx.x : 2 * blockIdx.x + 1;
                float4 *po = part_o(a, slot, stream);
                const auto put = [&](int d, const float (&y)[32]) {
                    if (!live) return;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        po[(d / 4 + i) * kTurnRows + row] =
                            make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
                };
                if (ok && other) read_o<true>(o_addr, w, other, w_other, put);
                else if (ok) read_o<false>(o_addr, w, 0, 0.f, put);
                if (live) part_ml(a, slot, stream)[row] = make_float2(st.m, st.l);
                __threadfence();
                sync_threads(1 + stream, kTurnRows);
                int32_t *counter = a.part_counters + 2 * c0 + stream;
                if (row == 0) sm.last[stream] = ok && arrive(counter) == c1 - c0;
                sync_threads(1 + stream, kTurnRows);
                if (sm.last[stream]) {   // the item's last piece to finish: merge all, in order
                    __threadfence();
                    if (row == 0) *counter = 0;
                    if (live) {
                        float m = -INFINITY;
                        for (int c = c0; c <= c1; ++c)
                            m = fmaxf(m, __ldcg(part_ml(a, c == c0 ? 2 * c + 1 : 2 * c, stream) + row).x);
                        const float ref = m == -INFINITY ? 0.f : m;
                        float l = 0.f;
                        for (int c = c0; c <= c1; ++c) {
                            const float2 v = __ldcg(part_ml(a, c == c0 ? 2 * c + 1 : 2 * c, stream) + row);
                            l = __fmaf_rn(ex2(v.x - ref), v.y, l);
                        }
                        const float inv = l > 0.f || l != l ? __frcp_rn(l) : 0.f;
#pragma unroll 1
                        for (int d = 0; d < kHeadDim; d += 32) {
                            float y[32] = {};
                            for (int c = c0; c <= c1; ++c) {
                                const int from = c == c0 ? 2 * c + 1 : 2 * c;
                                const float f = ex2(__ldcg(part_ml(a, from, stream) + row).x - ref);
                                const float4 *pc = part_o(a, from, stream) + d / 4 * kTurnRows + row;
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    const float4 o = __ldcg(pc + i * kTurnRows);
                                    y[4 * i] = __fmaf_rn(f, o.x, y[4 * i]);
                                    y[4 * i + 1] = __fmaf_rn(f, o.y, y[4 * i + 1]);
                                    y[4 * i + 2] = __fmaf_rn(f, o.z, y[4 * i + 2]);
                                    y[4 * i + 3] = __fmaf_rn(f, o.w, y[4 * i + 3]);
                                }
                            }
#pragma unroll
                            for (int i = 0; i < 32; ++i) y[i] *= inv;
                            store_out(a, out_row, d, y);
                        }
                    }
                }
            }
        }
        // Once per item: by the piece that has its last key tile.
        if (!a.masks && r.t1 == r.tiles) store_new_kv(a, s, r, threadIdx.x, 2 * kTurnRows);
        fence_before();
        // Stream 1's O is free for its next product once stream 0 has read it.
        if (r.narrow) sync_threads(3, 2 * kTurnRows);
    }
}

__global__ void __launch_bounds__(kThreads, 1) turn_kernel(const __grid_constant__ TurnArgs a,
                                                           const __grid_constant__ Maps maps) {
    extern __shared__ uint8_t raw[];
    Smem &sm = *reinterpret_cast<Smem *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == kCopyWarp) make_plan(a, sm.plan, lane);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sm.kv_full[i], 1);
            mbar_init(&sm.kv_empty[i], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sm.q_full[s], 1);
            mbar_init(&sm.s_full[s], 1);
            mbar_init(&sm.p_full[s], kTurnRows);
            mbar_init(&sm.o_full[s], 1);
        }
        mbar_init(&sm.q_empty, 1);
        mbar_init(&sm.drained, 1);
        sm.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (blockIdx.x < sm.plan.pieces) {
        if (warp < 8) {
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
            softmax_role(a, sm, warp >> 2);
        } else {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
            if (warp == kCopyWarp) copy_role(a, maps, sm, lane);
            else if (warp == kMmaWarp) mma_role(a, sm);
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x == 0 && sm.abort) atomicOr(a.err, kErrTimeout);
    if (warp == kMmaWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sm.tmem), "r"(kTmemCols));
}

}  // namespace

// Floats and counters that a launch of `ctas` CTAs may need.
int64_t turn_part_floats(int ctas) { return int64_t(2) * ctas * 2 * kTurnRows * (kHeadDim + 2); }
int64_t turn_counters(int ctas) { return int64_t(2) * ctas; }

bool encode_turn_hot_map(CUtensorMap *map, void *hot_base, int64_t rows, const char **why) {
    const cuuint64_t dims[3] = {64, static_cast<cuuint64_t>(rows), 2};
    const cuuint64_t strides[2] = {kRowBytes, 128};
    const cuuint32_t box[3] = {64, kBoxRows, 1};
    return encode_bf16_map(map, hot_base, 3, dims, strides, box, why);
}

cudaError_t launch_turn(TurnArgs a, const CUtensorMap &hot, cudaStream_t st) {
    if (a.total < 1) return cudaSuccess;
    const int G = a.s.Hq / a.s.Hkv;
    Maps maps;
    maps.hot = hot;
    const cuuint64_t n = static_cast<cuuint64_t>(a.total);
    // [token][head][column half][64 columns], the halves outermost
    const cuuint64_t q_dims[4] = {64, static_cast<cuuint64_t>(a.s.Hq), n, 2};
    const cuuint64_t q_strides[3] = {kRowBytes, static_cast<cuuint64_t>(a.q_stride) * 2, 128};
    const cuuint32_t q_box[4] = {64, static_cast<cuuint32_t>(G), static_cast<cuuint32_t>(kTurnRows / G), 1};
    const cuuint64_t kv_dims[4] = {64, static_cast<cuuint64_t>(a.s.Hkv), n, 2};
    const cuuint64_t kv_strides[3] = {kRowBytes, static_cast<cuuint64_t>(a.kv_stride) * 2, 128};
    const cuuint32_t kv_box[4] = {64, 1, kBoxRows, 1};
    const char *why = nullptr;
    if (!encode_bf16_map(&maps.q, const_cast<uint16_t *>(a.q), 4, q_dims, q_strides, q_box, &why) ||
        !encode_bf16_map(&maps.k, const_cast<uint16_t *>(a.k_new), 4, kv_dims, kv_strides, kv_box, &why) ||
        !encode_bf16_map(&maps.v, const_cast<uint16_t *>(a.v_new), 4, kv_dims, kv_strides, kv_box, &why))
        return cudaErrorInvalidValue;
    // The scores' sign goes into the product, so that the largest score is the largest scaled one; a
    // scale of 0 (all weights equal) stays a positive one, which masked scores keep apart.
    a.negate = a.scale_log2 < 0.f;
    a.scale_log2 = fmaxf(fabsf(a.scale_log2), 1e-30f);
    turn_kernel<<<a.part_slots / 2, kThreads, kSmemBytes, st>>>(a, maps);
    return cudaGetLastError();
}

cudaError_t prepare_turn_kernel() {
    // The warps' register shares presume the launch's.
    cudaFuncAttributes f;
    cudaError_t e = cudaFuncGetAttributes(&f, turn_kernel);
    if (e == cudaSuccess && f.numRegs != kRegsLaunch) e = cudaErrorInvalidConfiguration;
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(turn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
}

}  // namespace kvt
