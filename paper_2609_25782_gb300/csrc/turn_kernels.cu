// Attention of several new tokens per session over the paged cache, for sm_103a:
// a turn's context or a whole prompt (causal, its K and V written into the hot
// pool), and drafted tokens (a bit mask per draft, nothing written).
//
// Per row, over key tiles: S = Q K^T; with c = scale log2(e), m the running maximum of c S and l the running
// sum, weights P = 2^(c S - m), O = O 2^(m_before - m) + P V, l likewise; out = O / l. Pieces i of a row's
// keys are merged with the weights 2^(m_i - m).
//
// turn_kernel: one persistent CTA per SM works through its piece of the line of items that
// turn_plan.h lays out. The query heads that share a kv-head are packed into the
// 128 rows of a row tile, so K and V are read once for all of them. A CTA has two
// streams, each with a row tile's scores and output in tensor memory: two row
// tiles of a pair against the same key tile, or (narrow items) every other key
// tile against one row tile. Roles, by warp:
//   0-3, 4-7  softmax of stream 0 and 1, a thread per row: scores from tensor
//             memory, running maximum and sum in 32 bits, weights back to tensor
//             memory in bf16; at the end the output
//   8         the plan, then copies: q tiles and key tiles (TMA, 128-byte swizzle)
//   9, 10     matrix products (tcgen05) of stream 0 and 1: S = Q K^T from shared
//             memory, O += P V with P from tensor memory
//   11        the new tokens' K and V, into the pool
// The tensor cores work on one stream while the other's softmax runs. P lies in S's place, so a stream's
// next scores wait for the product of its weights: a key tile of a pair takes 3 250 (turns) to 3 500 cycles
// (one long prompt), of which the products need 2 050, and that chain bounds both (tensor pipe 63 and 58 %
// active; no case got faster with three quarters of the exponentials left out, or the maximum). Tensor memory has room for S beside P with
// key tiles of 80: 5 % slower, because a product of 80 columns takes 80 % of one of 128. Two threads a row:
// 20 % slower, 64 scores do not fit the registers of 640 threads. Few rows over long caches are bound by HBM.
// In a CUDA graph of twenty calls (called one by one: 1 600, 962, 103 and 12 us):
//   one prompt of 16 391 tokens, 32 heads (4 KV)           1 590 us   1 385 TFLOP/s
//   turns of 300-3K tokens on 2K-24K, 4 sessions             945 us   1 320 TFLOP/s
//   16 sessions of 2K-30K tokens, 16 drafts each              99 us   5.5 TB/s, with the merge
//   one prompt of 37 tokens                                    9 us   plan, load, product, softmax, end in turn
//
// turn_combine_kernel merges the partial results of items that lie in several
// pieces, in the pieces' order; it is a programmatic dependent of turn_kernel.
#include <cuda_bf16.h>

#include <algorithm>

#include "kvt_internal.h"
#include "turn_plan.h"

namespace kvt {
namespace {

constexpr int kTileBytes = kTurnKeys * kRowBytes;   // a key or row tile, 32 KB
// Its rows' halves (columns 0-63 and 64-127, 128 B each) lie in one of two orders. Whole: all rows'
// first halves, then all second ones; a q tile, or a tile of the call's own tokens, is one copy or two.
// Grouped: eight rows' first halves, their second halves, the next eight rows'; so a block of the
// pool is one copy, whatever its place in the tile.
constexpr int kHalfWhole = kTileBytes / 2, kHalfGrouped = 1024;   // bytes from a row's half to the other
constexpr int kGroupWhole = 1024, kGroupGrouped = 2048;           // bytes from eight rows to the next
constexpr int kBoxRows = 16;                        // rows that a copy at the end of the keys has
constexpr int kStages = 5;                          // K or V tiles in flight
constexpr int kThreads = 384;
constexpr int kCopyWarp = 8, kMmaWarp = 9, kStoreWarp = 11;
// Registers per thread: at launch, then of the softmax warps and of the others. A softmax thread
// keeps its row's 128 scores; the shares add up to what the CTA was launched with.
constexpr int kRegsLaunch = 168, kRegsSoftmax = 184, kRegsOther = 136;
static_assert(256 * kRegsSoftmax + 128 * kRegsOther <= kThreads * kRegsLaunch, "a larger share would wait forever");
constexpr unsigned long long kWaitLimitNs = 2000000000ull;   // 2 s

// Tensor memory: 128 columns of 32 bits each for S (and P in its lower half) and O of both streams.
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256, kColStream = 128;

// A run of key tiles t0 .. t1 - 1 of one item; tiles 0: no more runs.
struct alignas(16) Run {
    int32_t lo, n, P, b;   // the session: first row, new tokens, cached ones, its number
    int32_t g, pair, t0, t1;
    int32_t tiles, cached_tiles, own_keys, narrow;
};
constexpr int kRuns = 4;        // runs that the copies may be ahead of the other roles
constexpr int kRunReaders = 11;   // warps: softmax, products, store

struct Plan {
    TurnPos begin, end;
    TurnSession first;   // the session of `begin`, n < 0: not at hand
};

struct alignas(1024) Smem {
    uint8_t q[2][kTileBytes];
    uint8_t kv[kStages][kTileBytes];
    // The ring's copies have landed: two barriers a stage, for its even and its odd rounds. A stream of a
    // narrow item does not look at the other's tiles, so it may ask for a stage's next round while the
    // present one is still on its way; with one barrier, a parity, that would pass as done.
    uint64_t kv_full[2 * kStages], kv_empty[kStages];
    uint64_t q_full[2], q_empty, s_full[2], p_full[2], o_full[2], drained[2];
    uint64_t run_full[kRuns], run_empty[kRuns], other_ready, other_free;
    Run runs[kRuns];
    Plan plan;
    float other_m[kTurnRows], other_l[kTurnRows];   // narrow items: stream 1's statistics
    uint32_t tmem;
    int32_t abort;
    int32_t issuing;                 // a stream's products are going out
};
constexpr int kSmemBytes = sizeof(Smem) + 1024;     // and the way to a 1 024-byte boundary
static_assert(kSmemBytes <= 227 * 1024, "shared memory of a CTA");

struct Maps {
    CUtensorMap q;                       // [half][token][head] rows, a row tile a copy
    CUtensorMap k, v, k_whole, v_whole;  // kBoxRows rows' halves a copy, or a tile
    CUtensorMap hot, hot_block;          // kBoxRows grouped rows a copy, or a block
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
#pragma unroll 1
    while (!mbar_try(bar, parity)) {
        if (*reinterpret_cast<volatile int32_t *>(&sm.abort)) return false;
        if (global_ns() - t0 > kWaitLimitNs) {
            *reinterpret_cast<volatile int32_t *>(&sm.abort) = 1;
            return false;
        }
    }
    return true;
}

__device__ __forceinline__ void copy_box(void *dst, const CUtensorMap *map, int c1, int c2, int c3, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}

// The same, its lines the first to leave the L2.
__device__ __forceinline__ uint64_t policy_once() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void copy_box_once(void *dst, const CUtensorMap *map, int c3, uint64_t *bar, uint64_t policy) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %2, %2, %3}], [%4], %5;" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(c3), "r"(smem_u32(bar)), "l"(policy)
        : "memory");
}

// Shared-memory operand, 128-byte swizzle: rows of 128 B in groups of eight, `group` bytes from one to
// the next. An operand that is summed over its rows (V) has its two column halves `half` bytes apart;
// where the sum runs along the rows (Q, K) that field is not used.
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t half, uint32_t group) {
    return static_cast<uint64_t>(addr >> 4 & 0x3FFF) | static_cast<uint64_t>(half >> 4) << 16 |
           static_cast<uint64_t>(group >> 4) << 32 | 1ull << 46 | 2ull << 61;
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

// One lane of the warp.
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(~0u, x, 0); }

#define KVT_R8(x, o) "=r"(x[o]), "=r"(x[o + 1]), "=r"(x[o + 2]), "=r"(x[o + 3]), "=r"(x[o + 4]), "=r"(x[o + 5]), \
        "=r"(x[o + 6]), "=r"(x[o + 7])
#define KVT_U8(x, o) "r"(x[o]), "r"(x[o + 1]), "r"(x[o + 2]), "r"(x[o + 3]), "r"(x[o + 4]), "r"(x[o + 5]), \
        "r"(x[o + 6]), "r"(x[o + 7])
#define KVT_RW8(x, o) "+r"(x[o]), "+r"(x[o + 1]), "+r"(x[o + 2]), "+r"(x[o + 3]), "+r"(x[o + 4]), "+r"(x[o + 5]), \
        "+r"(x[o + 6]), "+r"(x[o + 7])

// 32 or 16 columns of this thread's row. The values are there after tmem_wait on them.
__device__ __forceinline__ void tmem_load(uint32_t (&x)[32], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,"
        "%28,%29,%30,%31}, [%32];"
        : KVT_R8(x, 0), KVT_R8(x, 8), KVT_R8(x, 16), KVT_R8(x, 24)
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t (&x)[16], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : KVT_R8(x, 0), KVT_R8(x, 8)
        : "r"(addr)
        : "memory");
}
// 32 columns of 16 rows (from the address's lane on) shared out as a matrix fragment: lane l has columns
// 8 g + 2 (l % 4) and the next of rows l / 4, in x[4 g] and x[4 g + 1], and l / 4 + 8, in the two after.
__device__ __forceinline__ void tmem_load_rows(uint32_t (&x)[16], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : KVT_R8(x, 0), KVT_R8(x, 8)
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&x)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" : KVT_RW8(x, 0), KVT_RW8(x, 8)::"memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&x)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : KVT_RW8(x, 0), KVT_RW8(x, 8), KVT_RW8(x, 16), KVT_RW8(x, 24)::"memory");
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&x)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::KVT_U8(x, 0),
        KVT_U8(x, 8), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&x)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::KVT_U8(x, 0), "r"(addr)
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

// ---- the work ----------------------------------------------------------------------------

__host__ __device__ __forceinline__ TurnShape turn_shape(const TurnArgs &a, bool many = false) {
    return {a.token_shift, a.s.Hkv, a.masks == nullptr, many};
}

// Session b as the call describes it; n = 0 for one whose data is out of range.
__device__ __forceinline__ TurnSession session_of(const TurnArgs &a, int b, bool *bad = nullptr) {
    const int lo = a.cu[b], hi = a.cu[b + 1], T = a.seq_lens[b];
    const bool drafts = a.masks != nullptr, order = lo >= 0 && lo <= hi && hi <= a.total;
    const int n = order ? hi - lo : 0;
    const bool ok = order && T >= (drafts ? 0 : n) && T <= a.longest && !(drafts && n > kMaxDrafts);
    if (bad) *bad = !ok;
    return {ok ? n : 0, !ok ? 0 : drafts ? T : T - n, lo};
}

// Sum of x over the lanes before this one, and over all.
template <typename I>
__device__ __forceinline__ I scan(I x, int lane, I *all) {
    I y = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const I z = __shfl_up_sync(~0u, y, d);
        if (lane >= d) y += z;
    }
    *all = __shfl_sync(~0u, y, 31);
    return y - x;
}

// This CTA's piece, by one warp. (Short code: a call runs it once, and nothing else can begin before. So the
// costs are constants in it, and the launch has chosen them.)
template <typename I, bool kMany>
__device__ __forceinline__ void make_plan(const TurnArgs &a, Plan &plan, int lane) {
    const TurnShape s = turn_shape(a, kMany);
    TurnSession x = {0, 0, 0};   // up to 32 sessions: kept, with what goes before, for the cuts
    I head = 0, at = 0, W = 0, all;
#pragma unroll 1
    for (int b = lane; b - lane < a.B; b += 32) {
        head = 0;
        if (b < a.B) {
            bool bad;
            x = session_of(a, b, &bad);
            head = turn_head_cost<I>(s, x);
            if (bad && blockIdx.x == 0) atomicOr(a.err, kErrBadLength);
        }
        at = W + scan(s.Hkv * head, lane, &all);
        W += all;
    }
    const int pieces = W == 0 ? 0 : turn_pieces(s, W, gridDim.x), c = blockIdx.x;
    if (lane == 0) plan.begin = plan.end = {a.B, 0, 0, 0};   // no piece; a last piece's end
    __syncwarp();
    if (c >= pieces) return;
    const I u[2] = {turn_cut(W, pieces, c), turn_cut(W, pieces, c + 1)};
    W = 0;
#pragma unroll 1
    for (int b = lane; b - lane < a.B; b += 32) {
        if (a.B > 32) {
            head = 0;
            if (b < a.B) {
                x = session_of(a, b);
                head = turn_head_cost<I>(s, x);
            }
            at = W + scan(s.Hkv * head, lane, &all);
            W += all;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if (u[e] < at || u[e] >= at + s.Hkv * head) continue;
            TurnPos p = turn_locate<I>(s, x, b, head, u[e] - at);
            if (p.t >= turn_tiles(s, x, p.pair) || (a.whole && p.t > 0)) {   // the item's end: the next one's start
                p.t = 0;
                if (++p.pair >= turn_pairs(s, x)) {
                    p.pair = 0;
                    if (++p.g >= s.Hkv) {
                        p.g = 0;
                        ++p.b;   // an empty session here is passed over by the walk
                    }
                }
            }
            if (e) {
                plan.end = p;
            } else {
                plan.begin = p;
                plan.first = x;
                if (p.b != b) plan.first.n = -1;
            }
        }
    }
    __syncwarp();
}

// The runs of a piece, in order.
struct Walk {
    TurnPos at, end;
    TurnSession x;   // of at.b
    __device__ Walk(const TurnArgs &a, const Plan &plan) : at(plan.begin), end(plan.end), x(plan.first) {
        if (at.b < a.B && x.n < 0) x = session_of(a, at.b);
    }
    __device__ bool next(const TurnArgs &a, Run &r) {
        const TurnShape s = turn_shape(a);
        while (at.b < a.B) {
            const bool to_end = at.b == end.b && at.g == end.g && at.pair == end.pair;
            if ((to_end && at.t >= end.t) || (x.n == 0 && at.b == end.b)) return false;
            if (x.n > 0) {
                r.lo = x.lo;
                r.n = x.n;
                r.P = x.P;
                r.b = at.b;
                r.g = at.g;
                r.pair = at.pair;
                r.cached_tiles = turn_tiles_of(x.P);
                r.own_keys = turn_own_keys(s, x, at.pair);
                r.tiles = r.cached_tiles + turn_tiles_of(r.own_keys);
                r.narrow = turn_narrow(s, x, at.pair);
                r.t0 = at.t;
                r.t1 = to_end ? end.t : r.tiles;
                at.t = r.t1;
                if (to_end) return true;
                at.t = 0;
                if (++at.pair < turn_pairs(s, x)) return true;
                at.pair = 0;
                if (++at.g < s.Hkv) return true;
            }
            const bool any = x.n > 0;   // else nothing of this session: the next one
            at = {at.b + 1, 0, 0, 0};
            if (at.b < a.B) x = session_of(a, at.b);
            if (any) return true;
        }
        return false;
    }
};

// The runs as the copies' warp publishes them, for a warp of another role. Each is read once, then given back.
struct Reader {
    uint32_t count = 0;
    __device__ bool next(Smem &sm, Run &r) {
        const int slot = count % kRuns;
        if (!__all_sync(~0u, mbar_wait(sm, &sm.run_full[slot], count / kRuns & 1))) return false;
        r = sm.runs[slot];
        return r.tiles > 0;
    }
    __device__ void done(Smem &sm) {
        __syncwarp();
        if (threadIdx.x % 32 == 0) mbar_arrive(&sm.run_empty[count % kRuns]);
        ++count;
    }
};

// Keys of key tile t of an item.
__device__ __forceinline__ int keys_of(const Run &r, int t) {
    const int left = t < r.cached_tiles ? r.P - t * kTurnKeys : r.own_keys - (t - r.cached_tiles) * kTurnKeys;
    return min(left, kTurnKeys);
}

// ---- copies ------------------------------------------------------------------------------

// Lane l's block of key tile t: that of its keys 16 l and on, where there are any.
__device__ __forceinline__ int block_id(const TurnArgs &a, const Run &r, int t, int lane) {
    const int pos = t * kTurnKeys + lane * kBoxRows;
    if (t >= r.cached_tiles || lane >= kTurnKeys / kBoxRows || pos >= r.P) return 0;
    return a.tables[static_cast<int64_t>(r.b) * a.max_blocks + (a.s.bt == 64 ? pos >> 6 : pos >> 4)];
}
// The row of the pool (below 2^31) of those keys' K.
__device__ __forceinline__ int pool_row(const TurnArgs &a, const Run &r, int t, int blk, int lane) {
    const Shape &sh = a.s;
    if (blk < 0 || blk >= sh.num_blocks) {
        atomicOr(a.err, kErrBadBlock);
        blk = 0;   // the result is wrong, the access is not
    }
    return ((blk * sh.L + a.layer) * 2 * sh.Hkv + r.g) * sh.bt + ((t * kTurnKeys + lane * kBoxRows) & (sh.bt - 1));
}

// The keys past a tile's last full group of 16 come by plain loads, and rows up to the group's end are
// cleared: what they hold in memory may be anything, and a weight of 0 does not make a NaN go away in the
// product with V. A lane has 16 bytes of every other row. The loads go out before the copies wait for a
// stage: one after the other, or after that wait, they held up every item's end by thousands of cycles.
constexpr int kRestRows = kBoxRows / 2;
struct Rest {
    uint4 x[kRestRows];
};
__device__ __forceinline__ void load_rest(Rest &r, const uint16_t *src, int64_t step, int rest, int lane) {
#pragma unroll
    for (int i = 0; i < kRestRows; ++i)   // no branch, so that all are on their way together
        r.x[i] = *reinterpret_cast<const uint4 *>(src + min(2 * i + (lane >> 4), rest - 1) * step + (lane & 15) * 8);
}
__device__ __forceinline__ void store_rest(Rest &r, int rest, uint8_t *stage, int row0, bool grouped, int lane) {
    const int u = lane & 15, half = grouped ? kHalfGrouped : kHalfWhole, group = grouped ? kGroupGrouped : kGroupWhole;
#pragma unroll
    for (int i = 0; i < kRestRows; ++i) {
        const int rr = 2 * i + (lane >> 4), row = row0 + rr;
        if (rr >= rest) r.x[i] = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4 *>(stage + (row >> 3) * group + (u >> 3) * half + (row & 7) * 128 +
                                   (((u & 7) ^ (row & 7)) << 4)) = r.x[i];
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

// The full groups of a K (kv = 0) or V tile into a stage, by the warp: cached keys grouped, a copy per
// block (row: that of the lane's keys), the call's own whole.
__device__ __forceinline__ void copy_groups(const TurnArgs &a, const Maps &maps, const Run &r, int groups, int rest, bool cached,
                                            int first, int row, int kv, uint8_t *stage, uint64_t *full, bool once) {
    const bool leader = elected();
    // Own keys that fill their groups come in one copy; rows past them, of later tokens or other sessions,
    // are not read.
    if (leader) mbar_expect(full, cached || rest ? groups * kBoxRows * kRowBytes : kTileBytes);
    // Each copy names its map by itself: with the map selected before, a copy took three times as long to issue.
    if (cached) {   // coordinates: (column, row of eight, half, eight rows)
        const auto copy_all = [&](auto box) {
            int i = 0;
            if (a.s.bt == 64)   // whole blocks
                for (; i + 4 <= groups; i += 4) {
                    const int at = __shfl_sync(~0u, row, i) >> 3;
                    if (leader) box(stage + i * 2 * kGroupGrouped, &maps.hot_block, at);
                }
            if (i == 0 && groups == kTurnKeys / kBoxRows) {
#pragma unroll
                for (int k = 0; k < kTurnKeys / kBoxRows; ++k) {
                    const int at = __shfl_sync(~0u, row, k) >> 3;
                    if (leader) box(stage + k * 2 * kGroupGrouped, &maps.hot, at);
                }
            } else {
                for (; i < groups; ++i) {
                    const int at = __shfl_sync(~0u, row, i) >> 3;
                    if (leader) box(stage + i * 2 * kGroupGrouped, &maps.hot, at);
                }
            }
        };
        if (once) {
            const uint64_t policy = policy_once();
            copy_all([&](uint8_t *to, const CUtensorMap *map, int at) { copy_box_once(to, map, at, full, policy); });
        } else {
            copy_all([&](uint8_t *to, const CUtensorMap *map, int at) { copy_box(to, map, 0, 0, at, full); });
        }
    } else if (leader) {
        if (!rest) {                            // (column, token, half, head)
            if (kv) copy_box(stage, &maps.v_whole, first, 0, r.g, full);
            else copy_box(stage, &maps.k_whole, first, 0, r.g, full);
        } else {                                // (column, head, token, half)
#pragma unroll 1
            for (int i = 0; i < 2 * groups; ++i) {
                uint8_t *to = stage + (i & 1) * kHalfWhole + (i >> 1) * kBoxRows * 128;
                if (kv) copy_box(to, &maps.v, r.g, first + (i >> 1) * kBoxRows, i & 1, full);
                else copy_box(to, &maps.k, r.g, first + (i >> 1) * kBoxRows, i & 1, full);
            }
        }
    }
    __syncwarp();
}

__device__ void copy_role(const TurnArgs &a, const Maps &maps, Smem &sm, int lane) {
    const TurnShape s = turn_shape(a);
    int stage = 0, round = 0, items = 0, pairs = 0;
    uint32_t filled = 0, runs = 0;   // copies issued so far, saturating at kStages; runs published
    bool ok = true;                  // the same in all lanes until the last copy is out
    Walk walk(a, sm.plan);
    // (A test of the bounded waits, 0 in normal calls: the first copy's barrier expects more than comes.)
    if (a.inject_extra_tx && blockIdx.x == 0 && lane == 0)
        asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(&sm.kv_full[0])),
                     "r"(a.inject_extra_tx)
                     : "memory");
    __syncwarp();
#pragma unroll 1
    while (ok) {
        Run r;
        r.tiles = 0;
        const bool more = walk.next(a, r);
        if (runs >= kRuns)
            ok = __all_sync(~0u, mbar_wait(sm, &sm.run_empty[runs % kRuns], (runs / kRuns - 1) & 1));
        if (ok && lane == 0) {
            sm.runs[runs % kRuns] = r;
            mbar_arrive(&sm.run_full[runs % kRuns]);
        }
        ++runs;
        if (!more) break;
        int blk = block_id(a, r, r.t0, lane);
        // K and V that no other item reads (one pair) leave the L2 first: what every call needs stays there, the
        // tables, the maps and this code, without which a CTA's first copy went out 5 us later (16 sessions'
        // drafts 103 -> 99 us, 32 sessions' 125 -> 117.5).
        const bool once = r.n <= 2 << s.shift;
        if (ok && items > 0) ok = __all_sync(~0u, mbar_wait(sm, &sm.q_empty, (items - 1) & 1));
        if (!ok) break;
        ++items;
        pairs += !r.narrow;
        if (elected())   // coordinates: (column, head, token, half)
#pragma unroll 1
            for (int i = 0; i < turn_q_tiles(r.narrow); ++i) {
                mbar_expect(&sm.q_full[i], kTileBytes);
                copy_box(sm.q[i], &maps.q, r.g << (7 - s.shift), r.lo + ((2 * r.pair + i) << s.shift), 0, &sm.q_full[i]);
            }
        __syncwarp();
#pragma unroll 1
        for (int t = r.t0; ok && t < r.t1; ++t) {
            const int keys = keys_of(r, t), groups = keys / kBoxRows, rest = keys % kBoxRows;
            const bool cached = t < r.cached_tiles;
            const int first = r.lo + (t - r.cached_tiles) * kTurnKeys;   // own keys: row of k_new and v_new
            const int row = pool_row(a, r, t, blk, lane), v_rows = a.s.Hkv * a.s.bt;
            Rest extra;
            const uint16_t *rest_k = nullptr, *rest_v = nullptr;
            const int64_t step = cached ? kHeadDim : a.kv_stride;
            if (rest) {
                const int at = __shfl_sync(~0u, row, groups);
                const int64_t own = (static_cast<int64_t>(first) + groups * kBoxRows) * a.kv_stride + r.g * kHeadDim;
                rest_k = cached ? a.hot + static_cast<int64_t>(at) * kHeadDim : a.k_new + own;
                rest_v = cached ? rest_k + static_cast<int64_t>(v_rows) * kHeadDim : a.v_new + own;
                load_rest(extra, rest_k, step, rest, lane);
            }
            // The next tile's block ids are on their way while this one's copies go out.
            if (t + 1 < r.t1) blk = block_id(a, r, t + 1, lane);
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
                if (ok && round > 0) ok = __all_sync(~0u, mbar_wait(sm, &sm.kv_empty[stage], (round - 1) & 1));
                if (!ok) break;
                if (rest) {
                    store_rest(extra, rest, sm.kv[stage], groups * kBoxRows, cached, lane);
                    if (kv == 0) load_rest(extra, rest_v, step, rest, lane);
                }
                copy_groups(a, maps, r, groups, rest, cached, first, row + kv * v_rows, kv, sm.kv[stage],
                            &sm.kv_full[stage + (round & 1) * kStages], once);
                if (filled < kStages) ++filled;
                if (++stage == kStages) {
                    stage = 0;
                    ++round;
                }
            }
        }
    }
    // Every copy lands before the CTA ends, whatever became of the other roles; with all well,
    // every stage has been given back as well.
#pragma unroll 1
    for (uint32_t i = 0; i < filled; ++i) {
        const bool now = static_cast<int>(i) < stage;   // filled in this round, or in the one before
        const int last = now ? round : round - 1;
        if (ok) ok = mbar_wait(sm, &sm.kv_empty[i], last & 1);
        const unsigned long long t0 = global_ns();
        while (!mbar_try(&sm.kv_full[i + (last & 1) * kStages], last >> 1 & 1) && global_ns() - t0 < kWaitLimitNs) {}
    }
    if (ok && items > 0) ok = mbar_wait(sm, &sm.q_empty, (items - 1) & 1);
#pragma unroll 1
    for (int i = 0; !ok && i < 2; ++i) {   // and the last q tiles
        const int loads = i ? pairs : items;
        const unsigned long long t0 = global_ns();
        while (loads > 0 && !mbar_try(&sm.q_full[i], (loads - 1) & 1) && global_ns() - t0 < kWaitLimitNs) {}
    }
}

// ---- matrix products -----------------------------------------------------------------------

// S = Q K^T. The steps' operands lie a constant apart: one addition per step and operand, so that the
// issuing thread keeps up with the tensor cores (64 cycles a step).
__device__ __forceinline__ void product_qk(uint32_t d, uint32_t q, uint32_t k, bool grouped, uint32_t form) {
    const uint64_t a = operand(q, 16, kGroupWhole), b = operand(k, 16, grouped ? kGroupGrouped : kGroupWhole);
    const uint32_t half = (grouped ? kHalfGrouped : kHalfWhole) >> 4;
#pragma unroll
    for (int i = 0; i < kHeadDim / 16; ++i)
        mma_ss(d, a + (((i >> 2) * kHalfWhole + (i & 3) * 32) >> 4), b + ((i >> 2) * half + ((i & 3) * 32 >> 4)), form,
               i > 0);
}
// O += P V over 16 * steps keys, or (!add) O = P V.
__device__ __forceinline__ void product_pv(uint32_t d, uint32_t p, uint32_t v, bool grouped, int steps, bool add) {
    uint64_t b = grouped ? operand(v, kHalfGrouped, kGroupGrouped) : operand(v, kHalfWhole, kGroupWhole);
    const uint32_t step = 2 * (grouped ? kGroupGrouped : kGroupWhole) >> 4;
    const uint32_t form = mma_form(kHeadDim, true, false);
    if (steps == kTurnKeys / 16) {
#pragma unroll
        for (int i = 0; i < kTurnKeys / 16; ++i) mma_ts(d, p + i * 8, b + i * step, form, i > 0 || add);
    } else {
#pragma unroll 1
        for (int i = 0; i < steps; ++i, b += step) mma_ts(d, p + i * 8, b, form, i > 0 || add);
    }
}

// The products of one stream. The whole warp walks and waits, one lane issues: control flow and operands
// are the same in all lanes, which the compiler has to see (votes, shuffles) to keep them in uniform
// registers; with one lane doing everything a step took 90 cycles to issue. Each stream has a warp, so
// that one's waits do not stand in the way of the other's products.
__device__ void mma_role(const TurnArgs &a, Smem &sm, int stream) {
    const uint32_t tmem = uniform(sm.tmem);
    const uint32_t s_col = tmem + kColS + stream * kColStream, o_col = tmem + kColO + stream * kColStream;
    const bool negate = a.negate != 0;
    uint32_t items = 0, pairs = 0, p_phase = 0;
    uint32_t base = 0;   // tiles of the runs before: tile n has K at place 2n of the ring's sequence, V at 2n + 1
    bool ok = true;
    auto wait = [&](uint64_t *bar, uint32_t parity) { ok = __all_sync(~0u, mbar_wait(sm, bar, parity)); };
    Reader reader;
    Run r;
#pragma unroll 1
    while (ok && reader.next(sm, r)) {
        const int tiles = uniform(r.t1 - r.t0), t0 = uniform(r.t0), cached_tiles = uniform(r.cached_tiles);
        const int cached_keys = uniform(r.P), own_keys = uniform(r.own_keys);
        const bool narrow = uniform(r.narrow);
        reader.done(sm);
        const int by = narrow ? 2 : 1, first = narrow ? stream : 0;
        auto steps_of = [&](int i) {   // of 16 keys, of the run's tile i
            const int t = t0 + i;
            const int left = t < cached_tiles ? cached_keys - t * kTurnKeys : own_keys - (t - cached_tiles) * kTurnKeys;
            return left >= kTurnKeys ? kTurnKeys / 16 : (left + 15) / 16;
        };
        // A stage goes back to the copies once both streams' products are done with it; a narrow item's
        // tile has one stream.
        auto give_back = [&](int stage) {
            mma_commit(&sm.kv_empty[stage]);
            if (narrow) mma_commit(&sm.kv_empty[stage]);
        };
        const int q = narrow ? 0 : stream, q_waits = turn_q_waits(stream, narrow);
        if (q_waits & 1) wait(&sm.q_full[0], items & 1);
        if (ok && q_waits & 2) wait(&sm.q_full[1], pairs & 1);
        ++items;
        pairs += !narrow;
        // Place of the run's tile i in the ring's sequence: its stage, and the wait for it.
        auto landed = [&](uint32_t place) {
            if (ok) wait(&sm.kv_full[place % (2 * kStages)], place / (2 * kStages) & 1);
        };
        if (first >= tiles && elected()) mma_commit(&sm.q_empty);   // no tile for this stream
        __syncwarp();
        // Step i: the products with V of tile i - by, then those with K of tile i, whose scores take the weights'
        // place.
#pragma unroll 1
        for (int i = first; ok && first < tiles && i < tiles + by; i += by) {
            const bool has_v = i > first, has_k = i < tiles;
            const uint32_t k_place = 2 * (base + i), v_place = 2 * (base + i - by) + 1;
            // A pair's products wait for their weights; K is there by then. One stream's go out without the
            // other's between them: taking turns step by step, both streams' softmax would wait for both
            // products, and then both products for the softmax. (Order is all that the lock decides: past the
            // limit, which no holder needs, they mix.) A narrow item waits for HBM: V's stage is given back
            // before K is asked for.
            if (!narrow && has_k) landed(k_place);
            if (has_v) {
                landed(v_place);
                if (ok) wait(&sm.p_full[stream], p_phase);
                p_phase ^= 1;
            }
            fence_after();
            const bool leader = elected();
            if (ok && leader && !narrow)
                for (int n = 0; n < 1 << 16 && atomicCAS_block(&sm.issuing, 0, 1) != 0; ++n) {}
            if (ok && leader && has_v) {   // O += P V
                const int stage = v_place % kStages;
                product_pv(o_col, s_col, smem_u32(sm.kv[stage]), t0 + i - by < cached_tiles, steps_of(i - by),
                           i - by > first);
                give_back(stage);
                if (!has_k) mma_commit(&sm.o_full[stream]);
            }
            __syncwarp();
            if (narrow && has_k) {
                landed(k_place);
                fence_after();
            }
            if (ok && leader && has_k) {   // S = Q K^T
                const int stage = k_place % kStages;
                product_qk(s_col, smem_u32(sm.q[q]), smem_u32(sm.kv[stage]), t0 + i < cached_tiles,
                           mma_form(16 * steps_of(i), false, negate));
                mma_commit(&sm.s_full[stream]);
                give_back(stage);
                if (i + by >= tiles) mma_commit(&sm.q_empty);
            }
            if (ok && leader && !narrow) atomicExch_block(&sm.issuing, 0);
            __syncwarp();
        }
        base += tiles;
    }
    // Nothing of the tensor cores' is left behind.
    if (elected()) mma_commit(&sm.drained[stream]);
    __syncwarp();
    const unsigned long long t0 = global_ns();
    while (!mbar_try(&sm.drained[stream], 0) && global_ns() - t0 < kWaitLimitNs) {}
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
    template <int kN>
    __device__ __forceinline__ void add(const uint32_t (&x)[kN]) {
#pragma unroll
        for (int i = 0; i < kN; i += 2)
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
    for (int i = 0; i < kHeadDim; i += 16) {
        uint32_t o[16];
        tmem_load(o, o_addr + i);
        tmem_wait(o);
#pragma unroll
        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * c);
        tmem_store(o_addr + i, o);
    }
}

// Weights ex2(x * scale - ref) of scores, in bf16 to tensor memory; their sums (of the unrounded
// ones) are added to `sum`.
template <int kN>
__device__ __forceinline__ void put_weights(const uint32_t (&x)[kN], uint64_t scale, uint64_t ref, uint32_t p_addr,
                                            uint64_t (&sum)[4]) {
    uint32_t p[kN / 2];
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) {
        const float2 e = halves(fma2(pair_of(x[2 * i], x[2 * i + 1]), scale, ref));
        const float y0 = ex2(e.x), y1 = ex2(e.y);
        sum[i % 4] = add2(sum[i % 4], pair_of(__float_as_uint(y0), __float_as_uint(y1)));
        p[i] = pack_bf16(y0, y1);
    }
    tmem_store(p_addr, p);
}

// Scores of which the row sees those in `sees`; the others become -infinity, weight 0.
__device__ __forceinline__ void hide(uint32_t (&x)[16], uint32_t sees) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (!(sees >> i & 1)) x[i] = 0xFF800000u;
}

// This warp is done with tensor memory and what it has written up to here.
__device__ __forceinline__ void warp_done(uint64_t *bar) {
    fence_before();
    __syncwarp();
    if (threadIdx.x % 32 == 0) mbar_arrive(bar);
}

// A key tile's weights of this thread's row: S from tensor memory, P back over it (8 columns
// of P for 16 of S, so a chunk's weights never reach scores that are still to be read).
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
        // 16 at a time: such tiles are an item's last, and short code that is run once or twice a call
        // comes from the instruction caches sooner than its results from the arithmetic.
        const uint64_t bits = own && a.masks ? mask : ~0ull;   // drafts are at most 64 keys
        const int chunks = (keys + 15) / 16;
        auto sees = [&](int c) {
            const int n = seen - c * 16;
            return (n >= 16 ? ~0u : n > 0 ? (1u << n) - 1 : 0u) & (c < 4 ? static_cast<uint32_t>(bits >> (c * 16)) : ~0u);
        };
#pragma unroll 1
        for (int c = 0; c < chunks; ++c) {
            uint32_t x[16];
            tmem_load(x, s_addr + c * 16);
            tmem_wait(x);
            hide(x, sees(c));
            top.add(x);
        }
        move_top(top.all() * a.scale_log2, o_addr, first, st);
        const uint32_t minus = __float_as_uint(st.m == -INFINITY ? 0.f : -st.m);
        const uint64_t ref = pair_of(minus, minus);
#pragma unroll 1
        for (int c = 0; c < chunks; ++c) {
            uint32_t x[16];
            tmem_load(x, s_addr + c * 16);
            tmem_wait(x);
            hide(x, sees(c));
            put_weights(x, scale, ref, s_addr + c * 8, sum);
        }
    }
    const float2 y = halves(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])));
    st.l += y.x + y.y;
}

// A slot of partial results: 256 rows of 128 values; behind all slots, (m, l) of the rows. CTA c has slot 2c
// for an item that an earlier piece begins, and 2c + 1 for one that it begins and a later piece ends.
__device__ __forceinline__ float *part_o(const TurnArgs &a, int slot, int stream) {
    return a.part + (static_cast<int64_t>(slot) * 2 + stream) * kTurnRows * kHeadDim;
}
__device__ __forceinline__ float2 *part_ml(const TurnArgs &a, int slot, int stream) {
    return reinterpret_cast<float2 *>(a.part + static_cast<int64_t>(a.part_slots) * 2 * kTurnRows * kHeadDim) +
           (static_cast<int64_t>(slot) * 2 + stream) * kTurnRows;
}
// What a CTA tells the merge: the item that it begins and does not end, and whether an item passes
// through its piece.
struct PartRecord {
    int32_t opens, through;
    int32_t row;      // first row (token) of the item
    int32_t tokens, g;
};
__device__ __forceinline__ PartRecord *part_record(const TurnArgs &a, int cta) {
    return reinterpret_cast<PartRecord *>(a.part + static_cast<int64_t>(a.part_slots) * 2 * kTurnRows * (kHeadDim + 2)) +
           cta;
}

// Words w[g] of four lanes, of 16-byte units g = 0 .. 3 that the lanes hold a word each of: lane q of the
// four gets unit q whole.
__device__ __forceinline__ uint4 units_of(const uint32_t (&w)[4], int lane) {
    const bool odd = lane & 1, high = lane & 2;
    const uint32_t t0 = __shfl_xor_sync(~0u, odd ? w[0] : w[1], 1), t1 = __shfl_xor_sync(~0u, odd ? w[2] : w[3], 1);
    const uint32_t c0 = odd ? t0 : w[0], c1 = odd ? w[1] : t0, c2 = odd ? t1 : w[2], c3 = odd ? w[3] : t1;
    const uint32_t s0 = __shfl_xor_sync(~0u, high ? c0 : c2, 2), s1 = __shfl_xor_sync(~0u, high ? c1 : c3, 2);
    return high ? make_uint4(s0, s1, c2, c3) : make_uint4(c0, c1, s0, s1);
}

// The new tokens' K and V into their slots of the pool, by one warp beside the others' work, a token's
// K and V rows of the item's kv-head at a time: each item's once, by the piece that has its last key tile.
__device__ void store_role(const TurnArgs &a, Smem &sm, int lane) {
    const Shape &sh = a.s;
    const TurnShape s = turn_shape(a);
    const int kv = lane >> 4, c = lane & 15, bt_shift = sh.bt == 64 ? 6 : 4;
    Reader reader;
    Run r;
#pragma unroll 1
    for (; reader.next(sm, r); reader.done(sm)) {
        if (a.masks || r.t1 != r.tiles) continue;
        const int i0 = r.pair << (s.shift + 1), i1 = min(i0 + (2 << s.shift), r.n);
        const uint16_t *src = (kv ? a.v_new : a.k_new) + r.lo * a.kv_stride + r.g * kHeadDim + c * 8;
        const int32_t *table = a.tables + static_cast<int64_t>(r.b) * a.max_blocks;
        constexpr int kAhead = 4;
#pragma unroll 1
        for (int i = i0; i < i1; i += kAhead) {
            uint4 x[kAhead];
            int blk[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (i + k < i1) {
                    blk[k] = table[(r.P + i + k) >> bt_shift];
                    x[k] = *reinterpret_cast<const uint4 *>(src + (i + k) * a.kv_stride);
                }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (i + k >= i1) break;
                if (blk[k] < 0 || blk[k] >= sh.num_blocks) {
                    if (lane == 0) atomicOr(a.err, kErrBadBlock);
                    continue;
                }
                const int row = (((blk[k] * sh.L + a.layer) * 2 + kv) * sh.Hkv + r.g) * sh.bt +
                                ((r.P + i + k) & (sh.bt - 1));
                reinterpret_cast<uint4 *>(a.hot + static_cast<int64_t>(row) * kHeadDim)[c] = x[k];
            }
        }
    }
}

__device__ void softmax_role(const TurnArgs &a, Smem &sm, int stream) {
    const TurnShape s = turn_shape(a);
    const int g_shift = 7 - s.shift;                          // a token has 128 / tokens rows
    const int row = threadIdx.x & (kTurnRows - 1);
    const uint32_t lanes = static_cast<uint32_t>(row & ~31) << 16;   // a warp has 32 lanes of tensor memory
    const uint32_t tmem = sm.tmem + lanes;
    const uint32_t s_addr = tmem + kColS + stream * kColStream, o_addr = tmem + kColO + stream * kColStream;
    uint32_t s_phase = 0, o_phase = 0, other_phase = 0;
    bool ok = true;   // the same in a warp's lanes
    auto wait = [&](uint64_t *bar, uint32_t &phase) {
        ok = __all_sync(~0u, ok && mbar_wait(sm, bar, phase));
        phase ^= 1;
        fence_after();
    };
    PartRecord rec = {0, 0, 0, 0, 0};
    Reader reader;
    Run r;
#pragma unroll 1
    for (; ok && reader.next(sm, r); reader.done(sm)) {
        const int tile = r.narrow ? 2 * r.pair : 2 * r.pair + stream;
        const int token = (tile << s.shift) + (row >> g_shift);   // of the session's new ones
        const bool live = token < r.n;
        uint64_t mask = 0;
        if (a.masks && live) mask = a.masks[r.lo + token];
        Stats st = {-INFINITY, 0.f};
        const int step = r.narrow ? 2 : 1;
        const int t_first = r.narrow ? r.t0 + stream : r.t0;
        for (int t = t_first; ok && t < r.t1; t += step) {
            wait(&sm.s_full[stream], s_phase);
            if (!ok) break;
            softmax_tile(a, r, t, token, mask, s_addr, o_addr, t == t_first, st);
            tmem_stored();
            warp_done(&sm.p_full[stream]);
        }
        if (ok && t_first < r.t1) wait(&sm.o_full[stream], o_phase);
        // A narrow item: stream 0 takes both streams' results together.
        float w = 1.f, w_other = 0.f;
        uint32_t other = 0;
        if (r.narrow) {
            if (stream == 1) {
                sm.other_m[row] = st.m;
                sm.other_l[row] = st.l;
                warp_done(&sm.other_ready);
                wait(&sm.other_free, other_phase);   // before the next product into this O
                continue;
            }
            wait(&sm.other_ready, other_phase);
            if (r.t1 - r.t0 > 1) {
                const float m1 = sm.other_m[row], l1 = sm.other_l[row], m = fmaxf(st.m, m1);
                const float ref = m == -INFINITY ? 0.f : m;
                w = ex2(st.m - ref);
                w_other = ex2(m1 - ref);
                st.l = st.l * w + l1 * w_other;
                st.m = m;
                other = tmem + kColO + kColStream;
            }
        }
        {
            const bool whole = r.t0 == 0 && r.t1 == r.tiles;
            const int slot = r.t0 > 0 ? 2 * blockIdx.x : 2 * blockIdx.x + 1;
            if (whole) {
                const float inv = st.l > 0.f || st.l != st.l ? __frcp_rn(st.l) : 0.f;   // nothing seen: zeros
                w *= inv;
                w_other *= inv;
            } else {
                if (live) part_ml(a, slot, stream)[row] = make_float2(st.m, st.l);
                if (stream == 0 && row == 0) {
                    const int t0 = r.pair << (s.shift + 1);
                    if (r.t0 == 0) rec = {1, 0, r.lo + t0, min(2 << s.shift, r.n - t0), r.g};
                    else if (r.t1 < r.tiles) rec.through = 1;
                }
            }
            // The rows from tensor memory, 16 rows by 32 columns at a time, so that a store has the 64 or
            // 32 bytes of eight rows; with a row per thread each store had 16 bytes of 32 rows, and an
            // item's end took twice as long. Short code, as above.
            const int lane = row & 31;
            const uint32_t some = __ballot_sync(~0u, live);
            const bool bf16 = whole && a.out_bf16;
#pragma unroll 1
            for (int half = 0; half < 32; half += 16) {
                if (!ok || !(some >> half & 0xFFFFu)) continue;
                // This thread's rows, lane / 4 and 8 on: factors, and where their values go.
                float scale[2], scale_other[2];
                bool there[2];
                uint8_t *to[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int from = half + i * 8 + (lane >> 2), its = (row & ~31) + from;
                    const int t = (tile << s.shift) + (its >> g_shift);
                    const int64_t o_row = (static_cast<int64_t>(r.lo) + t) * a.s.Hq + (r.g << g_shift) +
                                          (its & ((1 << g_shift) - 1));
                    scale[i] = __shfl_sync(~0u, w, from);
                    scale_other[i] = __shfl_sync(~0u, w_other, from);
                    there[i] = t < r.n;
                    to[i] = bf16    ? static_cast<uint8_t *>(a.out) + o_row * kRowBytes + (lane & 3) * 16
                            : whole ? static_cast<uint8_t *>(a.out) + o_row * (2 * kRowBytes) + (lane & 3) * 8
                                    : reinterpret_cast<uint8_t *>(part_o(a, slot, stream) + its * kHeadDim) + (lane & 3) * 8;
                }
#pragma unroll 1
                for (int d = 0; d < kHeadDim; d += 32) {
                    uint32_t x[16];
                    float y[16];
                    tmem_load_rows(x, o_addr + (half << 16) + d);
                    tmem_wait(x);
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = __uint_as_float(x[i]) * scale[i >> 1 & 1];
                    if (other) {
                        tmem_load_rows(x, other + (half << 16) + d);
                        tmem_wait(x);
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = __fmaf_rn(__uint_as_float(x[i]), scale_other[i >> 1 & 1], y[i]);
                    }
                    if (bf16) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t v[4];
#pragma unroll
                            for (int g = 0; g < 4; ++g) v[g] = pack_bf16(y[4 * g + 2 * i], y[4 * g + 2 * i + 1]);
                            const uint4 unit = units_of(v, lane);
                            if (there[i]) *reinterpret_cast<uint4 *>(to[i] + d * 2) = unit;
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int g = 0; g < 4; ++g)
                                if (there[i])
                                    *reinterpret_cast<float2 *>(to[i] + d * 4 + g * 32) =
                                        make_float2(y[4 * g + 2 * i], y[4 * g + 2 * i + 1]);
                    }
                    __syncwarp();
                }
            }
        }
        fence_before();
        if (r.narrow) warp_done(&sm.other_free);
    }
    if (!a.whole && stream == 0 && row == 0) *part_record(a, blockIdx.x) = rec;
}

__global__ void __launch_bounds__(kThreads, 1) turn_kernel(const __grid_constant__ TurnArgs a,
                                                           const __grid_constant__ Maps maps) {
    extern __shared__ uint8_t raw[];
    if (!a.whole) asm volatile("griddepcontrol.launch_dependents;");   // the merge, which waits for all of this
    Smem &sm = *reinterpret_cast<Smem *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp == kStoreWarp && lane < sizeof(Maps) / sizeof(CUtensorMap))
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<const CUtensorMap *>(&maps) + lane) : "memory");
    if (threadIdx.x == 32) {   // a warp that has nothing else to do yet
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sm.kv_full[i], 1);
            mbar_init(&sm.kv_full[i + kStages], 1);
            mbar_init(&sm.kv_empty[i], 2);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sm.q_full[s], 1);
            mbar_init(&sm.s_full[s], 1);
            mbar_init(&sm.p_full[s], kTurnRows / 32);
            mbar_init(&sm.o_full[s], 1);
            mbar_init(&sm.drained[s], 1);
        }
        for (int i = 0; i < kRuns; ++i) {
            mbar_init(&sm.run_full[i], 1);
            mbar_init(&sm.run_empty[i], kRunReaders);
        }
        mbar_init(&sm.other_ready, kTurnRows / 32);
        mbar_init(&sm.other_free, kTurnRows / 32);
        mbar_init(&sm.q_empty, 2);
        sm.abort = 0;
        sm.issuing = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kCopyWarp) {
        if (!a.many) make_plan<int32_t, false>(a, sm.plan, lane);
        else if (a.small) make_plan<int32_t, true>(a, sm.plan, lane);
        else make_plan<int64_t, true>(a, sm.plan, lane);
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
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
        softmax_role(a, sm, warp >> 2);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
        if (warp == kCopyWarp) copy_role(a, maps, sm, lane);
        else if (warp < kMmaWarp + 2) mma_role(a, sm, warp - kMmaWarp);
        else store_role(a, sm, lane);
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    fence_after();
    if (threadIdx.x == 0 && sm.abort) atomicOr(a.err, kErrTimeout);
    if (warp == kMmaWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sm.tmem), "r"(kTmemCols));
}

// The pieces of each item that several have, merged in order: a warp for up to four of its rows, 64 apart,
// a lane for four values of each. CTA (c, j): the item that piece c begins, if any. Loads are what takes
// the time: the statistics of up to 32 pieces come in one round, a lane each, and the values 16 at a time.
constexpr int kCombineCtas = 8, kCombineWarps = 8;
constexpr int kCombineRows = 2 * kTurnRows / (kCombineCtas * kCombineWarps);
__global__ void __launch_bounds__(kCombineWarps * 32) turn_combine_kernel(const __grid_constant__ TurnArgs a) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int first = blockIdx.x, lane = threadIdx.x & 31, g_shift = 7 - a.token_shift, ctas = a.part_slots / 2;
    const int row0 = blockIdx.y * kCombineWarps + (threadIdx.x >> 5);
    const auto slot = [&](int c) { return c == first ? 2 * c + 1 : 2 * c; };
    constexpr int kApart = kCombineCtas * kCombineWarps;
    const auto stream_of = [&](int i) { return (row0 + i * kApart) / kTurnRows; };
    const auto row_of = [&](int i) { return (row0 + i * kApart) % kTurnRows; };
    // The record, the ends of up to 32 pieces and the rows' statistics in them (if they are the item's) in one
    // round; a slot that no piece has written is not used.
    const PartRecord rec = *part_record(a, first);
    bool ends = first + 1 + lane >= ctas || !part_record(a, first + 1 + lane)->through;
    float2 stats[kCombineRows];
#pragma unroll
    for (int i = 0; i < kCombineRows; ++i)
        stats[i] = part_ml(a, slot(min(first + lane, ctas - 1)), stream_of(i))[row_of(i)];
    if (!rec.opens) return;
    const int rows = rec.tokens << g_shift;
    if (row0 >= rows) return;
    int last = first + 1;   // the first piece that the item does not pass through
    for (;;) {
        const uint32_t any = __ballot_sync(~0u, ends);
        if (any) {
            last += __ffs(any) - 1;
            break;
        }
        last += 32;
        ends = last + lane >= ctas || !part_record(a, last + lane)->through;
    }
    float m[kCombineRows], l[kCombineRows];
    float4 y[kCombineRows];
#pragma unroll
    for (int i = 0; i < kCombineRows; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
        y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int c0 = first; c0 <= last; c0 += 32) {
        const int n = min(32, last + 1 - c0);
        float weight[kCombineRows];
#pragma unroll
        for (int i = 0; i < kCombineRows; ++i) {
            float2 v = make_float2(-INFINITY, 0.f);
            if (lane < n && row0 + i * kApart < rows)
                v = c0 == first ? stats[i] : part_ml(a, slot(c0 + lane), stream_of(i))[row_of(i)];
            float top = v.x;
#pragma unroll
            for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
            top = fmaxf(top, m[i]);
            const float ref = top == -INFINITY ? 0.f : top, c = ex2(m[i] - ref);   // of the pieces before
            weight[i] = ex2(v.x - ref);
            float sum = weight[i] * v.y;
#pragma unroll
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
            m[i] = top;
            l[i] = __fmaf_rn(l[i], c, sum);
            y[i] = make_float4(y[i].x * c, y[i].y * c, y[i].z * c, y[i].w * c);
        }
#pragma unroll 4
        for (int k = 0; k < n; ++k)
#pragma unroll
            for (int i = 0; i < kCombineRows; ++i) {
                const float w = __shfl_sync(~0u, weight[i], k);
                if (row0 + i * kApart >= rows) continue;
                const float4 x = reinterpret_cast<const float4 *>(part_o(a, slot(c0 + k), stream_of(i)) +
                                                                  row_of(i) * kHeadDim)[lane];
                y[i] = make_float4(__fmaf_rn(w, x.x, y[i].x), __fmaf_rn(w, x.y, y[i].y), __fmaf_rn(w, x.z, y[i].z),
                                   __fmaf_rn(w, x.w, y[i].w));
            }
    }
#pragma unroll
    for (int i = 0; i < kCombineRows; ++i) {
        const int row = row0 + i * kApart;
        if (row >= rows) break;
        const float inv = l[i] > 0.f || l[i] != l[i] ? __frcp_rn(l[i]) : 0.f;   // nothing seen: zeros
        const int64_t to = ((static_cast<int64_t>(rec.row) + (row >> g_shift)) * a.s.Hq + (rec.g << g_shift) +
                            (row & ((1 << g_shift) - 1))) * kHeadDim;
        const float4 z = make_float4(y[i].x * inv, y[i].y * inv, y[i].z * inv, y[i].w * inv);
        if (a.out_bf16)
            reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + to)[lane] =
                make_uint2(pack_bf16(z.x, z.y), pack_bf16(z.z, z.w));
        else
            reinterpret_cast<float4 *>(static_cast<float *>(a.out) + to)[lane] = z;
    }
}

}  // namespace

// Floats that launches of up to `ctas` CTAs need for partial results.
int64_t turn_part_floats(int ctas) {
    static_assert(sizeof(PartRecord) % sizeof(float) == 0, "records follow the rows");
    return int64_t(2) * ctas * 2 * kTurnRows * (kHeadDim + 2) + ctas * int64_t(sizeof(PartRecord) / sizeof(float));
}

bool encode_turn_hot_maps(CUtensorMap maps[2], void *hot_base, int64_t rows, int bt, const char **why) {
    // [eight rows][half][row of eight][64 columns]; a block's rows start at a multiple of 16
    const cuuint64_t dims[4] = {64, 8, 2, static_cast<cuuint64_t>(rows / 8)};
    const cuuint64_t strides[3] = {kRowBytes, 128, 8 * kRowBytes};
    const cuuint32_t part[4] = {64, 8, 2, kBoxRows / 8}, block[4] = {64, 8, 2, static_cast<cuuint32_t>(bt / 8)};
    return encode_bf16_map(&maps[0], hot_base, 4, dims, strides, part, why) &&
           encode_bf16_map(&maps[1], hot_base, 4, dims, strides, block, why);
}

cudaError_t launch_turn(TurnArgs a, const CUtensorMap hot[2], cudaStream_t st) {
    if (a.total < 1) return cudaSuccess;
    const int G = a.s.Hq / a.s.Hkv;
    Maps maps;
    maps.hot = hot[0];
    maps.hot_block = hot[1];
    const cuuint64_t n = static_cast<cuuint64_t>(a.total), hkv = static_cast<cuuint64_t>(a.s.Hkv);
    const cuuint64_t q_step = static_cast<cuuint64_t>(a.q_stride) * 2, kv_step = static_cast<cuuint64_t>(a.kv_stride) * 2;
    const char *why = nullptr;
    auto encode = [&](CUtensorMap *map, const uint16_t *base, const cuuint64_t (&dims)[4], const cuuint64_t (&strides)[3],
                      const cuuint32_t (&box)[4]) {
        return encode_bf16_map(map, const_cast<uint16_t *>(base), 4, dims, strides, box, &why);
    };
    // [half][token][head][64 columns], and for whole tiles [head][half][token][64 columns]
    const cuuint32_t per_tile = static_cast<cuuint32_t>(kTurnRows / G);
    bool ok = encode(&maps.q, a.q, {64, static_cast<cuuint64_t>(a.s.Hq), n, 2}, {kRowBytes, q_step, 128},
                     {64, static_cast<cuuint32_t>(G), per_tile, 2});
    for (int kv = 0; ok && kv < 2; ++kv) {
        const uint16_t *base = kv ? a.v_new : a.k_new;
        ok = encode(kv ? &maps.v : &maps.k, base, {64, hkv, n, 2}, {kRowBytes, kv_step, 128}, {64, 1, kBoxRows, 1}) &&
             encode(kv ? &maps.v_whole : &maps.k_whole, base, {64, n, 2, hkv}, {kv_step, 128, kRowBytes},
                    {64, kTurnKeys, 2, 1});
    }
    if (!ok) return cudaErrorInvalidValue;
    // The scores' sign goes into the product, so that the largest score is the largest scaled one; a
    // scale of 0 (all weights equal) stays a positive one, which masked scores keep apart.
    a.negate = a.scale_log2 < 0.f;
    a.scale_log2 = fmaxf(fabsf(a.scale_log2), 1e-30f);
    a.token_shift = G == 8 ? 4 : G == 4 ? 5 : G == 2 ? 6 : 7;
    // No more CTAs than there can be pieces.
    const int64_t longest = a.longest = turn_longest(a.max_blocks, a.s.bt);
    const int64_t bound = turn_cost_bound(turn_shape(a), a.total, a.B, longest);
    const unsigned ctas = static_cast<unsigned>(
        std::max<int64_t>(1, std::min<int64_t>(bound / kCostsFew.piece, a.part_slots / 2)));
    a.many = turn_many(bound, a.part_slots / 2);
    a.small = turn_cost_bound(turn_shape(a, true), a.total, a.B, longest) < int64_t(1) << 30;
    a.part_slots = 2 * ctas;
    a.whole = !turn_cuts(longest);
    turn_kernel<<<ctas, kThreads, kSmemBytes, st>>>(a, maps);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || a.whole) return e;
    cudaLaunchAttribute early[1];
    early[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas, kCombineCtas);
    cfg.blockDim = dim3(256);
    cfg.stream = st;
    cfg.attrs = early;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, turn_combine_kernel, a);
}

cudaError_t prepare_turn_kernel() {
    // The warps' register shares presume the launch's.
    cudaFuncAttributes f;
    cudaError_t e = cudaFuncGetAttributes(&f, turn_kernel);
    if (e == cudaSuccess && f.numRegs != kRegsLaunch) e = cudaErrorInvalidConfiguration;
    if (e != cudaSuccess || f.maxDynamicSharedSizeBytes >= kSmemBytes) return e;
    return cudaFuncSetAttribute(turn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
}

}  // namespace kvt
