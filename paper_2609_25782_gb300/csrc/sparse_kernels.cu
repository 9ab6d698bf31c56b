// Kernels that choose the part of the cache that a step reads, for sm_103a.
//
//   bounds_kernel   channelwise bounds of the keys of blocks, in 8 bits
//   select_kernel   scores of blocks from the bounds, and the `top` largest
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cache_ops.h"
#include "cluster.cuh"
#include "tile_ops.cuh"

namespace kvt {
namespace {

// ---- bounds ------------------------------------------------------------------------------------------

__device__ __forceinline__ float pow2(int biased) {   // 2^(biased - 127), biased in [-22, 254]
    return __int_as_float(biased >= 1 ? biased << 23 : 1 << (biased + 22));
}

constexpr uint32_t kInfBits = 0x7F80;

// A row's length that its table holds, and whose last block's end is still an int.
__device__ __forceinline__ bool good_length(int T, int max_blocks, int bt) {
    return T >= 0 && T <= INT32_MAX - 512 && T <= static_cast<int64_t>(max_blocks) * bt;
}

// Blocks of a row that a call does: [first, end) of its logical blocks; none where its length is bad.
__device__ __forceinline__ int2 bounds_blocks(const BoundsArgs &a, int b) {
    const int T = a.seq_lens[b];
    const int from = a.since ? a.since[b] : 0;
    if (!good_length(T, a.max_blocks, a.s.bt) || from < 0 || from > T) return make_int2(-1, -1);
    if (from >= T) return make_int2(0, 0);
    return make_int2(from / a.s.bt, (T + a.s.bt - 1) / a.s.bt);
}

__device__ __forceinline__ uint32_t max2(uint32_t x, uint32_t y) {   // of two bf16 each; a NaN stays
    const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&m);
}
__device__ __forceinline__ uint32_t min2(uint32_t x, uint32_t y) {
    const __nv_bfloat162 m = __hmin2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&m);
}

constexpr int kBoundsThreads = 256;
// CTAs per SM, each warp with 4 KiB on its way. us by 2, 3, 4, 5 and 6 of them, 48 layers, three sessions of 8K to 24K
// tokens: 287, 285, 312, 530, 852 (of 64-token blocks 262, 263, 279, 352, 512); one of 2 100 22.6, 21.9, 23.1, 34.9, 54.5.
constexpr int kBoundsPerSm = 3;
constexpr uint32_t kNegate2 = 0x80008000u, kMinusInf2 = 0xFF80FF80u;

// A warp per (block, layer, kv-head) in turn: the rows' block counts are summed up by every CTA first, so that the
// items are one line whatever the lengths. 16 tokens at a time; the next ones are on their way while an item's codes
// are made, and the item after that is looked up. Warps next to each other have items next to each other: in runs of
// items, each warp at another block of 1.5 MiB, the call took 1.1 times as long. Bound by HBM: 6.6 TB/s over three
// sessions of 8K to 24K tokens.
__global__ void __launch_bounds__(kBoundsThreads, kBoundsPerSm) bounds_kernel(const BoundsArgs a) {
    extern __shared__ int rows_smem[];               // [B] ends: items' blocks up to the row's; [B] its first block less those before
    __shared__ int sums[kBoundsThreads / 32];
    int *ends = rows_smem, *shift = rows_smem + a.B;
    const Shape sh = a.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    after_previous();
    int total = 0;
    for (int b0 = 0; b0 < a.B; b0 += kBoundsThreads) {
        const int b = b0 + threadIdx.x;
        int n = 0, from = 0;
        if (b < a.B) {
            const int2 r = bounds_blocks(a, b);
            n = r.y - r.x;
            from = r.x;
            if (r.x < 0 && blockIdx.x == 0) atomicOr(a.err, kErrBadLength);
        }
        const int mine = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(~0u, n, d);
            if (lane >= d) n += y;
        }
        if (lane == 31) sums[warp] = n;
        __syncthreads();
        int before = total;
        for (int w = 0; w < kBoundsThreads / 32; ++w) {
            if (w < warp) before += sums[w];
            total += sums[w];
        }
        if (b < a.B) {
            ends[b] = before + n;
            shift[b] = from - (before + n - mine);
        }
        __syncthreads();
    }
    // The warp's items are `warps` apart: blocks, layers and heads advance by these.
    const int per = a.nlayers * sh.Hkv, warps = gridDim.x * (kBoundsThreads / 32);
    const int dpair = warps / per, dl = (warps - dpair * per) / sh.Hkv, dg = warps - dpair * per - dl * sh.Hkv;
    const int first = blockIdx.x * (kBoundsThreads / 32) + warp;
    int pair = first / per, l = (first - pair * per) / sh.Hkv, g = first - pair * per - l * sh.Hkv;
    int row = 0;
    // An item: its records' and its keys' places, its block (-1: a bad id) and tokens.
    struct Item {
        int l, g, blk, tokens;
    };
    auto find = [&]() {                              // of `pair`, below `total`
        while (ends[row] <= pair) ++row;
        const int j = pair + shift[row];
        return Item{l, g, a.tables[static_cast<int64_t>(row) * a.max_blocks + j], min(sh.bt, a.seq_lens[row] - j * sh.bt)};
    };
    auto advance = [&]() {                           // (2^30 blocks at most, and a step of at most 2^13: in int)
        pair += dpair;
        l += dl;
        g += dg;
        if (g >= sh.Hkv) {
            g -= sh.Hkv;
            ++l;
        }
        if (l >= a.nlayers) {
            l -= a.nlayers;
            ++pair;
        }
    };
    // Half a warp per token, eight channels a lane. Past the end the last token again.
    uint4 v[8];
    auto load = [&](const Item &x, int t0) {
        if (x.blk < 0 || x.blk >= sh.num_blocks) return;
        const int64_t at = ((static_cast<int64_t>(x.blk) * sh.L + a.layer0 + x.l) * 2 * sh.Hkv + x.g) * sh.bt + t0;
        const uint4 *k = reinterpret_cast<const uint4 *>(a.hot + at * kHeadDim) + (lane & 15);
        const int half = lane >> 4, last = x.tokens - t0 - 1;
        if (last >= 15) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k[(2 * i + half) * 16];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = k[min(2 * i + half, last) * 16];
        }
    };
    if (pair >= total) return;
    Item now = find();
    load(now, 0);
    advance();
    Item next{};
    bool more = pair < total;
    if (more) next = find();
    int t0 = 0;
    uint32_t up[4], down[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        up[c] = kMinusInf2;
        down[c] = kMinusInf2 ^ kNegate2;
    }
#pragma unroll 1
    for (;;) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                up[c] = max2(up[c], w[c]);
                down[c] = min2(down[c], w[c]);
            }
        }
        t0 += 16;
        if (t0 < now.tokens) {
            load(now, t0);
            continue;
        }
        t0 = 0;
        const Item done = now;
        const bool go = more;
        if (go) {
            load(next, 0);
            now = next;
            advance();
            more = pair < total;
            if (more) next = find();
        }
        // Lanes 0-15 get their channels' largest values, the others the smallest negated.
        const bool high = lane < 16;
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t low = down[c] ^ kNegate2;
            const uint32_t got = __shfl_xor_sync(~0u, high ? low : up[c], 16);
            up[c] = max2(high ? up[c] : low, got);
            top = max(top, max(up[c] & 0x7FFFu, up[c] >> 16 & 0x7FFFu));
        }
        top = __reduce_max_sync(~0u, top);
        const bool fine = top < kInfBits;
        const int E = max(1, static_cast<int>(top >> 7)) + ((top & 0x7F) == 0x7F);
        if (done.blk >= 0 && done.blk < sh.num_blocks) {
            // 2^(133 - E) is up to 2^132: two factors where E is below 6, which no real key's is. A value too small for
            // the product still counts: it rounds outwards.
            const float scale = pow2(min(254, 260 - E)), rest = E < 6 ? pow2(133 - E) : 1.f;
            uint32_t out[2];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float x0 = __uint_as_float(up[c] << 16), x1 = __uint_as_float(up[c] & 0xFFFF0000u);
                if (E < 6) {
                    x0 *= rest;
                    x1 *= rest;
                }
                int y0 = max(__float2int_ru(x0 * scale), x0 > 0.f ? 1 : -127);
                int y1 = max(__float2int_ru(x1 * scale), x1 > 0.f ? 1 : -127);
                if (!fine) y0 = y1 = 127;
                if (!high) {
                    y0 = -y0;
                    y1 = -y1;
                }
                const uint32_t two = __byte_perm(static_cast<uint32_t>(y0), static_cast<uint32_t>(y1), 0x0040);
                out[c >> 1] = c & 1 ? __byte_perm(out[c >> 1], two, 0x5410) : two;
            }
            const int64_t rec = (static_cast<int64_t>(a.layer0 + done.l) * sh.Hkv + done.g) * sh.num_blocks + done.blk;
            reinterpret_cast<uint2 *>(a.codes + rec * kCodeRow)[lane] = make_uint2(out[0], out[1]);
            // The step as a bf16: 2^(E - 133), below 2^-126 by its fraction bit.
            if (lane == 0) a.steps[rec] = static_cast<uint16_t>(!fine ? kInfBits : E > 6 ? (E - 6) << 7 : 1u << E);
        } else if (lane == 0) {
            atomicOr(a.err, kErrBadBlock);
        }
        if (!go) break;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            up[c] = kMinusInf2;
            down[c] = kMinusInf2 ^ kNegate2;
        }
    }
}

// ---- selection ---------------------------------------------------------------------------------------

// A row's blocks for one kv-head (a unit) are one cluster's. Each warp scores 16 blocks at a time with whole numbers,
// codes times q's digits, as columns of an fp16 mma (int8 products are slow on this GPU: eight int8 mma of 16 blocks
// took 1 500 cycles, a dp4a loop as long). The scores' keys go to the first CTA's shared memory, which alone finds the
// key of the last block to be taken, by counts of the keys' leading bits within their range, and lists the blocks.
//
// A call of a few units is a chain of latencies and of instructions that run once: they come at some 8 cycles each,
// so the code on the way is kept short, its loops rolled.
constexpr int kSelectThreads = 512;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kBins = 4 * kSelectThreads;
constexpr int kWarpBlocks = 16;                      // that a warp scores at a time
constexpr int kDigits = 3;                           // of a sum over q's heads, in base 32
constexpr int kDigitRow = kCodeRow + 16;             // halves from one digit's row to the next (banks)

constexpr int select_smem(int blocks) { return (blocks + 3) / 4 * 16; }

// Scores in an order of their bits: larger scores have larger keys. NaN-free; no key is 0 or ~0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);   // one zero
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// D = A(16x16 fp16, row) * B(16x8 fp16, col) + D in fp32.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Four codes c as fp16 numbers 1152 + c: 0x6400, which is 1024, and c + 128 in its last bits.
__device__ __forceinline__ uint2 halves(uint32_t codes) {
    const uint32_t u = codes ^ 0x80808080u;
    return make_uint2(__byte_perm(u, 0x64646464u, 0x4140), __byte_perm(u, 0x64646464u, 0x4342));
}
constexpr int kCodeOffset = 1152;

// Sum of the threads' values before this one's. (Two counts in a word's halves: each sums up to at most
// kSelectBlocksMax.) One copy of its code: the second call finds it in the instruction cache.
__device__ __noinline__ uint32_t scan_before(uint32_t x, uint32_t *scratch) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t y = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t z = __shfl_up_sync(~0u, y, d);
        if (lane >= d) y += z;
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = y;
    __syncthreads();
    return y - x + __reduce_add_sync(~0u, lane < warp ? scratch[lane] : 0);
}

// Codes of the warp's 16 blocks, those of block `row` and of `row` + 8 (mma fragments), and a block's step per lane.
struct Fetched {
    uint32_t x[16], y[16];
    uint32_t step;
};

// 32 bytes at once: four lanes then read a whole 128-byte line of a record.
__device__ __forceinline__ void load_32(const int8_t *p, uint32_t *v) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "l"(p)
                 : "memory");
}

// kTwo: CTAs that have an SM each keep two fetches per warp on their way, 128 KiB in all; others one, two CTAs per SM.
template <bool kTwo>
__global__ void __launch_bounds__(kSelectThreads, kTwo ? 1 : 2) select_kernel(const SelectArgs a) {
    extern __shared__ uint4 keys4[];                 // keys of the unit's blocks; used in the first CTA
    uint32_t *keys = reinterpret_cast<uint32_t *>(keys4);
    __shared__ alignas(16) uint32_t hist[kBins];
    __shared__ uint32_t cand[kSelectThreads];
    __shared__ uint32_t scratch[kSelectWarps];
    __shared__ uint32_t least, most, found[4];
    __shared__ int qsum[kCodeRow], qtotal;           // sums of q's positive parts, then of its negative ones
    __shared__ alignas(16) __half digits[kDigits * kDigitRow];
    const Shape sh = a.s;
    const int C = gridDim.x, rank = blockIdx.x, g = blockIdx.y, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    after_previous();
    const int T = a.seq_lens[b];
    // The warp's blocks are j .. j + 15, then those `jump` on; lanes look up their places, the first ones before
    // T is known (entries past a row's end are not used).
    const int32_t *trow = a.tables + static_cast<int64_t>(b) * a.max_blocks;
    const int jump = C * kSelectWarps * kWarpBlocks;
    const int64_t start = a.first + static_cast<int64_t>(rank * kSelectWarps + warp) * kWarpBlocks;
    auto block_of = [&](int64_t at) { return at + (lane & 15) < a.max_blocks ? trow[at + (lane & 15)] : 0; };
    int blk0 = block_of(start), blk1 = kTwo ? block_of(start + jump) : 0;
    // q as one dim of two heads per thread.
    const int dim = tid & (kHeadDim - 1), head = tid / kHeadDim;
    static_assert(kMaxGroup == 2 * kSelectThreads / kHeadDim, "two heads per thread");
    const uint16_t *q = a.q + b * a.q_stride + static_cast<int64_t>(g * a.group + head) * kHeadDim + dim;
    uint32_t v[2];
    v[0] = head < a.group ? q[0] : 0;
    v[1] = head + kMaxGroup / 2 < a.group ? q[kMaxGroup / 2 * kHeadDim] : 0;
    int32_t *selected = a.selected + (static_cast<int64_t>(b) * sh.Hkv + g) * a.top;
    if (!good_length(T, a.max_blocks, sh.bt)) {      // (the whole cluster leaves)
        if (rank == 0) {
            if (tid == 0) atomicOr(a.err, kErrBadLength);
            for (int i = tid; i < a.top; i += kSelectThreads) selected[i] = -1;
        }
        return;
    }
    if (tid == 0) {
        least = ~0u;
        most = 0;
        qtotal = 0;
    }
    if (C > 1) cluster_arrive();                     // the first CTA's memory may be written from here on
    const int n = sh.bt == 16 ? (T + 15) >> 4 : (T + 63) >> 6;
    const int want = min(a.top, n);
    float *scores = a.scores ? a.scores + (static_cast<int64_t>(b) * sh.Hkv + g) * a.max_blocks : nullptr;
    // Blocks [j0, j1) are scored: the others are always taken. Where all are taken, only for the caller's scores.
    const int j0 = min(a.first, n), j1 = max(j0, n - a.last);
    const bool choose = n > a.top;
    const int end = choose || scores ? j1 : 0;
    int j = static_cast<int>(start < end ? start : end);

    const int quad = lane & 3, row = lane >> 2;
    const int8_t *codes = a.codes + static_cast<int64_t>(g) * sh.num_blocks * kCodeRow;
    const uint16_t *steps = a.steps + static_cast<int64_t>(g) * sh.num_blocks;
    auto fetch = [&](Fetched &f, int at, int blk) {
        if (at + (lane & 15) >= end) blk = 0;        // (not scored)
        if (blk < 0 || blk >= sh.num_blocks) {
            atomicOr(a.err, kErrBadBlock);
            blk = 0;
        }
        f.step = steps[blk];
        const int8_t *px = codes + static_cast<int64_t>(__shfl_sync(~0u, blk, row)) * kCodeRow + 32 * quad;
        const int8_t *py = codes + static_cast<int64_t>(__shfl_sync(~0u, blk, row + 8)) * kCodeRow + 32 * quad;
        load_32(px, f.x);
        load_32(py, f.y);
        load_32(px + 128, f.x + 8);
        load_32(py + 128, f.y + 8);
    };
    Fetched f0, f1;
    if (j < end) fetch(f0, j, blk0);
    if (kTwo && j + jump < end) fetch(f1, j + jump, blk1);
    if (j + jump < end) {
        blk0 = block_of(j + (kTwo ? 2 : 1) * static_cast<int64_t>(jump));
        if (kTwo) blk1 = block_of(j + 3 * static_cast<int64_t>(jump));
    }

    // q as whole numbers
    int top_bits = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int m = v[h] & 0x7FFF;
        if (m < static_cast<int>(kInfBits)) top_bits = max(top_bits, m);
    }
    top_bits = __reduce_max_sync(~0u, top_bits);
    if (lane == 0) scratch[warp] = top_bits;
    if (tid < kCodeRow) qsum[tid] = 0;
    if (rank == 0) {
        reinterpret_cast<uint4 *>(hist)[tid] = make_uint4(0u, 0u, 0u, 0u);
        // Blocks that are always taken; what is read behind the last.
        for (int i = tid; i < j0; i += kSelectThreads) keys[i] = ~0u;
        for (int i = j1 + tid; i < ((n + 3) & ~3); i += kSelectThreads) keys[i] = i < n ? ~0u : 0;
    }
    __syncthreads();
    top_bits = __reduce_max_sync(~0u, lane < kSelectWarps ? static_cast<int>(scratch[lane]) : 0);
    const int E = max(1, top_bits >> 7);
    const float s1 = pow2(min(254, 264 - E)), s2 = pow2(127 + max(0, 10 - E));   // 2^(137 - E)
    int up = 0, down = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = (v[h] & 0x7FFF) < kInfBits ? __float2int_rn(__uint_as_float(v[h] << 16) * s1 * s2) : 0;
        up += max(c, 0);
        down += min(c, 0);
    }
    atomicAdd(&qsum[dim], up);
    atomicAdd(&qsum[kHeadDim + dim], down);
    __syncthreads();
    if (tid < kCodeRow) {
        int x = qsum[tid];                           // |x| <= 8 * 2040
        const int total = __reduce_add_sync(~0u, x);
        if (lane == 0) atomicAdd(&qtotal, total);
#pragma unroll
        for (int d = kDigits - 1; d >= 0; --d) {     // digits of -16 .. 15, the first one of -16 .. 16
            const int low5 = d ? ((x + 16) & 31) - 16 : x;
            digits[d * kDigitRow + tid] = __int2half_rn(low5);
            x = (x - low5) >> 5;
        }
    }
    __syncthreads();
    // B fragments: columns 0 to 2 are the digits, the others any. The order of the dims within a product is the
    // loads': piece c of lane t (of four) is the record's 32 bytes t + 4 c.
    const uint4 *weights = reinterpret_cast<const uint4 *>(digits + min(row, kDigits - 1) * kDigitRow) + 4 * quad;
    const uint32_t offset = static_cast<uint32_t>(kCodeOffset * qtotal);
    if (C > 1) cluster_wait();
    const uint32_t keys_at = remote(smem_u32(keys), 0);
    uint32_t low = ~0u, high = 0;
    auto score = [&](const Fetched &f, int at) {
        // 64 products of up to 1279 x 16 a sum: whole numbers below 2^24, exact in fp32.
        float d[4][4] = {};
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 w = weights[16 * c + i];
                uint2 p = halves(f.x[8 * c + 2 * i]), o = halves(f.y[8 * c + 2 * i]);
                mma_f16(d[2 * (i & 1)], p.x, o.x, p.y, o.y, w.x, w.y);
                p = halves(f.x[8 * c + 2 * i + 1]), o = halves(f.y[8 * c + 2 * i + 1]);
                mma_f16(d[2 * (i & 1) + 1], p.x, o.x, p.y, o.y, w.z, w.w);
            }
        auto whole = [&](int i) { return static_cast<uint32_t>(__float2int_rn((d[0][i] + d[1][i]) + (d[2][i] + d[3][i]))); };
        // Lanes of quad 0 have the first two digits' sums, of quad 1 the last one's, each for blocks row and row + 8:
        // quad 0 keeps row. (Whole numbers modulo 2^32; the score's fits 32 bits.)
        uint32_t mine = whole(0), other = whole(2);
        if (quad == 0) {
            mine = mine * 1024 + whole(1) * 32;
            other = other * 1024 + whole(3) * 32;
        }
        const uint32_t got = __shfl_xor_sync(~0u, quad == 0 ? other : mine, 1);
        const int sum = static_cast<int>((quad == 0 ? mine : other) + got - offset);
        const int r = row + 8 * quad;
        const uint32_t st = __shfl_sync(~0u, f.step, r & 15);
        const float z = st < kInfBits ? __fmul_rn(__int2float_rn(sum), __uint_as_float(st << 16)) : INFINITY;
        if (quad < 2 && at + r < end) {
            const uint32_t key = key_of(z);
            low = min(low, key);
            high = max(high, key);
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(keys_at + (at + r) * 4), "r"(key) : "memory");
            if (scores) scores[at + r] = z;
        }
    };
#pragma unroll 1
    while (j < end) {
        score(f0, j);
        j += jump;
        if (!kTwo) {
            if (j >= end) break;
            fetch(f0, j, blk0);
            blk0 = block_of(j + static_cast<int64_t>(jump));
            continue;
        }
        if (j >= end) break;
        if (j + jump < end) {
            fetch(f0, j + jump, blk0);
            blk0 = block_of(j + 3 * static_cast<int64_t>(jump));
        }
        score(f1, j);
        j += jump;
        if (j + jump < end) {
            fetch(f1, j + jump, blk1);
            blk1 = block_of(j + 3 * static_cast<int64_t>(jump));
        }
    }
    next_may_come();
    low = __reduce_min_sync(~0u, low);
    high = __reduce_max_sync(~0u, high);
    if (lane == 0 && low <= high) {
        asm volatile("red.relaxed.cluster.shared::cluster.min.u32 [%0], %1;" ::"r"(remote(smem_u32(&least), 0)), "r"(low) : "memory");
        asm volatile("red.relaxed.cluster.shared::cluster.max.u32 [%0], %1;" ::"r"(remote(smem_u32(&most), 0)), "r"(high) : "memory");
    }
    if (C > 1) cluster_arrive();
    if (scores) {
        for (int i = rank * kSelectThreads + tid; i < a.max_blocks; i += C * kSelectThreads)
            if (i < j0 || i >= j1) scores[i] = i < n ? INFINITY : -INFINITY;
    }
    if (C > 1) cluster_wait();
    else __syncthreads();
    if (rank != 0) return;

    for (int i = want + tid; i < a.top; i += kSelectThreads) selected[i] = -1;
    if (!choose) {
        for (int i = tid; i < n; i += kSelectThreads) selected[i] = i;
        return;
    }
    const int quads = (n + 3) >> 2;                  // of keys
    // The largest key that is not taken whole, and how many of its blocks are: of the scored blocks `need`, the
    // larger keys first. Those in question are lo + [0, span]: neither ~0 nor 0.
    int need = want - (n - (j1 - j0));
    uint32_t edge = ~0u - 1;
    int ties = 0;
    if (need > 0) {
        uint32_t lo = least, span = most - lo;
        int shift = max(0, 21 - __clz(span | 1));
#pragma unroll 1
        for (;;) {
            auto count = [&](uint32_t key) {
                if (key - lo <= span) atomicAdd(&hist[(key - lo) >> shift], 1u);
            };
#pragma unroll 1
            for (int i = tid; i < quads; i += kSelectThreads) {
                const uint4 k = keys4[i];
                count(k.x), count(k.y), count(k.z), count(k.w);
            }
            __syncthreads();
            // From the top: thread t has bins kBins - 4 - 4 t and on.
            const uint4 h = reinterpret_cast<const uint4 *>(hist)[kSelectThreads - 1 - tid];
            const int four = static_cast<int>(h.x + h.y + h.z + h.w);
            const int above = static_cast<int>(scan_before(four, scratch));
            if (above < need && need <= above + four) {
                const int a1 = above + h.w, a2 = a1 + h.z, a3 = a2 + h.y;
                const int at = need <= a1 ? 3 : need <= a2 ? 2 : need <= a3 ? 1 : 0;
                found[0] = kBins - 4 - 4 * tid + at;
                found[1] = at == 3 ? above : at == 2 ? a1 : at == 1 ? a2 : a3;     // above the bin
                found[2] = at == 3 ? h.w : at == 2 ? h.z : at == 1 ? h.y : h.x;    // in it
                found[3] = 0;
            }
            __syncthreads();
            const int in = static_cast<int>(found[2]);
            need -= static_cast<int>(found[1]);
            lo += found[0] << shift;
            if (in == need) {                        // the whole bin
                edge = lo - 1;
                break;
            }
            if (shift == 0) {                        // one key
                edge = lo;
                ties = need;
                break;
            }
            span = (1u << shift) - 1;
            if (in <= kSelectThreads) {              // each one's place among them
                auto take = [&](uint32_t key) {
                    if (key - lo <= span) cand[atomicAdd(&found[3], 1u)] = key;
                };
#pragma unroll 1
                for (int i = tid; i < quads; i += kSelectThreads) {
                    const uint4 k = keys4[i];
                    take(k.x), take(k.y), take(k.z), take(k.w);
                }
                __syncthreads();
                if (tid < in) {
                    const uint32_t key = cand[tid];
                    int more = 0, same = 0;
#pragma unroll 4
                    for (int i = 0; i < in; ++i) {
                        more += cand[i] > key;
                        same += cand[i] == key;
                    }
                    if (more < need && need <= more + same) {
                        found[0] = key;              // (equal ones write the same)
                        found[1] = need - more;
                    }
                }
                __syncthreads();
                edge = found[0];
                ties = static_cast<int>(found[1]);
                break;
            }
            shift = max(0, shift - 11);
            reinterpret_cast<uint4 *>(hist)[tid] = make_uint4(0u, 0u, 0u, 0u);
            __syncthreads();
        }
    }
    // The list: each thread counts its blocks above the edge and at it, and places them behind the threads' before it.
    // (An odd number of 16-byte pieces each: no bank conflicts.)
    const int each = ((quads + kSelectThreads - 1) / kSelectThreads) | 1;
    const int from = min(quads, tid * each), to = min(quads, from + each);
    auto level = [&](uint32_t key) { return key > edge ? 1u << 16 : key == edge ? 1u : 0u; };
    uint32_t count = 0;
#pragma unroll 1
    for (int i = from; i < to; ++i) {
        const uint4 k = keys4[i];
        count += level(k.x) + level(k.y) + level(k.z) + level(k.w);
    }
    const uint32_t before = scan_before(count, scratch);
    if (count == 0) return;
    int e = static_cast<int>(before & 0xFFFF), at = static_cast<int>(before >> 16) + min(e, ties);
#pragma unroll 1
    for (int i = from; i < to; i += 8) {             // a bit per block
        uint32_t m = 0;
#pragma unroll 1
        for (int c = 0; c < 8 && i + c < to; ++c) {
            const uint4 k = keys4[i + c];
            m |= ((k.x >= edge) | (k.y >= edge) << 1 | (k.z >= edge) << 2 | (k.w >= edge) << 3) << (4 * c);
        }
#pragma unroll 1
        for (; m != 0; m &= m - 1) {
            const int block = 4 * i + __ffs(m) - 1;
            const bool tie = keys[block] == edge;
            if (!tie || e < ties) selected[at++] = block;
            e += tie;
        }
    }
}

}  // namespace

cudaError_t launch_bounds(const BoundsArgs &a, int num_sms, cudaStream_t st) {
    const int64_t most = (static_cast<int64_t>(a.B) * a.max_blocks * a.nlayers * a.s.Hkv + kBoundsThreads / 32 - 1) /
                         (kBoundsThreads / 32);
    const int64_t ctas = static_cast<int64_t>(kBoundsPerSm) * num_sms;   // all resident
    return launch_behind(bounds_kernel, dim3(static_cast<unsigned>(most < ctas ? most : ctas)), 0, kBoundsThreads, a.B * 8, st, a);
}

cudaError_t prepare_select_kernel(SelectFit *fit) {
    cudaError_t e = cudaSuccess;
    for (int two = 0; two < 2 && e == cudaSuccess; ++two)
        e = fit_clusters(two ? select_kernel<true> : select_kernel<false>, kSelectThreads, select_smem(kSelectBlocksMax),
                         select_smem(8192), fit->clusters[two]);
    // The longest rows of which two CTAs still share an SM: their keys are in shared memory.
    fit->pair_blocks = 0;
    for (int blocks = 8192, ctas = 2; e == cudaSuccess && ctas >= 2 && blocks <= kSelectBlocksMax; blocks += 1024) {
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, select_kernel<false>, kSelectThreads, select_smem(blocks));
        if (e == cudaSuccess && ctas >= 2) fit->pair_blocks = blocks;
    }
    return e;
}

cudaError_t launch_select(const SelectArgs &a, const SelectFit &fit, cudaStream_t st) {
    // The largest clusters that are all resident at once, of at least 64 blocks a CTA. us with the widest that fits
    // and the next wider one (rotating inputs): 8 units of 1 250 blocks 6.5 (8 CTAs) and 10.0, 32 of up to 7 500 14.4
    // (4) and 18.1, 64 of up to 1 875 9.0 (2) and 13.2. Too many units for two CTAs of an SM each: two to an SM, 512
    // units of up to 1 250 28.4, by CTAs of an SM each 32.0. Where the tables are too wide for two to an SM, CTAs of an
    // SM each and no clusters: 152 units of 1 250 blocks in tables of 40 000 13.1, as if two still shared an SM 22.9;
    // 512 units of 40 000 blocks 660 and 938.
    const int64_t units = static_cast<int64_t>(a.B) * a.s.Hkv;
    int two = 1, log = 4;
    while (log > 0 && (units > fit.clusters[1][log] || a.max_blocks < 64 << log)) --log;
    if (log == 0 && units > fit.clusters[1][0] / 2 && a.max_blocks <= fit.pair_blocks) {
        two = 0;
        log = 4;
        while (log > 0 && (units > fit.clusters[0][log] || a.max_blocks < 64 << log)) --log;
    }
    return launch_behind(two ? select_kernel<true> : select_kernel<false>, dim3(1 << log, a.s.Hkv, a.B), 1 << log,
                         kSelectThreads, select_smem(a.max_blocks), st, a);
}

}  // namespace kvt
