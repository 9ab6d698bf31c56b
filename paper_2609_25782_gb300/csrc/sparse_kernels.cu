// Kernels of attention over a part of the cache, for sm_103a.
//
//   bounds_kernel   channelwise bounds of the keys of blocks, in 8 bits
//   select_kernel   scores of blocks from the bounds, and the `top` largest
//   sparse_kernel   attention of one new token per session over listed blocks
#include <cuda_bf16.h>

#include "cache_ops.h"
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

constexpr int kBoundsThreads = 256;

// A warp per (block, layer, kv-head). The rows' block counts are summed up by every CTA first, so that the
// items are one line whatever the lengths; a warp finds its row in it by bisection.
__global__ void __launch_bounds__(kBoundsThreads) bounds_kernel(const BoundsArgs a) {
    __shared__ int ends[kBoundsRowsMax];
    __shared__ int sums[kBoundsThreads / 32];
    const Shape sh = a.s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int total = 0;
    for (int b0 = 0; b0 < a.B; b0 += kBoundsThreads) {
        const int b = b0 + threadIdx.x;
        int n = 0;
        if (b < a.B) {
            const int2 r = bounds_blocks(a, b);
            n = r.y - r.x;
            if (r.x < 0 && blockIdx.x == 0) atomicOr(a.err, kErrBadLength);
        }
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
        if (b < a.B) ends[b] = before + n;
        __syncthreads();
    }
    const int per = a.nlayers * sh.Hkv;              // items of a block
    const int64_t items = static_cast<int64_t>(total) * per;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kBoundsThreads / 32);
    for (int64_t it = static_cast<int64_t>(blockIdx.x) * (kBoundsThreads / 32) + warp; it < items; it += warps) {
        const int pair = static_cast<int>(it / per);
        const int rest = static_cast<int>(it - static_cast<int64_t>(pair) * per);
        const int l = a.layer0 + rest / sh.Hkv, g = rest % sh.Hkv;
        int lo = 0, hi = a.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (ends[mid] > pair) hi = mid;
            else lo = mid + 1;
        }
        const int2 r = bounds_blocks(a, lo);
        const int j = r.x + pair - (lo ? ends[lo - 1] : 0);
        const int blk = a.tables[static_cast<int64_t>(lo) * a.max_blocks + j];
        if (blk < 0 || blk >= sh.num_blocks) {
            if (lane == 0) atomicOr(a.err, kErrBadBlock);
            continue;
        }
        const int tokens = min(sh.bt, a.seq_lens[lo] - j * sh.bt);
        const int64_t row = ((static_cast<int64_t>(blk) * sh.L + l) * 2 * sh.Hkv + g) * sh.bt;
        const uint4 *k = reinterpret_cast<const uint4 *>(a.hot + row * kHeadDim);
        // Half a warp per token, eight channels a lane.
        __nv_bfloat162 up[4], down[4];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            up[i] = __float2bfloat162_rn(-INFINITY);
            down[i] = __float2bfloat162_rn(INFINITY);
        }
        for (int t0 = 0; t0 < sh.bt; t0 += 16) {
            uint4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (t0 + 2 * i + (lane >> 4) < tokens) v[i] = k[(t0 + 2 * i) * 16 + lane];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (t0 + 2 * i + (lane >> 4) >= tokens) continue;
                const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&w[c]);
                    up[c] = __hmax2(up[c], x);
                    down[c] = __hmin2(down[c], x);
                    most = __vmaxu2(most, w[c] & 0x7FFF7FFFu);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t u = __shfl_xor_sync(~0u, *reinterpret_cast<uint32_t *>(&up[c]), 16);
            const uint32_t d = __shfl_xor_sync(~0u, *reinterpret_cast<uint32_t *>(&down[c]), 16);
            up[c] = __hmax2(up[c], *reinterpret_cast<const __nv_bfloat162 *>(&u));
            down[c] = __hmin2(down[c], *reinterpret_cast<const __nv_bfloat162 *>(&d));
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) most = __vmaxu2(most, __shfl_xor_sync(~0u, most, d));
        const uint32_t top = max(most & 0xFFFFu, most >> 16);
        const bool fine = top < kInfBits;
        const int E = max(1, static_cast<int>(top >> 7)) + ((top & 0x7F) == 0x7F);
        // 2^(133 - E) is up to 2^132: two factors. A value too small for the product still counts: it rounds outwards.
        const float s1 = pow2(min(254, 260 - E)), s2 = pow2(127 + max(0, 6 - E));
        uint32_t bytes[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __nv_bfloat162 p = lane < 16 ? up[i >> 1] : down[i >> 1];
            float x = i & 1 ? __high2float(p) : __low2float(p);
            if (lane >= 16) x = -x;
            const float y = ceilf(x * s1 * s2);
            int c = static_cast<int>(x > 0.f ? fmaxf(y, 1.f) : y);
            if (!fine) c = 127;
            bytes[i] = static_cast<uint32_t>(lane < 16 ? c : -c) & 0xFF;
        }
        const int64_t rec = (static_cast<int64_t>(l) * sh.Hkv + g) * sh.num_blocks + blk;
        uint2 out;
        out.x = bytes[0] | bytes[1] << 8 | bytes[2] << 16 | bytes[3] << 24;
        out.y = bytes[4] | bytes[5] << 8 | bytes[6] << 16 | bytes[7] << 24;
        reinterpret_cast<uint2 *>(a.codes + rec * kCodeRow)[lane] = out;
        // The step as a bf16: 2^(E - 133), below 2^-126 by its fraction bit.
        if (lane == 0)
            a.steps[rec] = static_cast<uint16_t>(!fine ? kInfBits : E > 6 ? (E - 6) << 7 : 1u << E);
    }
}

// ---- selection ---------------------------------------------------------------------------------------

constexpr int kSelectThreads = 256;

// Scores in an order of their bits: larger scores have larger keys. All NaN-free.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);   // one zero
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The whole of a block of threads: the sum of x.
__device__ __forceinline__ int block_sum(int x, int *scratch) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    x = __reduce_add_sync(~0u, x);
    __syncthreads();
    if (lane == 0) scratch[warp] = x;
    __syncthreads();
    int s = 0;
    for (int w = 0; w < kSelectThreads / 32; ++w) s += scratch[w];
    return s;
}

// One CTA per (row, kv-head).
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const SelectArgs a) {
    extern __shared__ uint32_t keys[];
    __shared__ int scratch[kSelectThreads / 32];
    __shared__ int qp[kHeadDim], qn[kHeadDim];
    const Shape sh = a.s;
    const int g = blockIdx.x % sh.Hkv, b = blockIdx.x / sh.Hkv;
    const int G = sh.Hq / sh.Hkv;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int T = a.seq_lens[b];
    const bool bad = !good_length(T, a.max_blocks, sh.bt);
    const int n = bad ? 0 : (T + sh.bt - 1) / sh.bt;
    if (bad && tid == 0) atomicOr(a.err, kErrBadLength);
    int32_t *selected = a.selected + (static_cast<int64_t>(b) * sh.Hkv + g) * a.top;
    float *scores = a.scores ? a.scores + (static_cast<int64_t>(b) * sh.Hkv + g) * a.max_blocks : nullptr;

    // q as whole numbers
    const uint16_t *q = a.q + b * a.q_stride + static_cast<int64_t>(g) * G * kHeadDim;
    int most = 0;
    for (int i = tid; i < G * kHeadDim; i += kSelectThreads) {
        const int m = q[i] & 0x7FFF;
        if (m < static_cast<int>(kInfBits)) most = max(most, m);
    }
    most = __reduce_max_sync(~0u, most);
    if (lane == 0) scratch[warp] = most;
    __syncthreads();
    for (int w = 0; w < kSelectThreads / 32; ++w) most = max(most, scratch[w]);
    const int E = max(1, most >> 7);
    const float s1 = pow2(min(254, 264 - E)), s2 = pow2(127 + max(0, 10 - E));   // 2^(137 - E)
    for (int d = tid; d < kHeadDim; d += kSelectThreads) {
        int p = 0, m = 0;
        for (int h = 0; h < G; ++h) {
            const uint32_t w = q[h * kHeadDim + d];
            if ((w & 0x7FFF) >= kInfBits) continue;
            const int c = __float2int_rn(__uint_as_float(w << 16) * s1 * s2);
            p += max(c, 0);
            m += min(c, 0);
        }
        qp[d] = p;
        qn[d] = m;
    }
    __syncthreads();

    for (int j = warp; j < n; j += kSelectThreads / 32) {
        uint32_t key = 0xFFFFFFFFu;
        float x = INFINITY;
        if (j >= a.first && j < n - a.last) {
            int blk = a.tables[static_cast<int64_t>(b) * a.max_blocks + j];
            if (blk < 0 || blk >= sh.num_blocks) {
                if (lane == 0) atomicOr(a.err, kErrBadBlock);
                blk = 0;
            }
            const int64_t rec = static_cast<int64_t>(g) * sh.num_blocks + blk;
            const int8_t *codes = a.codes + rec * kCodeRow;
            int sum = 0;
            for (int d = lane; d < kHeadDim; d += 32) sum += qp[d] * codes[d] + qn[d] * codes[kHeadDim + d];
            sum = __reduce_add_sync(~0u, sum);
            const uint32_t step = a.steps[rec];
            if (step < kInfBits) x = __fmul_rn(__int2float_rn(sum), __uint_as_float(step << 16));
            key = key_of(x);
        }
        if (lane == 0) {
            keys[j] = key;
            if (scores) scores[j] = x;
        }
    }
    if (scores && !bad)
        for (int j = n + tid; j < a.max_blocks; j += kSelectThreads) scores[j] = -INFINITY;
    __syncthreads();

    // The key that the top-th largest has, bit by bit: the largest with at least `want` keys not below it.
    const int want = min(a.top, n);
    uint32_t edge = 0;
    int above = 0;                                   // keys larger than edge
    if (want > 0) {
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t probe = edge | 1u << bit;
            int c = 0;
            for (int j = tid; j < n; j += kSelectThreads) c += keys[j] >= probe;
            c = block_sum(c, scratch);
            if (c >= want) edge = probe;
        }
        int c = 0;
        for (int j = tid; j < n; j += kSelectThreads) c += keys[j] > edge;
        above = block_sum(c, scratch);
    }
    // In the blocks' order: all above the edge, and the first of those at it.
    int done = 0, ties = 0;
    for (int j0 = 0; j0 < n; j0 += kSelectThreads) {
        const int j = j0 + tid;
        const uint32_t key = j < n ? keys[j] : 0;
        const bool gt = j < n && key > edge, eq = j < n && key == edge;
        const unsigned mg = __ballot_sync(~0u, gt), me = __ballot_sync(~0u, eq);
        __syncthreads();
        if (lane == 0) scratch[warp] = __popc(mg) | __popc(me) << 16;
        __syncthreads();
        const unsigned below = (1u << lane) - 1;
        int bg = __popc(mg & below), be = __popc(me & below), tg = 0, te = 0;
        for (int w = 0; w < kSelectThreads / 32; ++w) {
            const int s = scratch[w];
            if (w < warp) {
                bg += s & 0xFFFF;
                be += s >> 16;
            }
            tg += s & 0xFFFF;
            te += s >> 16;
        }
        const int rank = ties + be;                  // ties before this one
        if (gt || (eq && rank < want - above)) selected[done + bg + min(rank, want - above)] = j;
        done += tg;
        ties += te;
    }
    for (int i = want + tid; i < a.top; i += kSelectThreads) selected[i] = -1;
}

// ---- attention ---------------------------------------------------------------------------------------

constexpr int kSparseThreads = 128;

// One CTA per (row, query head), a warp per token in turn, four dims a lane.
__global__ void __launch_bounds__(kSparseThreads) sparse_kernel(const SparseArgs a) {
    constexpr int kWarps = kSparseThreads / 32;
    __shared__ float s_m[kWarps], s_l[kWarps];
    __shared__ float4 s_o[kWarps][32];
    const Shape sh = a.s;
    const int h = blockIdx.x % sh.Hq, b = blockIdx.x / sh.Hq;
    const int G = sh.Hq / sh.Hkv, g = h / G;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int T = a.seq_lens[b];
    if (!good_length(T, a.max_blocks, sh.bt)) {
        if (threadIdx.x == 0) atomicOr(a.err, kErrBadLength);
        return;
    }
    const int32_t *trow = a.tables + static_cast<int64_t>(b) * a.max_blocks;
    const int32_t *list = a.selected + (static_cast<int64_t>(b) * sh.Hkv + g) * a.top;
    auto four = [&](const uint16_t *row) {
        const uint2 w = reinterpret_cast<const uint2 *>(row)[lane];
        return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u),
                           __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u));
    };
    auto row_of = [&](int blk, int t, int kv) {
        const int j = t / sh.bt;
        return (((static_cast<int64_t>(blk) * sh.L + a.layer) * 2 + kv) * sh.Hkv + g) * sh.bt + t - j * sh.bt;
    };
    const uint16_t *k_new = a.k_new ? a.k_new + b * a.kv_stride + g * kHeadDim : nullptr;
    const uint16_t *v_new = a.k_new ? a.v_new + b * a.kv_stride + g * kHeadDim : nullptr;
    if (k_new && T > 0 && h == g * G && warp == 0) {
        const int blk = trow[(T - 1) / sh.bt];
        if (blk < 0 || blk >= sh.num_blocks) {
            if (lane == 0) atomicOr(a.err, kErrBadBlock);
        } else {
            reinterpret_cast<uint2 *>(a.hot + row_of(blk, T - 1, 0) * kHeadDim)[lane] = reinterpret_cast<const uint2 *>(k_new)[lane];
            reinterpret_cast<uint2 *>(a.hot + row_of(blk, T - 1, 1) * kHeadDim)[lane] = reinterpret_cast<const uint2 *>(v_new)[lane];
        }
    }
    const float4 q = four(a.q + b * a.q_stride + static_cast<int64_t>(h) * kHeadDim);
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int e = 0; e < a.top; ++e) {
        const int j = list[e];
        if (j < 0) continue;
        const int blk = static_cast<int64_t>(j) * sh.bt < T ? trow[j] : -1;
        if (blk < 0 || blk >= sh.num_blocks) {
            if (threadIdx.x == 0) atomicOr(a.err, kErrBadBlock);
            continue;
        }
        const int end = min(T, (j + 1) * sh.bt);
        for (int t = j * sh.bt + warp; t < end; t += kWarps) {
            const bool fresh = k_new && t == T - 1;
            const float4 k = four(fresh ? k_new : a.hot + row_of(blk, t, 0) * kHeadDim);
            const float4 v = four(fresh ? v_new : a.hot + row_of(blk, t, 1) * kHeadDim);
            float x = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) x += __shfl_xor_sync(~0u, x, d);
            x *= a.scale_log2;
            const float mn = fmaxf(m, x), c = ex2(m - mn), w = ex2(x - mn);
            m = mn;
            l = l * c + w;
            o = make_float4(o.x * c + w * v.x, o.y * c + w * v.y, o.z * c + w * v.z, o.w * c + w * v.w);
        }
    }
    if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
    }
    s_o[warp][lane] = o;
    __syncthreads();
    if (warp != 0) return;
    float M = -INFINITY;
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w]);
    float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    for (int w = 0; w < kWarps; ++w) {
        const float c = M == -INFINITY ? 0.f : ex2(s_m[w] - M);
        const float4 y = s_o[w][lane];
        sum += c * s_l[w];
        r = make_float4(r.x + c * y.x, r.y + c * y.y, r.z + c * y.z, r.w + c * y.w);
    }
    const float inv = sum > 0.f ? __frcp_rn(sum) : 0.f;
    r = make_float4(r.x * inv, r.y * inv, r.z * inv, r.w * inv);
    const int64_t row = static_cast<int64_t>(b) * sh.Hq + h;
    if (a.out_bf16) {
        float r0, r1;
        uint2 pk;
        pk.x = pack_bf16(r.x, r.y, r0, r1);
        pk.y = pack_bf16(r.z, r.w, r0, r1);
        reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + row * kHeadDim)[lane] = pk;
    } else {
        reinterpret_cast<float4 *>(static_cast<float *>(a.out) + row * kHeadDim)[lane] = r;
    }
}

}  // namespace

cudaError_t launch_bounds(const BoundsArgs &a, int num_sms, cudaStream_t st) {
    const int64_t most = (static_cast<int64_t>(a.B) * a.max_blocks * a.nlayers * a.s.Hkv + kBoundsThreads / 32 - 1) /
                         (kBoundsThreads / 32);
    const int64_t ctas = 8ll * num_sms;
    bounds_kernel<<<static_cast<unsigned>(most < ctas ? most : ctas), kBoundsThreads, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_select(const SelectArgs &a, int, cudaStream_t st) {
    const int bytes = a.max_blocks * 4;
    if (bytes > 40 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   kSelectBlocksMax * 4);
        if (e != cudaSuccess) return e;
    }
    select_kernel<<<a.B * a.s.Hkv, kSelectThreads, bytes, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_sparse(const CUtensorMap &, const SparseArgs &a, int, cudaStream_t st) {
    sparse_kernel<<<a.B * a.s.Hq, kSparseThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace kvt
