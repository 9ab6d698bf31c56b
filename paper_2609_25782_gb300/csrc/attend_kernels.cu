// Attention of one new token per session over listed blocks, for sm_103a.
//
// A row's heads of one kv-head (a unit) are one cluster's. Its tiles (16 tokens of a listed block, K and V, 8 KiB)
// go round robin to the cluster's warps, each of which copies its own by TMA into a ring of its own and keeps
// one running softmax over them: S^T[16 tok x 8 heads] = K Q^T and O^T[128 x 8] += V^T P^T on mma.sync. The states
// of a CTA's warps merge in its shared memory; each head's are then sent to one CTA of the cluster, which merges
// and writes it. So a call needs no workspace and no second launch, and the same list gives the same bits.
//
// Bound by HBM where there is much to read: 48 sessions, 8 KV heads, 64 blocks of 64 tokens a head (805 MB) 119 us,
// 6.75 TB/s. A call of one session is a chain of latencies: list, table, copy, products, two merges, 6 us for 128
// blocks of 16 tokens a head.
#include <cuda_bf16.h>

#include "cache_ops.h"
#include "cluster.cuh"
#include "tile_ops.cuh"

namespace kvt {
namespace {

constexpr int kItems = 64;           // places of tiles that a warp holds: two lists of 32

// Two shapes: few units get clusters of CTAs of 8 warps that have an SM each, so that a warp has few tiles one after
// another; many get a CTA of 4 warps each, three per SM.
template <int kWarps, int kStages>
struct Layout {
    static constexpr bool kCluster = kWarps == 8;
    static constexpr int kRows = kCluster ? 16 : 0;   // that a CTA receives: its ceil(8 / C) heads from C CTAs
    static constexpr int kRing = kWarps * kStages * kTileBytes;
    static constexpr int kRecvO = kRing;
    static constexpr int kRecvMl = kRecvO + kRows * kHeadDim * 4;
    static constexpr int kPlaces = kRecvMl + kRows * 8;
    static constexpr int kBars = kPlaces + kWarps * kItems * 8;
    static constexpr int kBytes = kBars + kWarps * kStages * 8 + 1024;  // and alignment
};

struct State {
    float m0, m1;   // running maximum (log2 units) of heads 2 * (lane % 4) and + 1, lazily moved
    float l0, l1;   // this lane's share of the sums
    float o[8][4];  // O^T fragments
};

// A reference that differences can be taken with: nothing seen yet, or only scores of -inf.
__device__ __forceinline__ float finite(float m) { return m == -INFINITY ? 0.f : m; }

template <int kWarps, int kStages>
__global__ void __launch_bounds__(kWarps * 32, kWarps == 8 ? 1 : 3)
    sparse_kernel(const __grid_constant__ CUtensorMap map, const SparseArgs a) {
    using Lay = Layout<kWarps, kStages>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const Shape sh = a.s;
    // A row of the grid is a cluster.
    const int C = Lay::kCluster ? gridDim.x : 1, rank = Lay::kCluster ? blockIdx.x : 0, g = blockIdx.y, b = blockIdx.z;
    const int G = a.group;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    after_previous();
    const int T = a.seq_lens[b];
    const int32_t *trow = a.tables + static_cast<int64_t>(b) * a.max_blocks;
    const int32_t *list = a.selected + (static_cast<int64_t>(b) * sh.Hkv + g) * a.top;

    // The warp's tiles are first, first + step, ... of the list's; 32 places at a time, one a lane.
    const int per = sh.bt / kTileTokens, shift = sh.bt == kTileTokens ? 0 : 2;   // tiles of a block
    const int tiles = a.top * per;
    const int first = rank * kWarps + warp, step = C * kWarps;
    const int mine = first < tiles ? (tiles - first + step - 1) / step : 0;
    auto entry = [&](int c) {                         // of the lane's tile in list c
        const int k = c * 32 + lane;
        return k < mine ? list[(first + k * step) >> shift] : -1;
    };
    auto token = [&](int c, int j) {                  // its first one, or -1 where there is none
        const int64_t t = static_cast<int64_t>(j) * sh.bt + ((first + (c * 32 + lane) * step) & (per - 1)) * kTileTokens;
        return j >= 0 && t < T ? static_cast<int>(t) : -1;
    };
    int j_now = entry(0), j_next = entry(1);
    // (A row of a bad length is left by the whole cluster.)
    if (T < 0 || T > INT32_MAX - 512 || T > static_cast<int64_t>(a.max_blocks) * sh.bt) {
        if (rank == 0 && threadIdx.x == 0) atomicOr(a.err, kErrBadLength);
        return;
    }
    if (C > 1) cluster_arrive();                      // this CTA has started
    int t_now = token(0, j_now);
    int blk_now = t_now >= 0 ? trow[j_now] : 0;

    uint8_t *ring = smem + warp * kStages * kTileBytes;
    const uint32_t ring_s = smem_u32(ring);
    int2 *places = reinterpret_cast<int2 *>(smem + Lay::kPlaces) + warp * kItems;   // pool row, first token
    const uint32_t bar0 = smem_u32(smem + Lay::kBars) + warp * kStages * 8;
    if (lane == 0) {
        for (int i = 0; i < kStages; ++i) mbar_init(bar0 + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const uint16_t *k_new = a.k_new ? a.k_new + b * a.kv_stride + g * kHeadDim : nullptr;
    const uint16_t *v_new = a.k_new ? a.v_new + b * a.kv_stride + g * kHeadDim : nullptr;
    // Lanes 0-15: the new token's K, 16-31: its V.
    const uint4 fresh = k_new ? reinterpret_cast<const uint4 *>(lane < 16 ? k_new : v_new)[lane & 15] : make_uint4(0u, 0u, 0u, 0u);

    // Places of the next 32 tiles, those that there are one after the other; what a later list needs is loaded.
    int placed = 0, list_no = 0;
    const int lists = (mine + 31) >> 5;
    auto place = [&]() {
        const int part = t_now & (sh.bt - 1);
        bool ok = t_now >= 0;
        if (j_now >= 0 && static_cast<int64_t>(j_now) * sh.bt >= T) atomicOr(a.err, kErrBadBlock);
        if (ok && (blk_now < 0 || blk_now >= sh.num_blocks)) {
            atomicOr(a.err, kErrBadBlock);
            ok = false;
        }
        const unsigned m = __ballot_sync(~0u, ok);
        if (ok)   // the pool has fewer than 2^31 rows
            places[(placed + __popc(m & ((1u << lane) - 1))) & (kItems - 1)] =
                make_int2(((blk_now * sh.L + a.layer) * 2 * sh.Hkv + g) * sh.bt + part, t_now);
        placed += __popc(m);
        ++list_no;
        j_now = j_next;
        t_now = token(list_no, j_now);
        blk_now = t_now >= 0 ? trow[j_now] : 0;
        j_next = entry(list_no + 1);
        __syncwarp();
    };
    // inject_extra_tx (a test of the bounded wait, 0 in normal calls): this one barrier then never completes.
    const int inject = rank == 0 && g == 0 && b == 0 && warp == 0 ? a.inject_extra_tx : 0;
    int issued = 0;
    auto issue = [&]() {                              // the next tile, if there is one, into its slot
        while (issued == placed && list_no < lists) place();
        if (issued == placed) return;
        if (lane == 0) {
            const uint32_t bar = bar0 + 8 * (issued % kStages);
            mbar_expect_tx(bar, kTileBytes + (issued == 0 ? inject : 0));
            tma_load_tile<false>(ring_s + (issued % kStages) * kTileBytes, &map, places[issued & (kItems - 1)].x, bar, 0);
        }
        ++issued;
    };
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) issue();

    if (k_new && rank == 0 && warp == 0 && T > 0) {   // the new token's slot, listed or not
        const int j = (T - 1) / sh.bt, blk = trow[j];
        if (blk < 0 || blk >= sh.num_blocks) {
            if (lane == 0) atomicOr(a.err, kErrBadBlock);
        } else {
            const int row = ((blk * sh.L + a.layer) * 2 * sh.Hkv + g) * sh.bt + (T - 1 - j * sh.bt) + (lane >> 4) * sh.Hkv * sh.bt;
            reinterpret_cast<uint4 *>(a.hot + static_cast<int64_t>(row) * kHeadDim)[lane & 15] = fresh;
        }
    }
    // Q^T fragments (mma B operand): head lane / 4 of the group, dims 16 i + 2 (lane % 4) + {0, 1} and + 8.
    uint32_t qb[8][2];
    {
        const int n = lane >> 2;
        const uint32_t *q = reinterpret_cast<const uint32_t *>(a.q + b * a.q_stride + (static_cast<int64_t>(g) * G + (n < G ? n : 0)) * kHeadDim) + (lane & 3);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            qb[i][0] = n < G ? q[i * 8] : 0u;
            qb[i][1] = n < G ? q[i * 8 + 4] : 0u;
        }
    }
    uint32_t koff[4], voff[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        koff[i] = k_offset(lane, i);
        voff[i] = v_offset(lane, i);
    }
    State s;
    s.m0 = s.m1 = -INFINITY;
    s.l0 = s.l1 = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s.o[i][0] = s.o[i][1] = s.o[i][2] = s.o[i][3] = 0.f;

#pragma unroll 1
    for (int k = 0; k < issued; ++k) {
        const uint32_t bar = bar0 + 8 * (k % kStages);
        if (!__all_sync(~0u, mbar_wait(bar, (k / kStages) & 1))) {
            // No copy may land after the CTA has gone.
            if (lane == 0) atomicOr(a.err, kErrTimeout);
#pragma unroll 1
            for (int i = k; i < issued; ++i) mbar_wait(bar0 + 8 * (i % kStages), (i / kStages) & 1);
            break;
        }
        const uint32_t slot = ring_s + (k % kStages) * kTileBytes;
        const int t0 = places[k & (kItems - 1)].y;
        const bool tail = t0 + kTileTokens >= T;      // the session's last token or what lies behind it
        if (tail) {
            uint8_t *tile = ring + (k % kStages) * kTileBytes;
            if (k_new)
                *reinterpret_cast<uint4 *>(tile + (lane >> 4) * 2 * kHalfBytes + ((lane >> 3) & 1) * kHalfBytes +
                                           swz(T - 1 - t0, lane & 7)) = fresh;
            clear_tail_v(T, t0, tile, lane);
        }
        float sa[4] = {0.f, 0.f, 0.f, 0.f}, sb[4] = {0.f, 0.f, 0.f, 0.f}, x[4];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            uint32_t f[2][4];
            ldsm_x4(slot + koff[i & 3] + (i >> 2) * kHalfBytes, f[0][0], f[0][1], f[0][2], f[0][3]);
            ldsm_x4(slot + koff[(i + 1) & 3] + (i >> 2) * kHalfBytes, f[1][0], f[1][1], f[1][2], f[1][3]);
            mma_bf16(sa, f[0][0], f[0][1], f[0][2], f[0][3], qb[i][0], qb[i][1]);
            mma_bf16(sb, f[1][0], f[1][1], f[1][2], f[1][3], qb[i + 1][0], qb[i + 1][1]);
        }
        uint32_t vf[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            ldsm_x4_t(slot + voff[i & 3] + (i >> 2) * kHalfBytes, vf[i][0], vf[i][1], vf[i][2], vf[i][3]);
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = t0 + (lane >> 2) + (c >> 1) * 8 < T ? (sa[c] + sb[c]) * a.scale_log2 : -INFINITY;
        // The reference moves when a score exceeds it by more than kLazyLog2: weights are 2^kLazyLog2 at most.
        const bool grows = (x[0] > s.m0 + kLazyLog2) | (x[2] > s.m0 + kLazyLog2) | (x[1] > s.m1 + kLazyLog2) |
                           (x[3] > s.m1 + kLazyLog2);
        if (__any_sync(~0u, grows)) {
            float mx0 = fmaxf(x[0], x[2]), mx1 = fmaxf(x[1], x[3]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) {
                mx0 = fmaxf(mx0, __shfl_xor_sync(~0u, mx0, d));
                mx1 = fmaxf(mx1, __shfl_xor_sync(~0u, mx1, d));
            }
            const float n0 = fmaxf(s.m0, mx0), n1 = fmaxf(s.m1, mx1);
            const float c0 = ex2(s.m0 - finite(n0)), c1 = ex2(s.m1 - finite(n1));
            s.m0 = n0;
            s.m1 = n1;
            s.l0 *= c0;
            s.l1 *= c1;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s.o[i][0] *= c0;
                s.o[i][1] *= c1;
                s.o[i][2] *= c0;
                s.o[i][3] *= c1;
            }
        }
        // Weights in bf16, as the product with V sees them; the sum is of the rounded ones.
        float q0, q1, q2, q3;
        const float r0 = finite(s.m0), r1 = finite(s.m1);
        const uint32_t p01 = pack_bf16(ex2(x[0] - r0), ex2(x[1] - r1), q0, q1);
        const uint32_t p23 = pack_bf16(ex2(x[2] - r0), ex2(x[3] - r1), q2, q3);
        s.l0 += q0 + q2;
        s.l1 += q1 + q3;
        const uint32_t pb0 = movmatrix_t(p01), pb1 = movmatrix_t(p23);
#pragma unroll
        for (int i = 0; i < 8; ++i) mma_bf16(s.o[i], vf[i][0], vf[i][1], vf[i][2], vf[i][3], pb0, pb1);
        // The slot's next copy comes behind this warp's reads and, through the other proxy, its own stores.
        if (tail) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        issue();
    }

    next_may_come();
    // States into the warp's own ring, which no copy writes any more.
    {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            s.l0 += __shfl_xor_sync(~0u, s.l0, d);
            s.l1 += __shfl_xor_sync(~0u, s.l1, d);
        }
        float *ws = reinterpret_cast<float *>(ring), *wm = ws + kMaxGroup * kOStride;
        const int h = 2 * (lane & 3), d = lane >> 2;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ws[h * kOStride + 16 * i + d] = s.o[i][0];
            ws[(h + 1) * kOStride + 16 * i + d] = s.o[i][1];
            ws[h * kOStride + 16 * i + d + 8] = s.o[i][2];
            ws[(h + 1) * kOStride + 16 * i + d + 8] = s.o[i][3];
        }
        if (lane < 4) {
            wm[h] = s.m0;
            wm[h + 1] = s.m1;
            wm[kMaxGroup + h] = s.l0;
            wm[kMaxGroup + h + 1] = s.l1;
        }
    }
    __syncthreads();
    if (C > 1) cluster_wait();                        // every CTA has started: its memory may be written

    auto store = [&](int h, float4 r, float l) {
        const float inv = l != 0.f ? __frcp_rn(l) : 0.f;
        r = make_float4(r.x * inv, r.y * inv, r.z * inv, r.w * inv);
        const int64_t row = static_cast<int64_t>(b) * sh.Hq + g * G + h;
        if (a.out_bf16) {
            float y0, y1;
            uint2 pk;
            pk.x = pack_bf16(r.x, r.y, y0, y1);
            pk.y = pack_bf16(r.z, r.w, y0, y1);
            reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + row * kHeadDim)[lane] = pk;
        } else {
            reinterpret_cast<float4 *>(static_cast<float *>(a.out) + row * kHeadDim)[lane] = r;
        }
    };
    // A warp per head, four dims a lane.
#pragma unroll 1
    for (int h = warp; h < G; h += kWarps) {
        float m[kWarps], M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            m[w] = reinterpret_cast<const float *>(smem + w * kStages * kTileBytes)[kMaxGroup * kOStride + h];
            M = fmaxf(M, m[w]);
        }
        float l = 0.f;
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float *ws = reinterpret_cast<const float *>(smem + w * kStages * kTileBytes);
            const float c = ex2(m[w] - finite(M));
            const float4 o = reinterpret_cast<const float4 *>(ws + h * kOStride)[lane];
            l += c * ws[kMaxGroup * kOStride + kMaxGroup + h];
            r = make_float4(r.x + c * o.x, r.y + c * o.y, r.z + c * o.z, r.w + c * o.w);
        }
        if (C == 1) {
            store(h, r, l);
            continue;
        }
        const uint32_t to = h % C, at = (h / C) * C + rank;
        const uint32_t o_at = remote(smem_u32(smem + Lay::kRecvO) + (at * kHeadDim + 4 * lane) * 4, to);
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(o_at), "f"(r.x), "f"(r.y), "f"(r.z), "f"(r.w) : "memory");
        if (lane == 0) {
            const uint32_t ml_at = remote(smem_u32(smem + Lay::kRecvMl) + at * 8, to);
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(ml_at), "f"(M), "f"(l) : "memory");
        }
    }
    if (C == 1) return;
    cluster_arrive();
    cluster_wait();
#pragma unroll 1
    for (int h = rank + warp * C, at = warp * C; h < G; h += kWarps * C, at += kWarps * C) {
        const float2 *ml = reinterpret_cast<const float2 *>(smem + Lay::kRecvMl) + at;
        const float4 *o = reinterpret_cast<const float4 *>(smem + Lay::kRecvO) + at * (kHeadDim / 4) + lane;
        float M = -INFINITY, l = 0.f;
        float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i = 0; i < C; ++i) M = fmaxf(M, ml[i].x);
        for (int i = 0; i < C; ++i) {
            const float c = ex2(ml[i].x - finite(M));
            const float4 y = o[i * (kHeadDim / 4)];
            l += c * ml[i].y;
            r = make_float4(r.x + c * y.x, r.y + c * y.y, r.z + c * y.z, r.w + c * y.w);
        }
        store(h, r, l);
    }
}

}  // namespace

cudaError_t prepare_sparse_kernels(SparseFit *fit) {
    const cudaError_t e = cudaFuncSetAttribute(sparse_kernel<4, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<4, 2>::kBytes);
    return e != cudaSuccess ? e : fit_clusters(sparse_kernel<8, 3>, 8 * 32, Layout<8, 3>::kBytes, Layout<8, 3>::kBytes, fit->clusters);
}

cudaError_t launch_sparse(const CUtensorMap &map, const SparseArgs &a, const SparseFit &fit, cudaStream_t st) {
    const int64_t units = static_cast<int64_t>(a.B) * a.s.Hkv;
    const int64_t tiles = static_cast<int64_t>(a.top < a.max_blocks ? a.top : a.max_blocks) * (a.s.bt / kTileTokens);
    // As many CTAs of 8 warps, an SM each, as are resident at once, of at least a tile a warp; where there are more
    // units than those, CTAs of 4 warps and no clusters. us by (warps, CTAs of a cluster), inputs rotating, one layer:
    // 4 units of 128 tiles (8, 16) 6.0, (8, 8) 6.4, (8, 4) 7.7, (4, 8) 6.6; 16 units (8, 4) 7.6, (8, 8) 11.3 (not
    // resident at once), (4, 8) 7.2; 64 units (8, 2) 16.2, (8, 1) 15.9, (4, 4) 15.9, (4, 8) 20.6; 256 units (4, 1) 43.9,
    // (8, 1) 45.9, (4, 2) 51.0; 384 units of 256 tiles (4, 1) 119.3, (8, 1) 116.9, (4, 4) 120.7.
    int log = 4;
    while (log > 0 && (units > fit.clusters[log] || tiles < 8 << log)) --log;
    const bool wide = units <= fit.clusters[0];
    return wide ? launch_behind(sparse_kernel<8, 3>, dim3(1 << log, a.s.Hkv, a.B), 1 << log, 8 * 32, Layout<8, 3>::kBytes, st, map, a)
                : launch_behind(sparse_kernel<4, 2>, dim3(1, a.s.Hkv, a.B), 0, 4 * 32, Layout<4, 2>::kBytes, st, map, a);
}

}  // namespace kvt
