// Attention of several new tokens per session over the paged cache, for sm_103a:
// a turn's context or a whole prompt (causal, its K and V written into the hot
// pool), and drafted tokens (a bit mask per draft, nothing written).
#include <cuda_bf16.h>

#include "kvt_internal.h"

namespace kvt {
namespace {

__device__ __forceinline__ float2 unpack2(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

__device__ __forceinline__ float4 load4(const uint16_t *p, int lane) {
    const uint2 w = reinterpret_cast<const uint2 *>(p)[lane];
    const float2 a = unpack2(w.x), b = unpack2(w.y);
    return make_float4(a.x, a.y, b.x, b.y);
}

// One CTA per (new token, kv-head), one warp per query head of the group: the
// keys one by one, an online softmax in 32 bits.
__global__ void __launch_bounds__(kMaxGroup * 32) turn_simple_kernel(const TurnArgs a) {
    const Shape sh = a.s;
    const int row = blockIdx.x, g = blockIdx.y;
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int b = 0;
    while (b < a.B && !(a.cu[b] <= row && row < a.cu[b + 1])) ++b;
    if (b == a.B) return;
    const int lo = a.cu[b], n = a.cu[b + 1] - lo, T = a.seq_lens[b];
    const int P = a.masks ? T : T - n;
    if (lo < 0 || lo + n > a.total || P < 0 || T > static_cast<int64_t>(a.max_blocks) * sh.bt ||
        (a.masks && n > kMaxDrafts)) {
        if (threadIdx.x == 0) atomicOr(a.err, kErrBadLength);
        return;
    }
    const int i = row - lo, G = sh.Hq / sh.Hkv;
    const int32_t *table = a.tables + static_cast<int64_t>(b) * a.max_blocks;
    auto pool_row = [&](int t, int kv) -> uint16_t * {
        const int blk = table[t / sh.bt];
        if (blk < 0 || blk >= sh.num_blocks) {
            if (lane == 0) atomicOr(a.err, kErrBadBlock);
            return nullptr;
        }
        return a.hot + ((((static_cast<int64_t>(blk) * sh.L + a.layer) * 2 + kv) * sh.Hkv + g) * sh.bt + t % sh.bt) *
                           kHeadDim;
    };
    if (!a.masks && w == 0) {   // the token's K and V go to their slots
        for (int kv = 0; kv < 2; ++kv) {
            const uint16_t *src = (kv ? a.v_new : a.k_new) + row * a.kv_stride + g * kHeadDim;
            uint16_t *dst = pool_row(P + i, kv);
            if (dst) reinterpret_cast<uint2 *>(dst)[lane] = reinterpret_cast<const uint2 *>(src)[lane];
        }
    }
    if (w >= G) return;
    const int h = g * G + w;
    const float4 q = load4(a.q + row * a.q_stride + h * kHeadDim, lane);
    float m = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const uint64_t mask = a.masks ? a.masks[row] : 0;
    for (int t = 0; t < P + n; ++t) {
        const int j = t - P;   // >= 0: one of the call's own tokens
        if (j >= 0 && !(a.masks ? mask >> j & 1 : j <= i)) continue;
        const uint16_t *kr, *vr;
        if (j >= 0) {
            kr = a.k_new + (lo + j) * a.kv_stride + g * kHeadDim;
            vr = a.v_new + (lo + j) * a.kv_stride + g * kHeadDim;
        } else {
            kr = pool_row(t, 0);
            vr = pool_row(t, 1);
            if (!kr) continue;
        }
        const float4 k = load4(kr, lane), v = load4(vr, lane);
        float x = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
        for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
        x *= a.scale_log2;
        const float mn = fmaxf(m, x), c = exp2f(m - mn), p = exp2f(x - mn);
        m = mn;
        l = l * c + p;
        acc = make_float4(acc.x * c + p * v.x, acc.y * c + p * v.y, acc.z * c + p * v.z, acc.w * c + p * v.w);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    const int64_t to = (static_cast<int64_t>(row) * sh.Hq + h) * kHeadDim;
    const float4 y = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (a.out_bf16) {
        const __nv_bfloat162 y0 = __floats2bfloat162_rn(y.x, y.y), y1 = __floats2bfloat162_rn(y.z, y.w);
        reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + to)[lane] =
            make_uint2(*reinterpret_cast<const uint32_t *>(&y0), *reinterpret_cast<const uint32_t *>(&y1));
    } else {
        reinterpret_cast<float4 *>(static_cast<float *>(a.out) + to)[lane] = y;
    }
}

}  // namespace

cudaError_t launch_turn(const TurnArgs &a, cudaStream_t st) {
    if (a.total < 1) return cudaSuccess;
    turn_simple_kernel<<<dim3(a.total, a.s.Hkv), kMaxGroup * 32, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace kvt
