// What the kernels that read K and V tile by tile share (decode_kernels.cu, sparse_kernels.cu): barriers
// with bounded waits, the copy of a tile, the fragments of its products.
#pragma once

#include <cuda_bf16.h>
#include <cuda.h>

#include <cstdint>

#include "kvt_internal.h"

namespace kvt {
namespace {

constexpr int kTileBytes = 8192;           // K 4 KiB + V 4 KiB
constexpr int kHalfBytes = 2048;           // 16 rows x 128 B (64 dims)
// Lazy softmax maximum: the reference moves when a logit exceeds it by more
// than this many powers of two (P then stays at most 2^8 = 256).
constexpr float kLazyLog2 = 8.f;
constexpr unsigned long long kWaitLimitNs = 2000000000ull;   // 2 s


__device__ __forceinline__ uint32_t smem_u32(const void *p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

__device__ __forceinline__ unsigned long long global_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}

__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                 : "memory");
}

__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Non-blocking form: has the phase completed?
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Wait for a phase with a wall-clock limit; false means the limit expired.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_ns();
    while (!mbar_try_wait(bar, parity)) {
        if (global_ns() - t0 > kWaitLimitNs) return false;
    }
    return true;
}

// One tile: the box (64 columns, 16 rows, 2 column halves, K and V) of the
// hot pool's 4-D view, starting at K row `row`.
template <bool kPolicy>
__device__ __forceinline__ void tma_load_tile(uint32_t dst, const CUtensorMap *map, int row,
                                              uint32_t bar, uint64_t policy) {
    if constexpr (!kPolicy) {
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(0), "r"(0), "r"(bar)
            : "memory");
        return;
    }
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        ".L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(row), "r"(0), "r"(0), "r"(bar),
        "l"(policy)
        : "memory");
}

__device__ __forceinline__ void ldsm_x4(uint32_t addr, uint32_t &r0, uint32_t &r1, uint32_t &r2,
                                        uint32_t &r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
                 : "r"(addr));
}

__device__ __forceinline__ void ldsm_x4_t(uint32_t addr, uint32_t &r0, uint32_t &r1,
                                          uint32_t &r2, uint32_t &r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
                 : "r"(addr));
}

// D = A(16x16 bf16, row) * B(16x8 bf16, col) + D, fp32 accumulate.
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
        "{%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t movmatrix_t(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi, float &rlo, float &rhi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    rlo = __low2float(v);
    rhi = __high2float(v);
    return *reinterpret_cast<uint32_t *>(&v);
}

// Byte offset, inside a 16-row x 128-byte box written with the 128-byte
// swizzle, of 16-byte unit `c` (0..7) of row `r`.
__device__ __forceinline__ uint32_t swz(int r, int c) {
    return static_cast<uint32_t>(r * 128 + ((c ^ (r & 7)) << 4));
}

// Offset of a lane's ldmatrix row in a tile, for 16-dim step i of K (A operand
// of S^T, row = token) and of V (A operand of O^T, loaded transposed, row =
// token). Steps i and i + 4 lie one half apart.
__device__ __forceinline__ uint32_t k_offset(int lane, int i) {
    return (i >> 2) * kHalfBytes + swz((lane & 7) + ((lane >> 3) & 1) * 8, 2 * (i & 3) + (lane >> 4));
}
__device__ __forceinline__ uint32_t v_offset(int lane, int i) {
    return (2 + (i >> 2)) * kHalfBytes + swz((lane & 7) + (lane >> 4) * 8, 2 * (i & 3) + ((lane >> 3) & 1));
}

// Slots past T may hold anything (NaN); P is 0 there but 0 * NaN is not, so
// their V rows are cleared.
__device__ __forceinline__ void clear_tail_v(int T, int tok_base, uint8_t *slot, int lane) {
    const int row = T - tok_base + (lane >> 4);   // this lane's rows: row, row + 2, ...
    uint8_t *vp = slot + (2 + ((lane >> 3) & 1)) * kHalfBytes + row * 128 + (lane & 7) * 16;
#pragma unroll
    for (int j = 0; j < kTileTokens / 2; ++j)
        if (row + 2 * j < kTileTokens)
            *reinterpret_cast<uint4 *>(vp + j * 256) = make_uint4(0u, 0u, 0u, 0u);
    __syncwarp();
}

constexpr int kOStride = kHeadDim + 4;   // floats per head row of a state in shared memory (bank skew)
constexpr int kAccFloats = kMaxGroup * kOStride + 2 * kMaxGroup;   // O rows, m[8], l[8]

}  // namespace
}  // namespace kvt
