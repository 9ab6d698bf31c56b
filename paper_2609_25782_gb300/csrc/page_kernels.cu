// Kernels of forks and compactions, for sm_103a.
//
//   copy_jobs_kernel  rows of a block into another block of the pool (a fork's partly filled block; in
//                     residency mode all of a fork's blocks), with the table entries that name them
//   compact_kernel    the kept rows of a session towards its front, in place
#include <cstdint>

#include "cache_ops.h"

namespace kvt {
namespace {

constexpr int kChunkRows = 8;        // rows that a warp moves at a time, 2 KiB

// One warp per chunk of a (job, layer, K|V, kv-head) run, as migrations move them: 16 bytes a lane, four loads
// in flight. Bound by HBM where jobs are many.
__global__ void __launch_bounds__(kCopyThreads) copy_jobs_kernel(const __grid_constant__ CopyJobs a) {
    const Shape sh = a.s;
    const int nthreads = gridDim.x * blockDim.x;
    const int thread = blockIdx.x * blockDim.x + threadIdx.x;
    // The children's first entries. A child's row and its parent's are different memory.
    const int32_t *from = a.tables + static_cast<int64_t>(a.parent) * a.table_stride;
    for (int c = 0; c < a.children; ++c) {
        int32_t *row = a.tables + static_cast<int64_t>(a.child[c]) * a.table_stride;
        for (int j = thread; j < a.shared; j += nthreads) row[j] = from[j];
    }
    const int runs = sh.L * 2 * sh.Hkv;
    const int chunks = sh.bt / kChunkRows;
    const int64_t items = static_cast<int64_t>(a.n) * runs * chunks;
    const int lane = threadIdx.x & 31;
    const int nwarps = nthreads >> 5;
    for (int64_t it = thread >> 5; it < items; it += nwarps) {
        const int jb = static_cast<int>(it / (runs * chunks));
        const int rem = static_cast<int>(it - static_cast<int64_t>(jb) * runs * chunks);
        const int c = rem / chunks;
        const int r0 = (rem - c * chunks) * kChunkRows;
        const CopyJob &b = a.job[jb];
        if (b.from < 0 || b.from >= sh.num_blocks || b.to < 0 || b.to >= sh.num_blocks) {
            if (lane == 0 && rem == 0) atomicOr(a.err, kErrBadBlock);
            continue;
        }
        if (rem == 0 && lane == 0) a.tables[static_cast<int64_t>(b.sid) * a.table_stride + b.j] = b.to;
        const int units = (min(b.rows, r0 + kChunkRows) - r0) * (kRowBytes / 16) - lane;
        const int64_t at = (static_cast<int64_t>(c) * sh.bt + r0) * kRowBytes;
        const int64_t block = static_cast<int64_t>(runs) * sh.bt * kRowBytes;
        const uint4 *src = reinterpret_cast<const uint4 *>(a.hot + b.from * block + at) + lane;
        uint4 *dst = reinterpret_cast<uint4 *>(a.hot + b.to * block + at) + lane;
        uint4 v[kChunkRows / 2];
#pragma unroll
        for (int k = 0; k < kChunkRows / 2; ++k)
            if (k * 32 < units) v[k] = src[k * 32];
#pragma unroll
        for (int k = 0; k < kChunkRows / 2; ++k)
            if (k * 32 < units) dst[k * 32] = v[k];
    }
}

// A CTA per (layer, K|V, kv-head) run takes its tokens in chunks, in ascending order. Lists ascend, so token t
// comes from a row at or behind t: a chunk's stores only overwrite rows that no later chunk reads, and the
// barriers keep them behind the chunk's own loads.
constexpr int kCompactThreads = 256;
constexpr int kCompactRows = 64;

__global__ void __launch_bounds__(kCompactThreads) compact_kernel(const __grid_constant__ CompactArgs a) {
    const Shape sh = a.s;
    const int run = blockIdx.x;                      // (l * 2 + kv) * Hkv + g
    const int runs = sh.L * 2 * sh.Hkv;
    const int g = run % sh.Hkv;
    const int l = run / (2 * sh.Hkv);
    const int32_t *keep = a.keep + l * a.layer_stride + g * a.head_stride;
    const int u = threadIdx.x & 15;                  // 16-byte unit of a row
    const int r0 = threadIdx.x >> 4;
    auto row_of = [&](int blk, int t, int j) {
        return (static_cast<int64_t>(blk) * runs + run) * sh.bt + (t - j * sh.bt);
    };
    for (int t0 = a.t_begin; t0 < a.t_end; t0 += kCompactRows) {
        uint4 v[kCompactRows / 16];
        uint4 *to[kCompactRows / 16];
#pragma unroll
        for (int k = 0; k < kCompactRows / 16; ++k) {
            const int t = t0 + k * 16 + r0;
            to[k] = nullptr;
            if (t >= a.t_end) continue;
            int from = t;
            if (t >= a.prefix) {
                from = keep[t - a.prefix];
                const int before = t > a.prefix ? keep[t - a.prefix - 1] : a.prefix - 1;
                // (from >= t is what the order of loads and stores rests on.)
                if (from >= a.T || from < t || from <= before) {
                    if (u == 0) atomicOr(a.err, kErrBadIndex);
                    continue;
                }
            }
            const int js = from / sh.bt, jd = t / sh.bt;
            const int bs = a.table[js];
            int bd = a.fresh ? a.slot[jd - a.fresh_at] : -1;
            if (bd < 0) bd = a.table[jd];
            if (bs < 0 || bs >= sh.num_blocks || bd < 0 || bd >= sh.num_blocks) {
                if (u == 0) atomicOr(a.err, kErrBadBlock);
                continue;
            }
            v[k] = reinterpret_cast<const uint4 *>(a.hot + row_of(bs, from, js) * kRowBytes)[u];
            to[k] = reinterpret_cast<uint4 *>(a.hot + row_of(bd, t, jd) * kRowBytes) + u;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kCompactRows / 16; ++k)
            if (to[k] != nullptr) *to[k] = v[k];
        __syncthreads();
    }
}

}  // namespace

cudaError_t launch_copy_jobs(const CopyJobs &a, int max_ctas, cudaStream_t st) {
    if (a.n <= 0 && (a.shared <= 0 || a.children <= 0)) return cudaSuccess;
    const int64_t items = static_cast<int64_t>(a.n) * a.s.L * 2 * a.s.Hkv * (a.s.bt / kChunkRows);
    const int64_t entries = (a.shared + 31) / 32;
    copy_jobs_kernel<<<item_grid(items > entries ? items : entries, max_ctas), kCopyThreads, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_compact(const CompactArgs &a, int, cudaStream_t st) {
    if (a.t_end <= a.t_begin) return cudaSuccess;
    compact_kernel<<<a.s.L * 2 * a.s.Hkv, kCompactThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace kvt
