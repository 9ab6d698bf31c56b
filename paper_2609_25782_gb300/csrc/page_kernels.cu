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
template <int kMost>
__global__ void __launch_bounds__(kCopyThreads) copy_jobs_kernel(const __grid_constant__ CopyJobs<kMost> a) {
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

// A CTA per (layer, kv-head) and column of its rows, 256 / kSplit bytes wide, takes the tokens in chunks, in ascending
// order, K and V together (a list's positions and their blocks are looked up once; each alone took 79 us where both
// take 65). Lists ascend, so token t comes from a row at or behind t: a chunk's stores only overwrite rows
// that no later chunk reads, and a barrier keeps them behind the loads of all chunks up to it. A chunk's positions,
// their blocks and their rows are each loaded while the chunk before is at the next of these steps.
constexpr int kCompactThreads = 256;
constexpr int kCompactPerSm = 3;
constexpr int kCompactDeep = 4;                      // rows of a thread in a chunk

template <int kSplit>
__global__ void __launch_bounds__(kCompactThreads, kCompactPerSm) compact_kernel(const __grid_constant__ CompactArgs a) {
    constexpr int kUnits = kRowBytes / 16 / kSplit;  // threads of a row, 16 bytes each
    constexpr int kRows = kCompactThreads / kUnits;
    constexpr int kChunk = kRows * kCompactDeep;
    const Shape sh = a.s;
    const int unit = blockIdx.x / kSplit;            // l * Hkv + g
    const int g = unit % sh.Hkv, l = unit / sh.Hkv;
    const int runs = sh.L * 2 * sh.Hkv, run = l * 2 * sh.Hkv + g;   // of K
    const int32_t *keep = a.keep + l * a.layer_stride + g * a.head_stride;
    const int u = (blockIdx.x % kSplit) * kUnits + threadIdx.x % kUnits;   // 16-byte unit of a row
    const int r0 = threadIdx.x / kUnits;
    const int shift = sh.bt == 16 ? 4 : 6;
    uint4 *base = reinterpret_cast<uint4 *>(a.hot) + u;
    const int64_t values = static_cast<int64_t>(sh.Hkv) << shift << 4;     // from a K row to its V row, in 16 bytes
    auto at = [&](int blk, int t) {                  // the pool has fewer than 2^31 rows
        return base + static_cast<int64_t>(((blk * runs + run) << shift) + (t & (sh.bt - 1))) * (kRowBytes / 16);
    };
    int from[kCompactDeep], before[kCompactDeep];    // positions of the next chunk, and those they have to exceed
    int src[kCompactDeep], dst[kCompactDeep];        // blocks
    uint4 v[kCompactDeep][2];
    uint4 *to[kCompactDeep];                         // places of the chunk that was loaded, or null
    // (Nothing here waits for a value that is loaded: the loads are all on their way before the first is used.)
    auto positions = [&](int t0) {
#pragma unroll
        for (int k = 0; k < kCompactDeep; ++k) {
            const int t = t0 + k * kRows + r0;
            from[k] = t;
            before[k] = t < a.prefix ? t - 1 : a.prefix - 1;
            if (t >= a.prefix && t < a.t_end) from[k] = keep[t - a.prefix];
            if (t > a.prefix && t < a.t_end) before[k] = keep[t - a.prefix - 1];
        }
    };
    positions(a.t_begin);
#pragma unroll
    for (int k = 0; k < kCompactDeep; ++k) to[k] = nullptr;
#pragma unroll 1
    for (int t0 = a.t_begin;; t0 += kChunk) {
        bool ok[kCompactDeep];
        bool bad = false;
#pragma unroll
        for (int k = 0; k < kCompactDeep; ++k) {
            const int t = t0 + k * kRows + r0;
            // (from >= t is what the order of loads and stores rests on.)
            const bool good = from[k] < a.T && from[k] >= t && from[k] > before[k];
            ok[k] = t < a.t_end && good;
            bad |= t < a.t_end && !good;
            src[k] = ok[k] ? a.table[from[k] >> shift] : -1;
            dst[k] = ok[k] ? (a.fresh ? a.slot[(t >> shift) - a.fresh_at] : -1) : -1;
            if (ok[k] && dst[k] < 0) dst[k] = a.table[t >> shift];
        }
        if (bad && u == 0) atomicOr(a.err, kErrBadIndex);
        int row[kCompactDeep];
#pragma unroll
        for (int k = 0; k < kCompactDeep; ++k) row[k] = from[k];
        positions(t0 + kChunk);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kCompactDeep; ++k)
            if (to[k] != nullptr) {
                *to[k] = v[k][0];
                to[k][values] = v[k][1];
            }
        if (t0 >= a.t_end) return;
        bad = false;
#pragma unroll
        for (int k = 0; k < kCompactDeep; ++k) {
            const bool in = src[k] >= 0 && src[k] < sh.num_blocks && dst[k] >= 0 && dst[k] < sh.num_blocks;
            bad |= ok[k] && !in;
            ok[k] = ok[k] && in;
            to[k] = ok[k] ? at(dst[k], t0 + k * kRows + r0) : nullptr;
            if (ok[k]) {
                const uint4 *x = at(src[k], row[k]);
                v[k][0] = *x;
                v[k][1] = x[values];
            }
        }
        if (bad && u == 0) atomicOr(a.err, kErrBadBlock);
    }
}

}  // namespace

template <int kMost>
cudaError_t launch_copy_jobs(const CopyJobs<kMost> &a, int max_ctas, cudaStream_t st) {
    if (a.n <= 0 && (a.shared <= 0 || a.children <= 0)) return cudaSuccess;
    const int64_t items = static_cast<int64_t>(a.n) * a.s.L * 2 * a.s.Hkv * (a.s.bt / kChunkRows);
    const int64_t entries = (a.shared + 31) / 32;
    copy_jobs_kernel<kMost><<<item_grid(items > entries ? items : entries, max_ctas), kCopyThreads, 0, st>>>(a);
    return cudaGetLastError();
}
template cudaError_t launch_copy_jobs(const CopyJobs<kCopyJobsFew> &, int, cudaStream_t);
template cudaError_t launch_copy_jobs(const CopyJobs<kCopyJobsMax> &, int, cudaStream_t);

template <int kSplit>
static void start_compact(const CompactArgs &a, cudaStream_t st) {
    compact_kernel<kSplit><<<a.s.L * a.s.Hkv * kSplit, kCompactThreads, 0, st>>>(a);
}

cudaError_t launch_compact(const CompactArgs &a, int num_sms, cudaStream_t st) {
    if (a.t_end <= a.t_begin) return cudaSuccess;
    // The narrowest columns whose CTAs are all resident: one chunk after another is a chain. us by columns 1, 2, 4 and 8:
    // 192 units (48 layers, 4 heads), 2 040 tokens kept of 8 200: -, 65, 68, 85; 128 units (64-token blocks, one of three
    // calls) 47, 30, 33, 34; 112 units, 14 000 of 24 000: 529, 315, 249, 298; 64 units, 8 100 of 9 000: 264, 158, 104,
    // 124; 16 units, 2 700 of 9 000: 63, 29, 17, 12.
    const int64_t units = static_cast<int64_t>(a.s.L) * a.s.Hkv, fit = static_cast<int64_t>(kCompactPerSm) * num_sms;
    if (units * 8 <= fit) start_compact<8>(a, st);
    else if (units * 4 <= fit) start_compact<4>(a, st);
    else if (units * 2 <= fit) start_compact<2>(a, st);
    else start_compact<1>(a, st);
    return cudaGetLastError();
}

}  // namespace kvt
