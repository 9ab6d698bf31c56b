// Internal interface of the calls on parts of the cache: sparse.cpp with sparse_kernels.cu (bounds of blocks,
// selection) and attend_kernels.cu (attention over listed blocks), pages.cpp with page_kernels.cu (forks,
// compaction).
#pragma once

#include "kvt_internal.h"

namespace kvt {

constexpr int32_t kErrBadIndex = 16;   // a kept position out of range or out of order

constexpr int kCodeRow = 2 * kHeadDim;          // a block's codes of one layer and kv-head: hi, then lo
constexpr int kBoundsRowsMax = 4096;            // rows of a bounds call, planned in shared memory
constexpr int kSelectBlocksMax = 49152;         // blocks of a row, whose keys lie in one CTA's shared memory

struct BoundsArgs {
    const uint16_t *hot;
    const int32_t *tables;    // [B][max_blocks]
    const int32_t *seq_lens;  // [B]
    const int32_t *since;     // [B] or null
    int8_t *codes;            // [L][Hkv][num_blocks][2][D]
    uint16_t *steps;          // [L][Hkv][num_blocks] bf16
    int32_t *err;
    int32_t B, max_blocks, layer0, nlayers;
    Shape s;
};

struct SelectArgs {
    const uint16_t *q;        // [B][Hq][D] bf16, q_stride elements from row to row
    const int8_t *codes;      // of the layer: [Hkv][num_blocks][2][D]
    const uint16_t *steps;    // of the layer: [Hkv][num_blocks]
    const int32_t *tables;
    const int32_t *seq_lens;
    int32_t *selected;        // [B][Hkv][top]
    float *scores;            // [B][Hkv][max_blocks] or null
    int32_t *err;
    int64_t q_stride;
    int32_t B, max_blocks, first, last, top;
    int32_t group;            // Hq / Hkv
    Shape s;
};

struct SparseArgs {
    const uint16_t *q;        // [B][Hq][D] bf16, q_stride elements from row to row
    const uint16_t *k_new, *v_new;   // [B][Hkv][D] bf16, kv_stride elements from row to row, or null
    const int32_t *selected;  // [B][Hkv][top]
    const int32_t *tables;
    const int32_t *seq_lens;
    void *out;                // [B][Hq][D], fp32 or (out_bf16) bf16
    uint16_t *hot;
    int32_t *err;
    int64_t q_stride, kv_stride;
    int32_t B, max_blocks, layer, top, out_bf16;
    int32_t group;            // Hq / Hkv
    float scale_log2;         // scale * log2(e)
    int32_t inject_extra_tx;  // test hook: extra bytes expected on one tile (0 normally)
    Shape s;
};

// Copies of a block's first rows within the pool, which also become entry j of a session's table row.
struct CopyJob {
    int32_t from, to;         // slots
    int32_t sid, j;
    int32_t rows;
};
constexpr int kCopyJobsMax = 1300;   // keeps the parameter block under 32 KB
constexpr int kCopyJobsFew = 24;     // and a small fork's under 1 KB
template <int kMost>
struct CopyJobs {
    uint8_t *hot;
    int32_t *err;
    int32_t *tables;          // the pool's table arena
    int64_t table_stride;
    Shape s;
    int32_t n;
    // Sessions whose first `shared` table entries become those of `parent` (of any launch, one does it).
    int32_t parent, shared, children;
    CopyJob job[kMost];
    int32_t child[kMost];
};

// Rows of a session that move towards its front: token t of [t_begin, t_end) of layer l and kv-head g is the old
// token keep[l * layer_stride + g * head_stride + t - prefix], or t itself where t < prefix.
constexpr int kCompactFresh = 2048;  // new blocks that a launch names
struct CompactArgs {
    uint8_t *hot;
    int32_t *err;
    const int32_t *table;     // the session's row: where rows come from
    const int32_t *keep;
    int64_t layer_stride, head_stride;
    int32_t t_begin, t_end, prefix, T;
    // Where rows go: the table's blocks, or (fresh) block fresh_at + i is slot[i].
    int32_t fresh, fresh_at;
    Shape s;
    int32_t slot[kCompactFresh];
};

cudaError_t launch_bounds(const BoundsArgs &a, int num_sms, cudaStream_t st);
cudaError_t prepare_select_kernel(SelectFit *fit);
cudaError_t launch_select(const SelectArgs &a, const SelectFit &fit, cudaStream_t st);
cudaError_t prepare_sparse_kernels(SparseFit *fit);
cudaError_t launch_sparse(const CUtensorMap &map, const SparseArgs &a, const SparseFit &fit, cudaStream_t st);
template <int kMost>
cudaError_t launch_copy_jobs(const CopyJobs<kMost> &a, int max_ctas, cudaStream_t st);
cudaError_t launch_compact(const CompactArgs &a, int num_sms, cudaStream_t st);

}  // namespace kvt
