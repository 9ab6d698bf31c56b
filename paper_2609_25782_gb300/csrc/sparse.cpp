// Attention over a part of the cache (include/kvtier.h): bounds of blocks' keys, the selection of blocks from
// them, and attention over the selected ones. Kernels in sparse_kernels.cu and attend_kernels.cu.
#include <cmath>

#include "cache_ops.h"
#include "pool_state.h"

using kvt::DeviceGuard;
using kvt::fail;

namespace {

int64_t bounds_records(const kv_pool_config &c) {
    return static_cast<int64_t>(c.num_layers) * c.num_kv_heads * c.num_hot_blocks;
}

uintptr_t bits(const void *x) { return reinterpret_cast<uintptr_t>(x); }

// The arguments that the three calls share.
int check_rows(const kv_pool *p, int32_t layer, bool all_layers, const int32_t *block_tables,
               const int32_t *seq_lens, int32_t B, int32_t max_blocks) {
    if (!block_tables || !seq_lens) return fail(KV_ERR_INVALID_ARG, "null pointer");
    if ((bits(block_tables) | bits(seq_lens)) & 3)
        return fail(KV_ERR_INVALID_ARG, "block_tables and seq_lens need 4-byte alignment");
    if (layer < (all_layers ? -1 : 0) || layer >= p->cfg.num_layers) return fail(KV_ERR_INVALID_ARG, "bad layer");
    if (B < 1 || B > 65535) return fail(KV_ERR_INVALID_ARG, "B out of range");
    if (max_blocks < 1 || max_blocks > (1 << 26))
        return fail(KV_ERR_INVALID_ARG, "max_blocks out of range");
    return KV_OK;
}

// A pool's first call of a kind prepares its kernels. The call may be one that a graph records; the preparation is no
// part of the recording.
template <typename F>
int prepare(kv_pool *p, bool *ready, const char *what, F &&fn) {
    if (*ready) return KV_OK;
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    cudaThreadExchangeStreamCaptureMode(&mode);
    const int rc = p->cuda(what, fn);
    cudaThreadExchangeStreamCaptureMode(&mode);
    *ready = !rc;
    return rc;
}

int check_stride(int64_t *stride, int64_t row) {
    if (*stride == 0) *stride = row;
    if (*stride < row || *stride & 7 || *stride > (int64_t(1) << 32))
        return fail(KV_ERR_INVALID_ARG, "row strides must be multiples of 8 and hold a row's heads");
    return KV_OK;
}

}  // namespace

extern "C" {

int64_t kv_bounds_bytes(const kv_pool_config *c) {
    return c ? bounds_records(*c) * (kvt::kCodeRow + 2) : 0;
}

int kv_pool_block_bounds(kv_pool *p, int32_t layer, const int32_t *block_tables,
                         const int32_t *seq_lens, const int32_t *since, int32_t B,
                         int32_t max_blocks, void *bounds, kv_stream_t stream) {
    if (!p) return fail(KV_ERR_INVALID_ARG, "null pool");
    int rc = check_rows(p, layer, true, block_tables, seq_lens, B, max_blocks);
    if (rc) return rc;
    if (!bounds || bits(bounds) & 255) return fail(KV_ERR_INVALID_ARG, "bounds must be 256-byte aligned");
    if (bits(since) & 3) return fail(KV_ERR_INVALID_ARG, "since needs 4-byte alignment");
    if (B > kvt::kBoundsRowsMax || static_cast<int64_t>(B) * max_blocks > (1 << 30))
        return fail(KV_ERR_INVALID_ARG, "B out of range");
    if (p->host_only) return fail(KV_ERR_BAD_STATE, "bounds on a host-logic-only pool");
    DeviceGuard dg(p->cfg.device, true);
    kvt::BoundsArgs a;
    a.hot = static_cast<const uint16_t *>(p->cfg.hot_base);
    a.tables = block_tables;
    a.seq_lens = seq_lens;
    a.since = since;
    a.codes = static_cast<int8_t *>(bounds);
    a.steps = reinterpret_cast<uint16_t *>(a.codes + bounds_records(p->cfg) * kvt::kCodeRow);
    a.err = p->d_err;
    a.B = B;
    a.max_blocks = max_blocks;
    a.layer0 = layer < 0 ? 0 : layer;
    a.nlayers = layer < 0 ? p->cfg.num_layers : 1;
    a.s = p->shape;
    return p->cuda("bounds launch", [&] {
        return kvt::launch_bounds(a, p->num_sms, reinterpret_cast<cudaStream_t>(stream));
    });
}

int select_blocks(kv_pool *p, int32_t layer, const void *q, int64_t q_stride, const void *bounds,
                  const int32_t *block_tables, const int32_t *seq_lens, int32_t B, int32_t max_blocks,
                  int32_t first, int32_t last, int32_t top, int32_t *selected, float *scores,
                  kv_stream_t stream) {
    if (!p) return fail(KV_ERR_INVALID_ARG, "null pool");
    int rc = check_rows(p, layer, false, block_tables, seq_lens, B, max_blocks);
    if (rc) return rc;
    if (!q || !bounds || !selected) return fail(KV_ERR_INVALID_ARG, "null pointer");
    if (bits(q) & 15 || bits(bounds) & 255)
        return fail(KV_ERR_INVALID_ARG, "q needs 16-byte, bounds 256-byte alignment");
    if ((bits(selected) | bits(scores)) & 3)
        return fail(KV_ERR_INVALID_ARG, "selected and scores need 4-byte alignment");
    if (max_blocks > kvt::kSelectBlocksMax) return fail(KV_ERR_INVALID_ARG, "max_blocks above 49152");
    if (first < 0 || last < 0 || top < 1 || first > top || last > top - first)
        return fail(KV_ERR_INVALID_ARG, "need first, last >= 0, top >= 1 and first + last <= top");
    rc = check_stride(&q_stride, static_cast<int64_t>(p->cfg.num_q_heads) * kvt::kHeadDim);
    if (rc) return rc;
    if (p->host_only) return fail(KV_ERR_BAD_STATE, "selection on a host-logic-only pool");
    DeviceGuard dg(p->cfg.device, true);
    rc = prepare(p, &p->select_ready, "kernels of the selection", [&] { return kvt::prepare_select_kernel(&p->select_fit); });
    if (rc) return rc;
    const int64_t layer_records = static_cast<int64_t>(layer) * p->cfg.num_kv_heads * p->cfg.num_hot_blocks;
    kvt::SelectArgs a;
    a.q = static_cast<const uint16_t *>(q);
    a.codes = static_cast<const int8_t *>(bounds) + layer_records * kvt::kCodeRow;
    a.steps = reinterpret_cast<const uint16_t *>(static_cast<const int8_t *>(bounds) +
                                                 bounds_records(p->cfg) * kvt::kCodeRow) + layer_records;
    a.tables = block_tables;
    a.seq_lens = seq_lens;
    a.selected = selected;
    a.scores = scores;
    a.err = p->d_err;
    a.q_stride = q_stride;
    a.B = B;
    a.max_blocks = max_blocks;
    a.first = first;
    a.last = last;
    a.top = top;
    a.group = p->cfg.num_q_heads / p->cfg.num_kv_heads;
    a.s = p->shape;
    return p->cuda("selection launch", [&] {
        return kvt::launch_select(a, p->select_fit, reinterpret_cast<cudaStream_t>(stream));
    });
}

int sparse_attention(kv_pool *p, int32_t layer, const void *q, int64_t q_stride, const void *k_new,
                     const void *v_new, int64_t kv_stride, const int32_t *selected, int32_t top,
                     const int32_t *block_tables, const int32_t *seq_lens, int32_t B, int32_t max_blocks,
                     float scale, void *out, uint32_t flags, kv_stream_t stream) {
    if (flags & ~static_cast<uint32_t>(KV_DECODE_OUT_BF16)) return fail(KV_ERR_INVALID_ARG, "unknown flag");
    if (!p) return fail(KV_ERR_INVALID_ARG, "null pool");
    int rc = check_rows(p, layer, false, block_tables, seq_lens, B, max_blocks);
    if (rc) return rc;
    if (!q || !selected || !out) return fail(KV_ERR_INVALID_ARG, "null pointer");
    if (!k_new != !v_new) return fail(KV_ERR_INVALID_ARG, "k_new and v_new come together");
    if ((bits(q) | bits(k_new) | bits(v_new) | bits(out)) & 15)
        return fail(KV_ERR_INVALID_ARG, "q, k_new, v_new and out must be 16-byte aligned");
    if (bits(selected) & 3) return fail(KV_ERR_INVALID_ARG, "selected needs 4-byte alignment");
    if (top < 1 || top > (1 << 26)) return fail(KV_ERR_INVALID_ARG, "top out of range");
    rc = check_stride(&q_stride, static_cast<int64_t>(p->cfg.num_q_heads) * kvt::kHeadDim);
    if (!rc) rc = check_stride(&kv_stride, static_cast<int64_t>(p->cfg.num_kv_heads) * kvt::kHeadDim);
    if (rc) return rc;
    const float scale_log2 = scale * 1.4426950408889634f;
    if (!std::isfinite(scale_log2)) return fail(KV_ERR_INVALID_ARG, "scale not finite, or above 2^127");
    if (p->host_only) return fail(KV_ERR_BAD_STATE, "attention on a host-logic-only pool");
    DeviceGuard dg(p->cfg.device, true);
    rc = prepare(p, &p->sparse_ready, "kernels of sparse attention", [&] { return kvt::prepare_sparse_kernels(&p->sparse_fit); });
    if (rc) return rc;
    kvt::SparseArgs a;
    a.q = static_cast<const uint16_t *>(q);
    a.k_new = static_cast<const uint16_t *>(k_new);
    a.v_new = static_cast<const uint16_t *>(v_new);
    a.selected = selected;
    a.tables = block_tables;
    a.seq_lens = seq_lens;
    a.out = out;
    a.hot = static_cast<uint16_t *>(p->cfg.hot_base);
    a.err = p->d_err;
    a.q_stride = q_stride;
    a.kv_stride = kv_stride;
    a.B = B;
    a.max_blocks = max_blocks;
    a.layer = layer;
    a.top = top;
    a.group = p->cfg.num_q_heads / p->cfg.num_kv_heads;
    a.out_bf16 = (flags & KV_DECODE_OUT_BF16) ? 1 : 0;
    a.scale_log2 = scale_log2;
    a.inject_extra_tx = p->inject_timeout ? 16 : 0;
    a.s = p->shape;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    rc = p->cuda("attention launch", [&] { return kvt::launch_sparse(p->tmap, a, p->sparse_fit, st); });
    if (rc) return rc;
    p->inject_timeout = false;
    p->decoded = true;
    p->decode_stream = st;
    return KV_OK;
}

}  // extern "C"
