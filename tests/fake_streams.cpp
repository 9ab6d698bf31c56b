// A stand-in for the CUDA runtime calls and the kernels' launchers that pool.cpp, pages.cpp and sparse.cpp make, for
// tests/test_page_order_host.py: it notes launches, event records and waits by stream, in their order, and calls fail
// when told to.
#include <cuda_runtime_api.h>

#include <vector>

#include "cache_ops.h"
#include "decode_launch.h"
#include "kvt_internal.h"

namespace {
enum { kLaunch = 1, kRecord = 2, kWait = 3, kHostWait = 4 };
struct Entry {
    int64_t what, stream, event;
};
std::vector<Entry> calls;
int64_t made = 0, alive = 0;           // events
int fail_create = 0;                   // the n-th event creation from now on fails
int prepare_status = 0;                // what the kernels' preparation returns
cudaError_t last_error = cudaSuccess;

int64_t id(const void *x) { return static_cast<int64_t>(reinterpret_cast<uintptr_t>(x)); }
cudaError_t note(int what, const void *stream, const void *event) {
    calls.push_back({what, id(stream), id(event)});
    return cudaSuccess;
}
cudaError_t launch(cudaStream_t st) { return note(kLaunch, st, nullptr); }
}  // namespace

extern "C" {
int64_t fake_calls(int64_t *out, int64_t cap) {
    for (size_t i = 0; i < calls.size() && static_cast<int64_t>(i) < cap; ++i) {
        out[3 * i] = calls[i].what;
        out[3 * i + 1] = calls[i].stream;
        out[3 * i + 2] = calls[i].event;
    }
    const int64_t n = static_cast<int64_t>(calls.size());
    calls.clear();
    return n;
}
int64_t fake_events() { return alive; }
void fake_fail_create(int32_t n) { fail_create = n; }
void fake_prepare_status(int32_t e) { prepare_status = e; }
int32_t fake_last_error() { return last_error; }

cudaError_t cudaMalloc(void **p, size_t) { return *p = reinterpret_cast<void *>(uintptr_t(1) << 40), cudaSuccess; }
cudaError_t cudaFree(void *) { return cudaSuccess; }
cudaError_t cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode *) { return cudaSuccess; }
cudaError_t cudaGetLastError() {
    const cudaError_t e = last_error;
    last_error = cudaSuccess;
    return e;
}
const char *cudaGetErrorString(cudaError_t) { return "fake"; }
cudaError_t cudaMemset(void *, int, size_t) { return cudaSuccess; }
cudaError_t cudaMemcpy(void *, const void *, size_t, cudaMemcpyKind) { return cudaSuccess; }
cudaError_t cudaGetDevice(int *d) { return *d = 0, cudaSuccess; }
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
cudaError_t cudaDeviceSynchronize() { return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int *x, cudaDeviceAttr, int) { return *x = 152, cudaSuccess; }
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *ev, unsigned) {
    if (fail_create > 0 && --fail_create == 0) return last_error = cudaErrorMemoryAllocation;
    ++alive;
    *ev = reinterpret_cast<cudaEvent_t>(static_cast<uintptr_t>(++made));
    return cudaSuccess;
}
cudaError_t cudaEventDestroy(cudaEvent_t) { return --alive, cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t ev, cudaStream_t st) { return note(kRecord, st, ev); }
cudaError_t cudaEventSynchronize(cudaEvent_t ev) { return note(kHostWait, nullptr, ev); }
cudaError_t cudaStreamWaitEvent(cudaStream_t st, cudaEvent_t ev, unsigned) { return note(kWait, st, ev); }
}

namespace kvt {
bool encode_hot_tensor_map(CUtensorMap *, void *, int64_t, int64_t, const char **) { return true; }
bool encode_turn_hot_maps(CUtensorMap[2], void *, int64_t, int, const char **) { return true; }
cudaError_t prepare_kernels() { return cudaSuccess; }
cudaError_t prepare_turn_kernel() { return cudaSuccess; }
int64_t turn_part_floats(int ctas) { return int64_t(1000) * ctas; }
cudaError_t launch_decode(const CUtensorMap &, const DecodeArgs &, int, cudaStream_t st, bool) { return launch(st); }
cudaError_t launch_turn(TurnArgs, const CUtensorMap[2], cudaStream_t st) { return launch(st); }
cudaError_t launch_unpack(MigArgs, int, cudaStream_t st) { return launch(st); }
cudaError_t launch_unpack_inline(ResumeArgs &, int, cudaStream_t st) { return launch(st); }
cudaError_t launch_pack(MigArgs, int, cudaStream_t st) { return launch(st); }
cudaError_t launch_append(AppendArgs, int, cudaStream_t st) { return launch(st); }
cudaError_t launch_append_inline(AppendInlineArgs &, int, cudaStream_t st) { return launch(st); }
cudaError_t launch_block_jobs(BlockJobs &, bool, int, cudaStream_t st) { return launch(st); }
cudaError_t launch_table_write(const TableWriteArgs &, cudaStream_t st) { return launch(st); }
cudaError_t launch_gather(const GatherArgs &, cudaStream_t st) { return launch(st); }
cudaError_t launch_compact(const CompactArgs &, int, cudaStream_t st) { return launch(st); }
template <int kMost>
cudaError_t launch_copy_jobs(const CopyJobs<kMost> &, int, cudaStream_t st) { return launch(st); }
template cudaError_t launch_copy_jobs(const CopyJobs<kCopyJobsFew> &, int, cudaStream_t);
template cudaError_t launch_copy_jobs(const CopyJobs<kCopyJobsMax> &, int, cudaStream_t);
cudaError_t launch_bounds(const BoundsArgs &, int, cudaStream_t st) { return launch(st); }
cudaError_t prepare_select_kernel(SelectFit *) { return last_error = static_cast<cudaError_t>(prepare_status); }
cudaError_t launch_select(const SelectArgs &, const SelectFit &, cudaStream_t st) { return launch(st); }
cudaError_t prepare_sparse_kernels(SparseFit *) { return last_error = static_cast<cudaError_t>(prepare_status); }
cudaError_t launch_sparse(const CUtensorMap &, const SparseArgs &, const SparseFit &, cudaStream_t st) { return launch(st); }
}  // namespace kvt
