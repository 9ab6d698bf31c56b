// A stand-in for the CUDA runtime calls and the kernels' launchers that pool.cpp makes, for
// tests/test_pool_setup_host.py: it notes allocations and launches, and calls fail when told to.
#include <cuda_runtime_api.h>
#include <stdlib.h>

#include <map>
#include <vector>

#include "decode_launch.h"
#include "kvt_internal.h"

namespace {
std::map<void *, size_t> live;
std::vector<int64_t> sizes;            // of all allocations, in order
int fail_malloc = 0, turn_status = 0;  // the next cudaMalloc fails; what the turn kernel's preparation returns
cudaError_t last_error = cudaSuccess;
cudaStreamCaptureMode mode = cudaStreamCaptureModeGlobal;
int strict_mallocs = 0;                // allocations while a recording would have forbidden them
int turns = 0, decodes = 0;
const float *turn_part = nullptr;
}  // namespace

extern "C" {
int64_t fake_allocations(int64_t *out, int64_t cap) {
    for (size_t i = 0; i < sizes.size() && static_cast<int64_t>(i) < cap; ++i) out[i] = sizes[i];
    return static_cast<int64_t>(sizes.size());
}
int32_t fake_live() { return static_cast<int32_t>(live.size()); }
void fake_fail_malloc() { fail_malloc = 1; }
void fake_turn_status(int32_t e) { turn_status = e; }
int32_t fake_last_error() { return last_error; }
int32_t fake_turns() { return turns; }
int32_t fake_decodes() { return decodes; }
int32_t fake_has_part() { return turn_part != nullptr; }
int32_t fake_strict_mallocs() { return strict_mallocs; }
int32_t fake_mode() { return mode; }
int64_t part_bytes(int32_t sms) { return kvt::turn_part_floats(sms) * static_cast<int64_t>(sizeof(float)); }

cudaError_t cudaMalloc(void **p, size_t n) {
    if (mode != cudaStreamCaptureModeRelaxed) ++strict_mallocs;
    if (fail_malloc) {
        fail_malloc = 0;
        return last_error = cudaErrorMemoryAllocation;
    }
    *p = malloc(16);   // never read or written
    live[*p] = n;
    sizes.push_back(static_cast<int64_t>(n));
    return cudaSuccess;
}
cudaError_t cudaFree(void *p) {
    if (p && live.erase(p)) free(p);
    return cudaSuccess;
}
cudaError_t cudaThreadExchangeStreamCaptureMode(cudaStreamCaptureMode *m) {
    const cudaStreamCaptureMode was = mode;
    mode = *m;
    *m = was;
    return cudaSuccess;
}
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
cudaError_t cudaEventCreateWithFlags(cudaEvent_t *, unsigned) { return cudaSuccess; }
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaSuccess; }
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaStreamWaitEvent(cudaStream_t, cudaEvent_t, unsigned) { return cudaSuccess; }
}

namespace kvt {
bool encode_hot_tensor_map(CUtensorMap *, void *, int64_t, int64_t, const char **) { return true; }
bool encode_turn_hot_maps(CUtensorMap[2], void *, int64_t, int, const char **) { return true; }
cudaError_t prepare_kernels() { return cudaSuccess; }
cudaError_t prepare_turn_kernel() { return static_cast<cudaError_t>(turn_status); }
int64_t turn_part_floats(int ctas) { return int64_t(1000) * ctas; }
cudaError_t launch_decode(const CUtensorMap &, const DecodeArgs &, int, cudaStream_t, bool) {
    return ++decodes, cudaSuccess;
}
cudaError_t launch_turn(TurnArgs a, const CUtensorMap[2], cudaStream_t) {
    turn_part = a.part;
    return ++turns, cudaSuccess;
}
cudaError_t launch_unpack(MigArgs, int, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_unpack_inline(ResumeArgs &, int, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_pack(MigArgs, int, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_append(AppendArgs, int, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_append_inline(AppendInlineArgs &, int, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_block_jobs(BlockJobs &, bool, int, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_table_write(const TableWriteArgs &, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_gather(const GatherArgs &, cudaStream_t) { return cudaSuccess; }
}  // namespace kvt
