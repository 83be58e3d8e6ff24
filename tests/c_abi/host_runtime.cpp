// The part of the CUDA runtime that the library's host files call, over host memory: compiled with them, it lets a test drive
// handles and argument checks without a GPU and see what they would have asked of one, in order. Kernel launches are
// only counted. "Device" pointers are host pointers.
#include <cuda_runtime.h>

#include <cstring>
#include <string>

#include "speca_internal.h"
#include "speca_layer_internal.h"

namespace {
std::string events;  // one letter per call: S wait for the device, C copy, M set, L launch
int current = 0;
cudaError_t note(char e) {
    events.push_back(e);
    return cudaSuccess;
}
}  // namespace

extern "C" {
const char* host_events() { return events.c_str(); }
void host_events_clear() { events.clear(); }

cudaError_t cudaGetDeviceCount(int* n) {
    *n = 2;
    return cudaSuccess;
}
cudaError_t cudaGetDevice(int* d) {
    *d = current;
    return cudaSuccess;
}
cudaError_t cudaSetDevice(int d) {
    current = d;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int) {
    *v = a == cudaDevAttrComputeCapabilityMajor ? 10 : a == cudaDevAttrMultiProcessorCount ? 148 : 0;
    return cudaSuccess;
}
cudaError_t cudaDeviceSynchronize() { return note('S'); }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return note('S'); }
cudaError_t cudaMemcpy(void* d, const void* s, size_t n, cudaMemcpyKind) {
    std::memcpy(d, s, n);
    return note('C');
}
cudaError_t cudaMemcpyAsync(void* d, const void* s, size_t n, cudaMemcpyKind k, cudaStream_t) { return cudaMemcpy(d, s, n, k); }
cudaError_t cudaMemset(void* d, int v, size_t n) {
    std::memset(d, v, n);
    return note('M');
}
cudaError_t cudaMemsetAsync(void* d, int v, size_t n, cudaStream_t) { return cudaMemset(d, v, n); }
cudaError_t cudaGetLastError() { return cudaSuccess; }
const char* cudaGetErrorString(cudaError_t) { return "error"; }
}

namespace speca {
cudaError_t launch_modulate(const ModulateParams&, int, int, cudaStream_t) { return note('L'); }
cudaError_t launch_rope(const RopeParams&, int, bool, cudaStream_t) { return note('L'); }
cudaError_t launch_attention_f32(const AttnParams&, cudaStream_t) { return note('L'); }
cudaError_t launch_attention_bf16(const AttnParams&, int64_t, int, cudaStream_t) { return note('L'); }
cudaError_t launch_attention_join(const AttnParams&, int, cudaStream_t) { return cudaSuccess; }
// of the cache's kernels only what creating a handle asks for; the rest is never reached (bound lazily)
uint32_t stream_tile_bytes(int, bool) { return kTileSizes[0]; }
int max_resident_verify_clusters(int, int, int) { return 1; }
}  // namespace speca
