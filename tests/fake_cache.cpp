// A CUDA runtime for host tests of the paged cache's host side, linked with its object
// in place of libcudart and of the kernels' launch functions.  "Device" memory is host
// memory.  Fills, copies and launches wait in their stream until something makes the
// host wait for it: no stream waits for another (as non-blocking streams do not, nor
// they for the legacy one).
#include <cuda.h>
#include <cuda_runtime_api.h>

#include <cstdlib>
#include <cstring>
#include <deque>
#include <functional>
#include <map>
#include <string>

namespace {

std::map<cudaStream_t, std::deque<std::function<void()>>> queued;
int* error_word = nullptr;                       // what the host reads one int of
int* base = nullptr;                             // what lengths are copied to

void run(cudaStream_t s) {
    auto& q = queued[s];
    while (!q.empty()) {
        q.front()();
        q.pop_front();
    }
}
cudaError_t put(cudaStream_t s, std::function<void()> f) {
    queued[s].push_back(f);
    return cudaSuccess;
}
CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    return CUDA_SUCCESS;
}

}  // namespace

// Questions and orders of a test.
extern "C" {
void fake_reset() { queued.clear(); }
void fake_fill(void* st, int* at, int n, int value) {
    put((cudaStream_t)st, [=] { for (int i = 0; i < n; ++i) at[i] = value; });
}
void fake_finish() {
    for (auto& q : queued) run(q.first);
}
void fake_flag_error(int code) { *error_word = code; }       // by a kernel that runs at once
int fake_base(int seq) { return base[seq]; }
}

// The runtime calls that the host object makes.
extern "C" {
cudaError_t cudaGetLastError() { return cudaSuccess; }
const char* cudaGetErrorString(cudaError_t) { return "error"; }
cudaError_t cudaGetDevice(int* d) { return *d = 0, cudaSuccess; }
cudaError_t cudaSetDevice(int) { return cudaSuccess; }
cudaError_t cudaGetDeviceProperties(cudaDeviceProp* p, int) {
    std::memset(p, 0, sizeof *p);
    p->major = 10;
    p->minor = 3;
    p->multiProcessorCount = 152;
    return cudaSuccess;
}
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** fn, unsigned, unsigned long long,
                                             cudaDriverEntryPointQueryResult* q) {
    *fn = reinterpret_cast<void*>(encode);
    *q = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
cudaError_t cudaMalloc(void** p, size_t n) { return *p = std::calloc(1, n), cudaSuccess; }
cudaError_t cudaFree(void* p) { return std::free(p), cudaSuccess; }
cudaError_t cudaMemsetAsync(void* d, int v, size_t n, cudaStream_t s) {
    return put(s, [=] { std::memset(d, v, n); });
}
cudaError_t cudaMemset(void* d, int v, size_t n) { return cudaMemsetAsync(d, v, n, nullptr); }
cudaError_t cudaMemcpyAsync(void* d, const void* s, size_t n, cudaMemcpyKind, cudaStream_t st) {
    return put(st, [=] { std::memcpy(d, s, n); });
}
// Only copies to the host are waited for.
cudaError_t cudaMemcpy(void* d, const void* s, size_t n, cudaMemcpyKind kind) {
    cudaMemcpyAsync(d, s, n, kind, nullptr);
    if (kind == cudaMemcpyDeviceToDevice) base = static_cast<int*>(d);
    if (kind == cudaMemcpyDeviceToHost) {
        if (n == sizeof(int)) error_word = static_cast<int*>(const_cast<void*>(s));
        run(nullptr);
    }
    return cudaSuccess;
}
cudaError_t cudaStreamSynchronize(cudaStream_t s) { return run(s), cudaSuccess; }
cudaError_t cudaDeviceSynchronize() {
    // The legacy stream first: nothing says that the others' work comes before its own.
    run(nullptr);
    fake_finish();
    return cudaSuccess;
}
void** __cudaRegisterFatBinary(void*) { return nullptr; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
}

namespace tmoe {
struct CacheDev;
struct AppendParams;
struct AttendParams;
using St = cudaStream_t;
void set_global_error(const std::string&) {}
cudaError_t launch_cache_step(const CacheDev&, int, const int*, const int*, int, St) { return cudaSuccess; }
cudaError_t launch_cache_fork(const CacheDev&, int, const int*, const int*, St) { return cudaSuccess; }
cudaError_t launch_cache_truncate(const CacheDev&, int, const int*, const int*, St) { return cudaSuccess; }
cudaError_t launch_cache_accept(const CacheDev&, int, const int*, const int*, const int*, int, St) { return cudaSuccess; }
cudaError_t launch_cache_compact(const CacheDev&, St) { return cudaSuccess; }
cudaError_t launch_cache_append(const CacheDev&, const AppendParams&, St) { return cudaSuccess; }
cudaError_t launch_cache_attend(const CacheDev&, const CUtensorMap&, const CUtensorMap&, const CUtensorMap&,
                                const AttendParams&, int, St) {
    return cudaSuccess;
}
}  // namespace tmoe
