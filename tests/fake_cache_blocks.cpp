// The launch functions behind the calls of cache_blocks.cu, for host tests beside fake_cache.cpp: each launch
// is kept by name.
#include <cuda.h>
#include <cuda_runtime_api.h>

#include <string>

namespace {
std::string launched;
bool capturing = false;
cudaError_t note(const char* name) {
    launched += name;
    launched += ' ';
    return cudaSuccess;
}
}  // namespace

extern "C" {
const char* fake_launched() { return launched.c_str(); }
void fake_forget() { launched.clear(); }
void fake_capture(int on) { capturing = on != 0; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus* s) {
    *s = capturing ? cudaStreamCaptureStatusActive : cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
}

namespace tmoe {
struct CacheDev;
struct AttendParams;
struct BlocksParams;
struct SelectParams;
using St = cudaStream_t;
cudaError_t launch_cache_bounds(const CacheDev&, int, int, int, int whole, St) { return note(whole ? "bounds_whole" : "bounds"); }
cudaError_t launch_cache_select(const CacheDev&, const SelectParams&, St, int& launches) { return launches = 2, note("select"); }
cudaError_t launch_cache_blocks(const CacheDev&, const CUtensorMap&, const CUtensorMap&, const BlocksParams&, St) { return note("blocks"); }
cudaError_t launch_cache_masks(const CacheDev&, const BlocksParams&, St) { return note("masks"); }
cudaError_t launch_cache_own(const CacheDev&, const CUtensorMap&, const CUtensorMap&, const BlocksParams&, St) { return note("own"); }
cudaError_t launch_cache_join(const CacheDev&, const AttendParams&, St) { return note("join"); }
cudaError_t launch_cache_share(const CacheDev&, int, const int*, int, int, int single, St) { return note(single ? "share_single" : "share"); }
int cache_blocks_splits(const CacheDev&, long long, int) { return 1; }
}  // namespace tmoe
