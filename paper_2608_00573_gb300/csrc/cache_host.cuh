// Host side of a cache handle, shared by the files that define its entry points.
#pragma once

#include <string>
#include <vector>

#include <nvtx3/nvToolsExt.h>

#include "cache.cuh"

using namespace tmoe;

struct trimmoe_cache {
    trimmoe_cache_config cfg;
    CacheDev d;
    CacheDev share;                           // d of a step with groups of sequences (its workspaces: first cache_share)
    int dev = 0;
    std::string err;
    std::vector<void*> allocs;
    std::vector<CUtensorMap> tm_k, tm_v;      // per layer: rows [n_pages * kv_heads * page][head_dim], one page and head a box
    std::vector<CUtensorMap> tm_k64, tm_v64;  // the same in boxes of 64 rows, for larger pages
    std::vector<uint32_t> stamp;              // per sequence: last call that listed it
    uint32_t call = 0;
    cudaStream_t last_stream = nullptr;
    uint64_t launches = 0;
    int T = -1, n = 0, max_q = 0;             // the current step (T < 0: none)
    std::vector<int> q_len;                   // [max_seqs] of its listed sequences
    long long triangle = 0;                   // pairs of new tokens of a sequence, the later one sees the other or is it
    // With groups of sequences: what attend launches beside the attention kernel for single tokens and what
    // behind both (set by cache_share).
    cudaError_t (*own)(const CacheDev&, const CUtensorMap&, const CUtensorMap&, const BlocksParams&, cudaStream_t) = nullptr;
    cudaError_t (*join)(const CacheDev&, const AttendParams&, cudaStream_t) = nullptr;
    bool single = false, small = false;       // groups of single tokens; and all of them small
    uint32_t* masks = nullptr;                // room for lists as bits (attend_blocks)
    size_t mask_words = 0;
    float theta = 0.f;                        // base of turn[]
    uint64_t turn[64];

    // Keeps "what: why" (nothing when there is no memory for it: no exception leaves a call).
    trimmoe_status fail(trimmoe_status s, const char* what, const char* why) noexcept {
        try {
            err.assign(what).append(": ").append(why);
        } catch (...) {
            err.clear();
        }
        return s;
    }
    trimmoe_status launched(cudaError_t e, int n_kernels, const char* what) noexcept {
        if (e == cudaSuccess) e = cudaGetLastError();
        if (e != cudaSuccess) return fail(TRIMMOE_ERR_CUDA, what, cudaGetErrorString(e));
        launches += n_kernels;
        return TRIMMOE_OK;
    }
};

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// The handle's device for the duration of a call.
struct OnDevice {
    int prev = -1, dev;
    explicit OnDevice(int d) : dev(d) {
        if (cudaGetDevice(&prev) != cudaSuccess) prev = -1;
        if (prev != dev) cudaSetDevice(dev);
    }
    ~OnDevice() {
        if (prev >= 0 && prev != dev) cudaSetDevice(prev);
    }
};

struct Range {
    explicit Range(const char* name) { nvtxRangePushA(name); }
    ~Range() { nvtxRangePop(); }
};

inline trimmoe_status check_layer(trimmoe_cache* c, const char* what, int layer) {
    if (layer < 0 || layer >= c->cfg.layers) return c->fail(TRIMMOE_ERR_ARG, what, "layer out of range");
    if (c->T < 0) return c->fail(TRIMMOE_ERR_ARG, what, "no step has been begun");
    return TRIMMOE_OK;
}

// Query rows [T][Hq][dh] with row stride ld, a box of one tile (its tokens by the heads of
// a key/value head) by 64 columns.
inline bool query_map(CUtensorMap* tm, const void* base, const CacheDev& d, int T, int ld) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)d.dh, (cuuint64_t)d.Hq, (cuuint64_t)T};
    cuuint64_t strides[2] = {(cuuint64_t)d.dh * 2, (cuuint64_t)ld * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)d.rep, (cuuint32_t)d.tile_tokens};
    cuuint32_t es[3] = {1, 1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Sets up a call on `stream` (after its checks): clears an error that other code
// left behind, so that the launches' own are seen.
inline cudaStream_t enter(trimmoe_cache* c, void* stream) {
    cudaGetLastError();
    c->last_stream = (cudaStream_t)stream;
    return c->last_stream;
}

}  // namespace
