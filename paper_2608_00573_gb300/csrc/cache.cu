// Host side of the paged key/value cache (trimmoe_cache_*): checks, workspaces,
// tensor maps, launches.  Lengths and page indices stay on the GPU.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include <nvtx3/nvToolsExt.h>

#include "cache.cuh"

using namespace tmoe;

struct trimmoe_cache {
    trimmoe_cache_config cfg;
    CacheDev d;
    int dev = 0;
    std::string err;
    std::vector<void*> allocs;
    std::vector<CUtensorMap> tm_k, tm_v;      // per layer: rows [n_pages * kv_heads * page][head_dim], one page and head a box
    std::vector<uint32_t> stamp;              // per sequence: last call that listed it
    uint32_t call = 0;
    cudaStream_t last_stream = nullptr;
    uint64_t launches = 0;
    int T = -1, n = 0, max_q = 0;             // the current step (T < 0: none)
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

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

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

trimmoe_status check_config(const trimmoe_cache_config& c, const char*& why) {
    auto bad = [&](trimmoe_status s, const char* m) {
        why = m;
        return s;
    };
    if (c.layers < 1 || c.q_heads < 1 || c.kv_heads < 1 || c.n_pages < 1 || c.max_seqs < 1 || c.max_pages < 1 ||
        c.T_max < 1)
        return bad(TRIMMOE_ERR_ARG, "sizes must be >= 1");
    if (c.q_heads % c.kv_heads) return bad(TRIMMOE_ERR_ARG, "q_heads must be a multiple of kv_heads");
    if (c.head_dim != 64 && c.head_dim != 128) return bad(TRIMMOE_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128)
        return bad(TRIMMOE_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128");
    if (c.q_heads / c.kv_heads > 128) return bad(TRIMMOE_ERR_UNSUPPORTED, "q_heads / kv_heads must be <= 128");
    if (c.q_heads > 4096) return bad(TRIMMOE_ERR_UNSUPPORTED, "q_heads must be <= 4096");
    if (c.max_seqs > kCacheMaxSeqs) return bad(TRIMMOE_ERR_UNSUPPORTED, "max_seqs must be <= 1024");
    if (c.T_max > (1 << 20)) return bad(TRIMMOE_ERR_UNSUPPORTED, "T_max must be <= 2^20");
    if ((double)c.n_pages * c.kv_heads * c.page_size >= 2147483648.0 || (double)c.max_pages * c.page_size >= 2147483648.0)
        return bad(TRIMMOE_ERR_UNSUPPORTED, "n_pages * kv_heads * page_size and max_pages * page_size must be < 2^31");
    return TRIMMOE_OK;
}

// Pool rows of one layer, a box of one page and head by 64 columns.
bool pool_map(CUtensorMap* tm, const void* base, const CacheDev& d) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)d.dh, (cuuint64_t)d.n_pages * d.Hkv * d.page};
    cuuint64_t strides[1] = {(cuuint64_t)d.dh * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)d.page};
    cuuint32_t es[2] = {1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Query rows [T][Hq][dh] with row stride ld, a box of one tile (its tokens by the heads of
// a key/value head) by 64 columns.
bool query_map(CUtensorMap* tm, const void* base, const CacheDev& d, int T, int ld) {
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

// Listed sequences: in range and distinct.
trimmoe_status check_list(trimmoe_cache* c, const char* what, int n, const int32_t* seq, bool fresh_stamp = true) {
    if (n < 0 || n > c->cfg.max_seqs) return c->fail(TRIMMOE_ERR_ARG, what, "n out of range");
    if (n > 0 && !seq) return c->fail(TRIMMOE_ERR_ARG, what, "NULL argument");
    if (fresh_stamp && ++c->call == 0) {
        std::fill(c->stamp.begin(), c->stamp.end(), 0u);
        c->call = 1;
    }
    for (int i = 0; i < n; ++i) {
        if (seq[i] < 0 || seq[i] >= c->cfg.max_seqs)
            return c->fail(TRIMMOE_ERR_ARG, what, "sequence out of range");
        if (c->stamp[seq[i]] == c->call)
            return c->fail(TRIMMOE_ERR_ARG, what, "a sequence is listed twice");
        c->stamp[seq[i]] = c->call;
    }
    return TRIMMOE_OK;
}

trimmoe_status check_layer(trimmoe_cache* c, const char* what, int layer) {
    if (layer < 0 || layer >= c->cfg.layers) return c->fail(TRIMMOE_ERR_ARG, what, "layer out of range");
    if (c->T < 0) return c->fail(TRIMMOE_ERR_ARG, what, "no step has been begun");
    return TRIMMOE_OK;
}

// Sets up a call on `stream` (after its checks): clears an error that other code
// left behind, so that the launches' own are seen.
cudaStream_t enter(trimmoe_cache* c, void* stream) {
    cudaGetLastError();
    c->last_stream = (cudaStream_t)stream;
    return c->last_stream;
}

}  // namespace

extern "C" trimmoe_status trimmoe_cache_create(const trimmoe_cache_config* cfg, const trimmoe_cache_state* st,
                                               trimmoe_cache_handle* out) {
    auto create_fail = [](trimmoe_status s, const char* m) noexcept {
        try {
            set_global_error(std::string("cache_create: ") + m);
        } catch (...) {
        }
        return s;
    };
    if (!out) return create_fail(TRIMMOE_ERR_ARG, "out is NULL");
    *out = nullptr;
    if (!cfg || !st || !st->k || !st->v || !st->table || !st->length || !st->ref)
        return create_fail(TRIMMOE_ERR_ARG, "NULL argument");
    if (!aligned16(st->k) || !aligned16(st->v))
        return create_fail(TRIMMOE_ERR_ARG, "k and v must be 16-byte aligned");
    const char* why = "";
    const trimmoe_status cs = check_config(*cfg, why);
    if (cs != TRIMMOE_OK) return create_fail(cs, why);
    trimmoe_cache* c = new (std::nothrow) trimmoe_cache();
    if (!c) return create_fail(TRIMMOE_ERR_OOM, "host allocation failed");
    auto bail = [&](trimmoe_status s, const char* m) noexcept {
        trimmoe_cache_destroy(c);
        return create_fail(s, m);
    };
    try {
        c->cfg = *cfg;
        CacheDev& d = c->d;
        d = CacheDev{};
        cudaGetLastError();
        cudaDeviceProp prop;
        if (cudaGetDevice(&c->dev) != cudaSuccess || cudaGetDeviceProperties(&prop, c->dev) != cudaSuccess)
            return bail(TRIMMOE_ERR_CUDA, "no CUDA device");
        if (prop.major != 10 || prop.minor != 3)
            return bail(TRIMMOE_ERR_UNSUPPORTED, "needs compute capability 10.3");
        d.layers = cfg->layers;
        d.Hq = cfg->q_heads;
        d.Hkv = cfg->kv_heads;
        d.rep = cfg->q_heads / cfg->kv_heads;
        d.dh = cfg->head_dim;
        d.page = cfg->page_size;
        d.page_shift = cfg->page_size == 16 ? 4 : cfg->page_size == 32 ? 5 : cfg->page_size == 64 ? 6 : 7;
        d.n_pages = cfg->n_pages;
        d.max_seqs = cfg->max_seqs;
        d.max_pages = cfg->max_pages;
        d.T_max = cfg->T_max;
        d.tile_tokens = kCacheTile / d.rep;
        d.num_sms = prop.multiProcessorCount;
        d.k = static_cast<__nv_bfloat16*>(st->k);
        d.v = static_cast<__nv_bfloat16*>(st->v);
        d.table = st->table;
        d.length = st->length;
        d.ref = st->ref;
        c->stamp.assign(cfg->max_seqs, 0u);
        cudaError_t e = cudaSuccess;
        auto alloc = [&](auto*& p, size_t n) {
            if (e != cudaSuccess) return;
            void* q = nullptr;
            e = cudaMalloc(&q, std::max<size_t>(n, 1) * sizeof(*p));
            if (e == cudaSuccess) {
                c->allocs.push_back(q);
                p = static_cast<std::remove_reference_t<decltype(p)>>(q);
            }
        };
        c->allocs.reserve(16);
        alloc(d.plan, 1);
        alloc(d.seqs, kCacheMaxSeqs);
        alloc(d.groups, (size_t)cfg->T_max / (2 * d.tile_tokens) + cfg->max_seqs + 1);
        alloc(d.shares, (size_t)d.num_sms);
        alloc(d.slot, cfg->T_max);
        alloc(d.pos, cfg->T_max);
        alloc(d.copies, (size_t)std::max(cfg->n_pages, cfg->max_seqs));
        alloc(d.fresh, cfg->n_pages);
        alloc(d.base, cfg->max_seqs);
        alloc(d.holders, cfg->n_pages);
        alloc(d.part_o, (size_t)2 * d.num_sms * 256 * d.dh);
        alloc(d.part_ml, (size_t)2 * d.num_sms * 256);
        alloc(d.arrived, (size_t)d.num_sms);
        alloc(d.err, 2);
        if (e != cudaSuccess)
            return bail(e == cudaErrorMemoryAllocation ? TRIMMOE_ERR_OOM : TRIMMOE_ERR_CUDA, cudaGetErrorString(e));
        d.refused = d.err + 1;
        e = cudaMemset(d.err, 0, 2 * sizeof(int));
        if (e == cudaSuccess) e = cudaMemset(d.plan, 0, sizeof(CachePlan));
        if (e == cudaSuccess) e = cudaMemset(d.holders, 0, sizeof(int) * (size_t)cfg->n_pages);
        // Without a step a sequence has no drafts to accept.  (The lengths may still be on their
        // way in any stream.)
        if (e == cudaSuccess) e = cudaDeviceSynchronize();
        if (e == cudaSuccess) e = cudaMemcpy(d.base, d.length, sizeof(int) * (size_t)cfg->max_seqs, cudaMemcpyDeviceToDevice);
        if (e == cudaSuccess) e = cudaDeviceSynchronize();
        if (e != cudaSuccess) return bail(TRIMMOE_ERR_CUDA, cudaGetErrorString(e));
        c->tm_k.resize(cfg->layers);
        c->tm_v.resize(cfg->layers);
        const size_t layer = (size_t)d.n_pages * d.Hkv * d.page * d.dh;
        for (int l = 0; l < cfg->layers; ++l)
            if (!pool_map(&c->tm_k[l], d.k + l * layer, d) || !pool_map(&c->tm_v[l], d.v + l * layer, d))
                return bail(TRIMMOE_ERR_CUDA, "cuTensorMapEncodeTiled failed");
    } catch (const std::bad_alloc&) {
        return bail(TRIMMOE_ERR_OOM, "host allocation failed");
    }
    *out = c;
    return TRIMMOE_OK;
}

extern "C" trimmoe_status trimmoe_cache_step(trimmoe_cache_handle c, int n, const int32_t* seq, const int32_t* q_len,
                                             void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    trimmoe_status s = check_list(c, "cache_step", n, seq);
    if (s != TRIMMOE_OK) return s;
    if (n > 0 && !q_len) return c->fail(TRIMMOE_ERR_ARG, "cache_step", "NULL argument");
    long long T = 0;
    int most = 0;
    for (int i = 0; i < n; ++i) {
        if (q_len[i] < 0) return c->fail(TRIMMOE_ERR_ARG, "cache_step", "q_len must be >= 0");
        T += q_len[i];
        most = std::max(most, q_len[i]);
    }
    if (T > c->cfg.T_max) return c->fail(TRIMMOE_ERR_ARG, "cache_step", "more than T_max new tokens");
    c->T = -1;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_step");
    s = c->launched(launch_cache_step(c->d, n, seq, q_len, (int)T, enter(c, stream)), 2, "cache_step");
    if (s != TRIMMOE_OK) return s;
    c->T = (int)T;
    c->n = n;
    c->max_q = most;
    return TRIMMOE_OK;
}

extern "C" trimmoe_status trimmoe_cache_append(trimmoe_cache_handle c, int layer, const trimmoe_append_args* a,
                                               void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    const trimmoe_status s = check_layer(c, "cache_append", layer);
    if (s != TRIMMOE_OK) return s;
    if (!a) return c->fail(TRIMMOE_ERR_ARG, "cache_append", "NULL argument");
    if (c->T == 0) return TRIMMOE_OK;
    const CacheDev& d = c->d;
    if (!a->qkv || !a->q_out || !a->gamma_q != !a->gamma_k)
        return c->fail(TRIMMOE_ERR_ARG, "cache_append", "NULL pointer (gamma_q and gamma_k come together)");
    if (!aligned16(a->qkv) || !aligned16(a->q_out) || !aligned16(a->gamma_q) || !aligned16(a->gamma_k) ||
        a->ld_qkv % 8 || a->ld_q % 8)
        return c->fail(TRIMMOE_ERR_ARG, "cache_append", "pointers must be 16-byte aligned and row strides multiples of 8");
    if (a->ld_qkv < (d.Hq + 2 * d.Hkv) * d.dh || a->ld_q < d.Hq * d.dh)
        return c->fail(TRIMMOE_ERR_ARG, "cache_append", "row stride shorter than a row");
    if (a->gamma_q && !(a->norm_eps >= 0.f && std::isfinite(a->norm_eps)))
        return c->fail(TRIMMOE_ERR_ARG, "cache_append", "norm_eps must be finite and >= 0");
    if (!(a->rope_theta >= 0.f && std::isfinite(a->rope_theta)) || (a->rope_theta > 0.f && a->rope_theta < 1.f))
        return c->fail(TRIMMOE_ERR_ARG, "cache_append", "rope_theta must be 0 or finite and >= 1");
    if (a->rope_theta > 0.f && a->rope_theta != c->theta) {
        // theta^(-2i/D) / 2 pi turns per position, as a fraction of 2^64.
        for (int i = 0; i < d.dh / 2; ++i)
            c->turn[i] = (uint64_t)(std::pow((double)a->rope_theta, -2.0 * i / d.dh) / (2.0 * M_PI) * 18446744073709551616.0);
        c->theta = a->rope_theta;
    }
    AppendParams p = {};
    p.qkv = static_cast<const __nv_bfloat16*>(a->qkv);
    p.q_out = static_cast<__nv_bfloat16*>(a->q_out);
    p.ld_qkv = a->ld_qkv;
    p.ld_q = a->ld_q;
    p.T = c->T;
    p.norm = a->gamma_q != nullptr;
    p.rope = a->rope_theta > 0.f;
    p.layer_off = (long long)layer * d.n_pages * d.Hkv * d.page * d.dh;
    p.gamma_q = static_cast<const __nv_bfloat16*>(a->gamma_q);
    p.gamma_k = static_cast<const __nv_bfloat16*>(a->gamma_k);
    p.eps = a->norm_eps;
    p.pos = a->pos;
    std::copy(c->turn, c->turn + 64, p.turn);
    OnDevice on(c->dev);
    Range range("trimmoe.cache_append");
    return c->launched(launch_cache_append(d, p, enter(c, stream)), 1, "cache_append");
}

extern "C" trimmoe_status trimmoe_cache_attend(trimmoe_cache_handle c, int layer, const trimmoe_attend_args* a,
                                               void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    const trimmoe_status s = check_layer(c, "cache_attend", layer);
    if (s != TRIMMOE_OK) return s;
    if (!a) return c->fail(TRIMMOE_ERR_ARG, "cache_attend", "NULL argument");
    if (c->T == 0) return TRIMMOE_OK;
    const CacheDev& d = c->d;
    if (!a->q || !a->out) return c->fail(TRIMMOE_ERR_ARG, "cache_attend", "NULL pointer");
    if (!aligned16(a->q) || !aligned16(a->out) || a->ld_q % 8 || a->ld_out % 8 || (reinterpret_cast<uintptr_t>(a->tree) & 7u))
        return c->fail(TRIMMOE_ERR_ARG, "cache_attend", "pointers must be aligned (q, out 16 bytes) and row strides multiples of 8");
    if (a->ld_q < d.Hq * d.dh || a->ld_out < d.Hq * d.dh)
        return c->fail(TRIMMOE_ERR_ARG, "cache_attend", "row stride shorter than a row");
    if (!(a->scale >= 0.f && std::isfinite(a->scale)))
        return c->fail(TRIMMOE_ERR_ARG, "cache_attend", "scale must be finite and >= 0");
    if (a->tree && c->max_q > kTreeMax)
        return c->fail(TRIMMOE_ERR_ARG, "cache_attend", "a tree has at most 64 tokens per sequence");
    CUtensorMap tm_q;
    if (!query_map(&tm_q, a->q, d, c->T, a->ld_q))
        return c->fail(TRIMMOE_ERR_CUDA, "cache_attend", "cuTensorMapEncodeTiled failed");
    AttendParams p = {};
    p.tree = a->tree;
    p.out = static_cast<__nv_bfloat16*>(a->out);
    p.ld_out = a->ld_out;
    p.scale_log2 = (a->scale > 0.f ? a->scale : 1.f / std::sqrt((float)d.dh)) * 1.4426950408889634f;
    const int max_rows = c->max_q > d.tile_tokens ? 2 * kCacheTile : c->max_q * d.rep;
    p.join_here = max_rows <= kJoinHereRows;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_attend");
    return c->launched(launch_cache_attend(d, tm_q, c->tm_k[layer], c->tm_v[layer], p, max_rows, enter(c, stream)),
                       p.join_here ? 1 : 2, "cache_attend");
}

extern "C" trimmoe_status trimmoe_cache_fork(trimmoe_cache_handle c, int n, const int32_t* src, const int32_t* dst,
                                             void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    trimmoe_status s = check_list(c, "cache_fork", n, dst);
    if (s != TRIMMOE_OK) return s;
    if (n > 0 && !src) return c->fail(TRIMMOE_ERR_ARG, "cache_fork", "NULL argument");
    for (int i = 0; i < n; ++i) {
        if (src[i] < 0 || src[i] >= c->cfg.max_seqs)
            return c->fail(TRIMMOE_ERR_ARG, "cache_fork", "sequence out of range");
        if (c->stamp[src[i]] == c->call)
            return c->fail(TRIMMOE_ERR_ARG, "cache_fork", "a source is also a destination");
    }
    if (n == 0) return TRIMMOE_OK;
    c->T = -1;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_fork");
    return c->launched(launch_cache_fork(c->d, n, src, dst, enter(c, stream)), 1, "cache_fork");
}

extern "C" trimmoe_status trimmoe_cache_truncate(trimmoe_cache_handle c, int n, const int32_t* seq,
                                                 const int32_t* length, void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    const trimmoe_status s = check_list(c, "cache_truncate", n, seq);
    if (s != TRIMMOE_OK) return s;
    if (n > 0 && !length) return c->fail(TRIMMOE_ERR_ARG, "cache_truncate", "NULL argument");
    for (int i = 0; i < n; ++i)
        if (length[i] < 0) return c->fail(TRIMMOE_ERR_ARG, "cache_truncate", "length must be >= 0");
    if (n == 0) return TRIMMOE_OK;
    c->T = -1;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_truncate");
    return c->launched(launch_cache_truncate(c->d, n, seq, length, enter(c, stream)), 1, "cache_truncate");
}

extern "C" trimmoe_status trimmoe_cache_accept(trimmoe_cache_handle c, int n, const int32_t* seq, const int32_t* n_acc,
                                               const int32_t* path, int ld_path, void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    const trimmoe_status s = check_list(c, "cache_accept", n, seq);
    if (s != TRIMMOE_OK) return s;
    if (n == 0) return TRIMMOE_OK;
    if (!n_acc || ld_path < 0 || (ld_path > 0 && !path))
        return c->fail(TRIMMOE_ERR_ARG, "cache_accept", "NULL argument");
    c->T = -1;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_accept");
    return c->launched(launch_cache_accept(c->d, n, seq, n_acc, path, ld_path, enter(c, stream)), 2, "cache_accept");
}

extern "C" trimmoe_status trimmoe_cache_compact(trimmoe_cache_handle c, void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    c->T = -1;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_compact");
    return c->launched(launch_cache_compact(c->d, enter(c, stream)), 5, "cache_compact");
}

extern "C" trimmoe_status trimmoe_cache_stats(trimmoe_cache_handle c, trimmoe_cache_stats_t* out, int reset) {
    if (!c) return TRIMMOE_ERR_ARG;
    if (!out) return c->fail(TRIMMOE_ERR_ARG, "cache_stats", "NULL argument");
    OnDevice on(c->dev);
    cudaGetLastError();
    cudaError_t e = cudaStreamSynchronize(c->last_stream);
    int code = 0, free_pages = 0;
    try {
        std::vector<int> ref(c->cfg.n_pages);
        if (e == cudaSuccess) e = cudaMemcpy(&code, c->d.err, sizeof code, cudaMemcpyDeviceToHost);
        if (e == cudaSuccess) e = cudaMemcpy(ref.data(), c->d.ref, sizeof(int) * ref.size(), cudaMemcpyDeviceToHost);
        for (int r : ref) free_pages += r == 0;
    } catch (const std::bad_alloc&) {
        return c->fail(TRIMMOE_ERR_OOM, "cache_stats", "host allocation failed");
    }
    if (e == cudaSuccess && reset) {
        // (Cleared when the call returns: what a kernel flags from then on stays.)
        e = cudaMemsetAsync(c->d.err, 0, 2 * sizeof code, c->last_stream);
        if (e == cudaSuccess) e = cudaStreamSynchronize(c->last_stream);
    }
    if (e != cudaSuccess) return c->fail(TRIMMOE_ERR_CUDA, "cache_stats", cudaGetErrorString(e));
    out->device_error = code;
    out->free_pages = free_pages;
    out->launches = c->launches;
    if (code == TRIMMOE_DEVERR_CACHE_ATTENTION)
        return c->fail(TRIMMOE_ERR_DEVICE_TIMEOUT, "cache", "a wait of the attention kernel ran out");
    if (code == TRIMMOE_DEVERR_CACHE_FULL)
        return c->fail(TRIMMOE_ERR_CACHE, "cache_step", "too few free pages, or a sequence longer than max_pages");
    if (code == TRIMMOE_DEVERR_CACHE_STATE)
        return c->fail(TRIMMOE_ERR_CACHE, "cache", "table, length or ref hold invalid values");
    if (code == TRIMMOE_DEVERR_CACHE_PATH)
        return c->fail(TRIMMOE_ERR_CACHE, "cache_accept", "n_acc or path does not fit the drafts");
    return code ? c->fail(TRIMMOE_ERR_CACHE, "cache", "device error") : TRIMMOE_OK;
}

extern "C" const char* trimmoe_cache_last_error(trimmoe_cache_handle c) { return c ? c->err.c_str() : ""; }

extern "C" void trimmoe_cache_destroy(trimmoe_cache_handle c) {
    if (!c) return;
    OnDevice on(c->dev);
    if (!c->allocs.empty()) cudaDeviceSynchronize();
    for (void* p : c->allocs) cudaFree(p);
    delete c;
}
