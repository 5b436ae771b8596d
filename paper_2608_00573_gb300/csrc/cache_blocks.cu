// Host side of the cache's attention that does not read all of it: groups of sequences with a
// common prompt, bounds of blocks, their selection, attention over chosen blocks.
#include <algorithm>
#include <cmath>
#include <new>

#include "cache_host.cuh"

namespace {

constexpr int kStageRows = 64;                // positions of a stage of the kernel that follows lists

// Room for the step's lists as bits: for all of T_max when that is 64 MB at most.  (None: the lists are followed.)
bool room_for_masks(trimmoe_cache* c, cudaStream_t st) {
    const size_t row = (size_t)c->d.Hkv * ((c->d.max_pages + 31) / 32 + 2);
    if (!c->masks) {
        const size_t words = std::min(row * c->d.T_max, (size_t)16 << 20);
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        if (row > words || cudaStreamIsCapturing(st, &cap) != cudaSuccess || cap != cudaStreamCaptureStatusNone) {
            cudaGetLastError();
            return false;
        }
        try {
            c->allocs.reserve(c->allocs.size() + 1);
        } catch (const std::bad_alloc&) {
            return false;
        }
        void* q = nullptr;
        if (cudaMalloc(&q, words * sizeof(uint32_t)) != cudaSuccess) {
            cudaGetLastError();
            return false;
        }
        c->allocs.push_back(q);
        c->masks = static_cast<uint32_t*>(q);
        c->mask_words = words;
    }
    return row * c->T <= c->mask_words;
}

}  // namespace

extern "C" trimmoe_status trimmoe_cache_share(trimmoe_cache_handle c, int n, const int32_t* counts, void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    if (c->T < 0) return c->fail(TRIMMOE_ERR_ARG, "cache_share", "no step has been begun");
    if (n < 0 || n > c->n) return c->fail(TRIMMOE_ERR_ARG, "cache_share", "n out of range");
    if (n > 0 && !counts) return c->fail(TRIMMOE_ERR_ARG, "cache_share", "NULL argument");
    long long sum = 0;
    int most = 0;
    for (int i = 0; i < n; ++i) {
        most = std::max(most, counts[i]);
        if (counts[i] < 1) return c->fail(TRIMMOE_ERR_ARG, "cache_share", "counts must be >= 1");
        sum += counts[i];
    }
    if (sum != c->n) return c->fail(TRIMMOE_ERR_ARG, "cache_share", "counts must add up to the step's sequences");
    if (c->T == 0 || (long long)c->T * c->d.Hq > kShareRows) return TRIMMOE_OK;
    // Query tiles of the groups' common pages against those of the sequences by themselves.  Not half as many: sequences
    // that read common pages out of L2 each for itself are as fast.  (With groups against without, 12 trees with up to 2000
    // positions of their own behind a common 12000, 32 heads on 8: 2 tokens each, 0.08 of the tiles, 31 us / 76; 8, 0.25, 49 / 77;
    // 16, 0.5, 65 / 84; 20, 0.67, 74 / 85; 24, 0.75, 86 / 85; 29, 0.92, 92 / 85; behind 2000: 24 41 / 34; 6 prompts of 200
    // to 400 behind 6000 211 / 185.)  The prefix's length counts too, but only the GPU knows it; with up to 200 positions of their own,
    // with / without: 12 trees of 8 behind 300, 1000, 4000, 12000 15.9 / 17.1, 19.4 / 22.9, 27.4 / 35.9, 41.3 / 70.5; of 16 (0.5) 17.3 /
    // 17.5, 22.6 / 23.1, 32.8 / 36.9, 55.4 / 76.9; 12 pairs of trees of 16 (0.5) 25.1 / 22.5, 35.3 / 31.7, 57.2 / 71.5, 112 /
    // 187; 16 heads on 16 36.1 / 28.6, 55.1 / 53.1, 107 / 160, 237 / 444: pairs behind a short prompt lose.
    // Nor where groups of one have four fifths of the tiles: all items' parts are joined then.  (Of 32 trees of 8 tokens 16, 8, 4 in
    // a group, the others with prompts of their own: behind 1000 positions 39.4 / 38.8, 41.4 / 39.5, 42.1 / 39.8, behind 6000
    // 89.6 / 96.8, 109 / 119, 123 / 130; 16 heads on 16 65.8 / 67.2, 69.1 / 67.3, 70.5 / 67.4 and 180 / 304, 236 / 304, 263 / 305.)
    if (c->max_q > 1 || c->d.rep > 16) {
        auto tiles = [&](long long tokens) { return (tokens + c->d.tile_tokens - 1) / c->d.tile_tokens; };
        long long shared = 0, alone = 0, others = 0;
        for (int i = 0, at = 0; i < n; ++i) {
            long long tokens = 0;
            for (int k = 0; k < counts[i]; ++k, ++at) {
                tokens += c->q_len[at];
                (counts[i] > 1 ? alone : others) += tiles(c->q_len[at]);
            }
            if (counts[i] > 1) shared += tiles(tokens);
        }
        if (2 * shared > alone || 4 * alone <= others) {
            c->d.shared = 0;
            return TRIMMOE_OK;
        }
    }
    OnDevice on(c->dev);
    Range range("trimmoe.cache_share");
    cudaStream_t st = enter(c, stream);
    if (!c->share.part_o) {
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(st, &cap) != cudaSuccess || cap != cudaStreamCaptureStatusNone)
            return c->fail(TRIMMOE_ERR_ARG, "cache_share", "the first call allocates and must not be captured");
        CacheDev d = c->d;
        cudaError_t e = cudaSuccess;
        size_t had = c->allocs.size();
        try {
            c->allocs.reserve(had + 10);
        } catch (const std::bad_alloc&) {
            return c->fail(TRIMMOE_ERR_OOM, "cache_share", "host allocation failed");
        }
        auto alloc = [&](auto*& p, size_t count) {
            void* q = nullptr;
            if (e == cudaSuccess) e = cudaMalloc(&q, count * sizeof(*p));
            if (e != cudaSuccess) return;
            c->allocs.push_back(q);
            p = static_cast<std::remove_reference_t<decltype(p)>>(q);
        };
        const size_t rows = (size_t)cache_share_part_rows(d);
        d.step_plan = d.plan;
        alloc(d.plan, 1);
        alloc(d.shares, (size_t)d.num_sms);
        alloc(d.groups, (size_t)cache_share_groups(d));
        alloc(d.parts_of, (size_t)cache_share_tokens(d));
        alloc(d.pieces, (size_t)kPieces);
        alloc(d.lists, (size_t)cache_share_tokens(d) * d.Hkv * 2);
        alloc(d.common, (size_t)d.max_seqs);
        alloc(d.cut, (size_t)cache_share_groups(d) * d.Hkv);
        alloc(d.part_ml, rows);
        alloc(d.part_o, rows * d.dh);
        if (e != cudaSuccess) {
            for (; c->allocs.size() > had; c->allocs.pop_back()) cudaFree(c->allocs.back());
            cudaGetLastError();
            return c->fail(e == cudaErrorMemoryAllocation ? TRIMMOE_ERR_OOM : TRIMMOE_ERR_CUDA, "cache_share",
                           cudaGetErrorString(e));
        }
        c->share = d;
    }
    c->share.shared = 1;
    // Single tokens: up to 16 query heads of a key/value head are a tile of the kernel that reads
    // pieces.
    c->own = launch_cache_own;
    c->join = launch_cache_join;
    c->single = c->max_q == 1 && c->d.rep <= 16;
    c->small = c->single && small_tiles(most, c->d.rep) <= kSmallTiles;
    const trimmoe_status s = c->launched(launch_cache_share(c->share, n, counts, c->n, c->T, c->single, st), 2, "cache_share");
    // (Without its list a step cannot be attended.)
    if (s != TRIMMOE_OK) c->T = -1;
    else c->d.shared = 1;
    return s;
}

extern "C" trimmoe_status trimmoe_cache_set_bounds(trimmoe_cache_handle c, int8_t* codes, float* scales) {
    if (!c) return TRIMMOE_ERR_ARG;
    if (!codes != !scales) return c->fail(TRIMMOE_ERR_ARG, "cache_set_bounds", "codes and scales come together");
    if (!aligned16(codes) || (reinterpret_cast<uintptr_t>(scales) & 3u))
        return c->fail(TRIMMOE_ERR_ARG, "cache_set_bounds", "pointers must be aligned (codes 16 bytes, scales 4)");
    if (codes && !c->d.scores) {
        OnDevice on(c->dev);
        cudaGetLastError();
        void* q = nullptr;
        try {
            c->allocs.reserve(c->allocs.size() + 1);
        } catch (const std::bad_alloc&) {
            return c->fail(TRIMMOE_ERR_OOM, "cache_set_bounds", "host allocation failed");
        }
        const cudaError_t e = cudaMalloc(&q, cache_score_keys(c->d) * sizeof(uint32_t));
        if (e != cudaSuccess) {
            cudaGetLastError();
            return c->fail(e == cudaErrorMemoryAllocation ? TRIMMOE_ERR_OOM : TRIMMOE_ERR_CUDA, "cache_set_bounds", cudaGetErrorString(e));
        }
        c->allocs.push_back(q);
        c->d.scores = static_cast<uint32_t*>(q);
    }
    c->d.codes = codes;
    c->d.scales = scales;
    return TRIMMOE_OK;
}

extern "C" trimmoe_status trimmoe_cache_summarize(trimmoe_cache_handle c, int layer, int whole, void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    const trimmoe_status s = check_layer(c, "cache_summarize", layer);
    if (s != TRIMMOE_OK) return s;
    if (!c->d.codes) return c->fail(TRIMMOE_ERR_ARG, "cache_summarize", "no bounds have been set");
    if (c->n == 0) return TRIMMOE_OK;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_summarize");
    return c->launched(launch_cache_bounds(c->d, layer, c->n, c->max_q, whole != 0, enter(c, stream)), 1, "cache_summarize");
}

extern "C" trimmoe_status trimmoe_cache_select(trimmoe_cache_handle c, int layer, const trimmoe_select_args* a, void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    const trimmoe_status s = check_layer(c, "cache_select", layer);
    if (s != TRIMMOE_OK) return s;
    const CacheDev& d = c->d;
    if (!a) return c->fail(TRIMMOE_ERR_ARG, "cache_select", "NULL argument");
    if (!d.codes) return c->fail(TRIMMOE_ERR_ARG, "cache_select", "no bounds have been set");
    if (a->n < 1 || a->first < 0 || a->last < 0 || a->first > a->n || a->last > a->n - a->first)
        return c->fail(TRIMMOE_ERR_ARG, "cache_select", "n must be >= 1, first and last >= 0 and together at most n");
    if (c->T == 0) return TRIMMOE_OK;
    if (!a->q || !a->blocks) return c->fail(TRIMMOE_ERR_ARG, "cache_select", "NULL pointer");
    if (!aligned16(a->q) || a->ld_q % 8 || (reinterpret_cast<uintptr_t>(a->blocks) & 3u))
        return c->fail(TRIMMOE_ERR_ARG, "cache_select", "pointers must be aligned (q 16 bytes) and the row stride a multiple of 8");
    if (a->ld_q < d.Hq * d.dh) return c->fail(TRIMMOE_ERR_ARG, "cache_select", "row stride shorter than a row");
    if ((long long)c->T * d.Hkv > 0x7fffffffLL) return c->fail(TRIMMOE_ERR_UNSUPPORTED, "cache_select", "T * kv_heads must be < 2^31");
    SelectParams p = {};
    p.q = static_cast<const __nv_bfloat16*>(a->q);
    p.blocks = a->blocks;
    p.ld_q = a->ld_q;
    p.T = c->T;
    p.n = a->n;
    p.first = a->first;
    p.last = a->last;
    p.layer = layer;
    p.max_q = c->max_q;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_select");
    int launches = 0;
    const cudaError_t e = launch_cache_select(d, p, enter(c, stream), launches);
    return c->launched(e, launches, "cache_select");
}

extern "C" trimmoe_status trimmoe_cache_attend_blocks(trimmoe_cache_handle c, int layer, const trimmoe_blocks_args* a,
                                                      void* stream) {
    if (!c) return TRIMMOE_ERR_ARG;
    const char* what = "cache_attend_blocks";
    const trimmoe_status s = check_layer(c, what, layer);
    if (s != TRIMMOE_OK) return s;
    if (!a) return c->fail(TRIMMOE_ERR_ARG, what, "NULL argument");
    if (a->n < 0) return c->fail(TRIMMOE_ERR_ARG, what, "n must be >= 0");
    if (c->T == 0) return TRIMMOE_OK;
    const CacheDev& d = c->d;
    if (!a->q || !a->out || (a->n > 0 && !a->blocks)) return c->fail(TRIMMOE_ERR_ARG, what, "NULL pointer");
    if (!aligned16(a->q) || !aligned16(a->out) || a->ld_q % 8 || a->ld_out % 8 || (reinterpret_cast<uintptr_t>(a->tree) & 7u) ||
        (reinterpret_cast<uintptr_t>(a->blocks) & 3u))
        return c->fail(TRIMMOE_ERR_ARG, what, "pointers must be aligned (q, out 16 bytes) and row strides multiples of 8");
    if (a->ld_q < d.Hq * d.dh || a->ld_out < d.Hq * d.dh) return c->fail(TRIMMOE_ERR_ARG, what, "row stride shorter than a row");
    if (!(a->scale >= 0.f && std::isfinite(a->scale))) return c->fail(TRIMMOE_ERR_ARG, what, "scale must be finite and >= 0");
    if (a->tree && c->max_q > kTreeMax) return c->fail(TRIMMOE_ERR_ARG, what, "a tree has at most 64 tokens per sequence");
    BlocksParams p = {};
    p.q = static_cast<const __nv_bfloat16*>(a->q);
    p.out = static_cast<__nv_bfloat16*>(a->out);
    p.blocks = a->blocks;
    p.tree = a->tree;
    p.ld_q = a->ld_q;
    p.ld_out = a->ld_out;
    p.T = c->T;
    p.n = a->n;
    p.row_tiles = (d.rep + 15) / 16;
    p.splits = cache_blocks_splits(d, (long long)c->T * d.Hkv * p.row_tiles, std::max(1, (int)std::min(1LL << 20, (long long)a->n * d.page / 64)));
    if ((long long)c->T * d.Hkv * p.row_tiles > (1LL << 26)) return c->fail(TRIMMOE_ERR_UNSUPPORTED, what, "more than 2^26 items");
    p.scale_log2 = (a->scale > 0.f ? a->scale : 1.f / std::sqrt((float)d.dh)) * 1.4426950408889634f;
    const bool large = d.page > 64;
    OnDevice on(c->dev);
    Range range("trimmoe.cache_attend_blocks");
    cudaStream_t st = enter(c, stream);
    // Tokens of prompts: where their lists name much of what their sequences hold, 128 rows at a time over all
    // pages, with the lists as masks, is faster.  The lengths decide, on the GPU (lists_dense); lists that are
    // followed in 45 us are not worth the launches, nor are tiles half empty.
    const long long rows = (long long)p.T * std::max(1LL, (long long)p.n * d.page / kStageRows) + c->triangle / kStageRows;
    const long long stages = rows * d.Hkv * p.row_tiles;
    int launches = 1;
    if (c->max_q >= (kCacheTile / 2 + d.rep - 1) / d.rep && stages * kStageCost >= 45000LL * d.num_sms && room_for_masks(c, st)) {
        p.lists = PageLists{c->masks, (d.max_pages + 31) / 32, stages};
        AttendParams m = {};
        m.lists = p.lists;
        m.tree = p.tree;
        m.out = p.out;
        m.ld_out = p.ld_out;
        m.scale_log2 = p.scale_log2;
        m.T = p.T;
        CUtensorMap tm_q;
        if (!query_map(&tm_q, a->q, d, c->T, a->ld_q)) return c->fail(TRIMMOE_ERR_CUDA, what, "cuTensorMapEncodeTiled failed");
        const int max_rows = c->max_q > d.tile_tokens ? 2 * kCacheTile : c->max_q * d.rep;
        cudaError_t e = launch_cache_masks(d, p, st);
        if (e == cudaSuccess) e = launch_cache_attend(d, tm_q, c->tm_k[layer], c->tm_v[layer], m, max_rows, st);
        if (e != cudaSuccess) return c->launched(e, 0, what);
        launches += 3;
    }
    return c->launched(launch_cache_blocks(d, large ? c->tm_k64[layer] : c->tm_k[layer], large ? c->tm_v64[layer] : c->tm_v[layer],
                                           p, st),
                       launches, what);
}
