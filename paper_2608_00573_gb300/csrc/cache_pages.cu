// Page bookkeeping of the key/value cache: room for a step's tokens (with copies
// of shared last pages and the attention's work list), forks, cuts, accepted
// drafts and compaction.
//
// Everything is decided on the GPU from table, length and ref, so that lengths
// that a previous kernel computed (accepted drafts) are used without a copy to
// the host.  Page indices do not depend on timing: free pages are taken lowest
// first in the order of the listed sequences, by prefix sums; only counts
// (ref) are changed by atomics, which commute.
//
// Bounds: the bookkeeping reads a few kB and is a chain of dependent reads in
// one block; page copies move 2 x layers x kv_heads x page_size x head_dim x 2
// bytes each way per page and are bound by HBM.
#include <algorithm>

#include "cache.cuh"

namespace tmoe {

namespace {

constexpr int kStepThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kCopyVecs = 4;           // 16-byte vectors in flight per thread
// Smallest share of a CTA, in key tiles: below it, fewer CTAs take part.  Two tiles
// keep both slots busy at once (decoding one sequence of 1500 positions takes 11.5 us so,
// 15.7 with three and more CTAs idle).
constexpr int kMinTiles = 2;

// Exclusive prefix sum over the block; every thread gets the total.  ws: 33 entries.
template <class V>
__device__ V block_scan(V v, V* ws, V& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    V x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) ws[warp] = x;
    __syncthreads();
    if (warp == 0) {
        V s = lane < (int)(blockDim.x >> 5) ? ws[lane] : V(0);
        const V own = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const V y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        ws[lane] = s - own;
        if (lane == 31) ws[32] = s;
    }
    __syncthreads();
    const V r = ws[warp] + x - v;
    total = ws[32];
    __syncthreads();
    return r;
}

// Largest i in [0, n) with off[i] <= x (off ascending, off[0] <= x).
template <class V>
__device__ __forceinline__ int find_le(const V* off, int n, V x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (off[m] <= x) lo = m;
        else hi = m;
    }
    return lo;
}

// Free pages (ref == 0) in [from, to), ascending, the first `want` of them into
// list; returns how many were written.  with_live: pages in use instead.
__device__ int collect_pages(const int* ref, int from, int to, bool live, int want, int* list, int stride, int* ws) {
    int found = 0;
    for (int b = from; b < to && found < want; b += kStepThreads * 4) {
        const int p0 = b + threadIdx.x * 4;
        bool f[4];
        int cnt = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            f[u] = p0 + u < to && (ref[p0 + u] > 0) == live;
            cnt += f[u];
        }
        int total;
        int at = found + block_scan(cnt, ws, total);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (f[u]) {
                if (at < want) list[(size_t)at * stride] = p0 + u;
                ++at;
            }
        found += total;
    }
    return min(found, want);
}

// One block: room for the new tokens and the work list (see the header for the
// rules).  A thread takes one listed sequence, then one taken page, then one
// group at a time.
template <int N>
__global__ void __launch_bounds__(kStepThreads) cache_step_kernel(const __grid_constant__ CacheDev c,
                                                                  const __grid_constant__ CacheList<N> l) {
    __shared__ int s_pages[kCacheMaxSeqs + 1], s_groups[kCacheMaxSeqs + 1];
    __shared__ int s_len[kCacheMaxSeqs], s_last[kCacheMaxSeqs], s_cow[kCacheMaxSeqs];
    __shared__ long long s_pre[kStepThreads], s_wsl[33];
    __shared__ int s_ws[33], s_bad, s_most, s_bucket[kStepThreads];
    pdl_wait();
    pdl_trigger();
    const int i = threadIdx.x, n = l.n, TT = c.tile_tokens;
    if (i == 0) s_bad = 0;
    __syncthreads();
    int len = 0, q = 0, seq = 0, had = 0, last = -1, cow = 0, fresh = 0;
    if (i < n) {
        seq = l.a[i];
        q = l.b[i];
        len = c.length[seq];
        if (len < 0 || len > (long long)c.max_pages * c.page) {
            s_bad = ERR_CACHE_STATE;
            len = 0;
        }
        had = (int)(((long long)len + c.page - 1) >> c.page_shift);
        const long long need = ((long long)len + q + c.page - 1) >> c.page_shift;
        if (need > c.max_pages) s_bad = ERR_CACHE_FULL;
        if (had > 0) {
            last = c.table[(size_t)seq * c.max_pages + had - 1];
            if (last < 0 || last >= c.n_pages) {
                s_bad = ERR_CACHE_STATE;
                last = -1;
            }
        }
        cow = q > 0 && (len & (c.page - 1)) && last >= 0 && c.ref[last] > 1;
        fresh = (int)min(need - had, (long long)c.max_pages) + cow;
    }
    int n_fresh, T, n_groups, n_cow;
    const int at_page = block_scan(fresh, s_ws, n_fresh);
    const int at_tok = block_scan(q, s_ws, T);
    const int at_group = block_scan((q + 2 * TT - 1) / (2 * TT), s_ws, n_groups);
    const int at_cow = block_scan(cow, s_ws, n_cow);
    if (i < n) {
        s_pages[i] = at_page;
        s_groups[i] = at_group;
        s_len[i] = len;
        s_last[i] = last;
        s_cow[i] = cow ? at_cow : -1;
    }
    __syncthreads();
    if (!s_bad) {
        const int found = collect_pages(c.ref, 0, c.n_pages, false, n_fresh, c.fresh, 1, s_ws);
        if (found < n_fresh && i == 0) s_bad = ERR_CACHE_FULL;
    }
    __syncthreads();
    if (s_bad) {
        if (i == 0) {
            *c.plan = CachePlan{};
            atomicCAS(c.err, 0, s_bad);
        }
        return;
    }
    // Pages: the k-th taken page belongs to the sequence whose range holds k.
    for (int k = i; k < n_fresh; k += kStepThreads) {
        const int s = find_le(s_pages, n, k);
        const int id = c.fresh[k];
        const int copied = s_cow[s] >= 0;
        const int first = (int)(((long long)s_len[s] + c.page - 1) >> c.page_shift) - copied;
        const int j = first + k - s_pages[s];
        if (copied && k == s_pages[s]) {
            c.copies[s_cow[s]] = make_int2(s_last[s], id);
            atomicSub(&c.ref[s_last[s]], 1);
        }
        c.table[(size_t)l.a[s] * c.max_pages + j] = id;
        c.ref[id] = 1;
    }
    if (i < n) {
        c.length[seq] = len + q;
        c.base[seq] = len;
        c.seqs[i] = CacheSeq{seq, at_tok, q, len + q};
    }
    __syncthreads();   // s_pages has been read: it takes the token offsets
    if (i < n) s_pages[i] = at_tok;
    __syncthreads();
    // The work list.  Groups are numbered in the order of the sequences; when whole
    // items will be drawn (below), they are stored longest first.
    auto group_of = [&](int r) {
        CacheGroup g;
        const int s = find_le(s_groups, n, r);
        const int q_len = l.b[s], tok = (r - s_groups[s]) * 2 * TT;
        g.seq = l.a[s];
        g.kv_len = s_len[s] + q_len;
        g.row = s_pages[s] + tok;
        g.ntok = min(2 * TT, q_len - tok);
        g.first = s_len[s] + tok;
        g.base = s_len[s];
        g.cost = (cache_group_tiles(q_len, g.kv_len, g.first, g.ntok) + 1) << cache_two_tiles(g.ntok, TT);
        g.pre = 0;
        return g;
    };
    long long cost = 0, total;
    int most = 0, two = 0;
    for (int r = i; r < n_groups; r += kStepThreads) {
        const CacheGroup g = group_of(r);
        cost += g.cost;
        most = max(most, g.cost);
        two |= cache_two_tiles(g.ntok, TT);
    }
    block_scan(cost, s_wsl, total);
    if (i == 0) s_most = 0;
    two = __syncthreads_or(two);
    if (i < n_groups) atomicMax(&s_most, most);
    __syncthreads();
    const long long W = total * c.Hkv;
    const bool whole = 2LL * s_most * c.num_sms <= W;
    const int n_ctas = !W || whole ? 0 : (int)max(1LL, min((long long)c.num_sms, W / (kMinTiles << (two ? 1 : 0))));
    if (whole) {
        // Counting sort by cost, costs past the last bucket together in the first one.
        if (i < kStepThreads) s_bucket[i] = 0;
        __syncthreads();
        for (int r = i; r < n_groups; r += kStepThreads) atomicAdd(&s_bucket[max(0, kStepThreads - 1 - group_of(r).cost)], 1);
        __syncthreads();
        int all;
        const int at = block_scan(s_bucket[i], s_ws, all);
        s_bucket[i] = at;
        __syncthreads();
        for (int r = i; r < n_groups; r += kStepThreads) {
            const CacheGroup g = group_of(r);
            c.groups[atomicAdd(&s_bucket[max(0, kStepThreads - 1 - g.cost)], 1)] = g;
        }
    } else {
        long long before = 0;
        for (int b = 0; b < n_groups; b += kStepThreads) {
            const int r = b + i;
            CacheGroup g;
            if (r < n_groups) g = group_of(r);
            long long sum;
            const long long pre = before + block_scan(r < n_groups ? (long long)g.cost : 0LL, s_wsl, sum);
            if (r < n_groups) {
                g.pre = pre;
                c.groups[r] = g;
                if (n_groups <= kStepThreads) s_pre[r] = pre;
            }
            before += sum;
        }
    }
    if (i == 0) *c.plan = CachePlan{W, n_groups, n_ctas, n_cow, 1, 0, 0};
    __syncthreads();
    for (int b = i; b < n_ctas; b += kStepThreads) {
        CacheShare sh;
        sh.begin = W * b / n_ctas;
        sh.end = W * (b + 1) / n_ctas;
        const long long x = sh.begin / c.Hkv;
        if (n_groups <= kStepThreads) {
            sh.group = find_le(s_pre, n_groups, x);
        } else {
            int lo = 0, hi = n_groups;
            while (hi - lo > 1) {
                const int m = (lo + hi) >> 1;
                if (c.groups[m].pre <= x) lo = m;
                else hi = m;
            }
            sh.group = lo;
        }
        sh.g = c.groups[sh.group];
        sh.within = sh.begin - sh.g.pre * c.Hkv;
        sh.head = (int)(sh.within / sh.g.cost);
        sh.within -= (long long)sh.head * sh.g.cost;
        // The CTAs that hold tiles of the item: every share covers at least one unless it
        // holds just the item's end.
        const long long start = sh.begin - sh.within;
        const int two_tiles = cache_two_tiles(sh.g.ntok, TT), tiles = cache_item_tiles(sh.g.cost, two_tiles);
        sh.first = sh.last = b;
        while (W * sh.first / n_ctas > start) --sh.first;
        while (cache_tiles_before(W * (sh.last + 1) / n_ctas - start, sh.g.cost, two_tiles) < tiles) ++sh.last;
        while (cache_tiles_before(W * sh.last / n_ctas - start, sh.g.cost, two_tiles) == tiles) --sh.last;
        c.shares[b] = sh;
    }
    if (i < c.num_sms) c.arrived[i] = 0;
}

// Page rows and positions of the T new tokens, and the page copies that the
// preceding kernel listed (all layers, K and V).
__global__ void __launch_bounds__(kCopyThreads) cache_fill_kernel(const __grid_constant__ CacheDev c, int n, int T) {
    pdl_wait();
    pdl_trigger();
    const int ok = c.plan->ok, copies = c.plan->copies;
    for (int t = blockIdx.x * kCopyThreads + threadIdx.x; t < T; t += gridDim.x * kCopyThreads) {
        int slot = -1, pos = 0;
        if (ok) {
            int lo = 0, hi = n;
            while (hi - lo > 1) {
                const int m = (lo + hi) >> 1;
                if (c.seqs[m].q_off <= t) lo = m;
                else hi = m;
            }
            const CacheSeq s = c.seqs[lo];
            pos = s.kv_len - s.q_len + (t - s.q_off);
            slot = (c.table[(size_t)s.seq * c.max_pages + (pos >> c.page_shift)] << c.page_shift) +
                   (pos & (c.page - 1));
        }
        c.slot[t] = slot;
        c.pos[t] = pos;
    }
    const size_t vecs = (size_t)c.Hkv * c.page * c.dh / 8;      // 16-byte vectors of a page in one layer
    constexpr int kPart = kCopyThreads * kCopyVecs;
    const int parts = (int)((vecs + kPart - 1) / kPart);
    const long long units = (long long)copies * c.layers * 2 * parts;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int part = (int)(u % parts);
        const long long blk = u / parts;
        const int kv = (int)(blk & 1), layer = (int)((blk >> 1) % c.layers), i = (int)((blk >> 1) / c.layers);
        const int2 cp = c.copies[i];
        uint4* pool = reinterpret_cast<uint4*>(kv ? c.v : c.k) + (size_t)layer * c.n_pages * vecs;
        const uint4* src = pool + (size_t)cp.x * vecs;
        uint4* dst = pool + (size_t)cp.y * vecs;
        const size_t v0 = (size_t)part * kPart + threadIdx.x;
        uint4 r[kCopyVecs];
#pragma unroll
        for (int w = 0; w < kCopyVecs; ++w)
            if (v0 + w * kCopyThreads < vecs) r[w] = src[v0 + w * kCopyThreads];
#pragma unroll
        for (int w = 0; w < kCopyVecs; ++w)
            if (v0 + w * kCopyThreads < vecs) dst[v0 + w * kCopyThreads] = r[w];
    }
}

// A thread takes one table entry of one continuation.
template <int N>
__global__ void __launch_bounds__(256) cache_fork_kernel(const __grid_constant__ CacheDev c,
                                                         const __grid_constant__ CacheList<N> l) {
    pdl_wait();
    pdl_trigger();
    const long long entries = (long long)l.n * c.max_pages;
    for (long long e = blockIdx.x * 256LL + threadIdx.x; e < entries; e += gridDim.x * 256LL) {
        const int i = (int)(e / c.max_pages), j = (int)(e - (long long)i * c.max_pages);
        const int src = l.a[i], dst = l.b[i];
        int* to = &c.table[(size_t)dst * c.max_pages + j];
        const int was = *to, now = c.table[(size_t)src * c.max_pages + j];
        if (was >= c.n_pages || now >= c.n_pages) atomicCAS(c.err, 0, ERR_CACHE_STATE);
        if (was != now) {
            if (was >= 0 && was < c.n_pages) atomicSub(&c.ref[was], 1);
            if (now >= 0 && now < c.n_pages) atomicAdd(&c.ref[now], 1);
            *to = now;
        }
        if (j == 0) {
            const int len = c.length[src];
            c.length[dst] = len;
            c.base[dst] = len;
        }
    }
}

// A thread takes one table entry of one sequence.  accepted: the new lengths
// come from the accept kernel (-1: leave the sequence) instead of the list.
template <int N>
__global__ void __launch_bounds__(256) cache_cut_kernel(const __grid_constant__ CacheDev c,
                                                        const __grid_constant__ CacheList<N> l, const int* accepted) {
    pdl_wait();
    pdl_trigger();
    const long long entries = (long long)l.n * c.max_pages;
    for (long long e = blockIdx.x * 256LL + threadIdx.x; e < entries; e += gridDim.x * 256LL) {
        const int i = (int)(e / c.max_pages), j = (int)(e - (long long)i * c.max_pages);
        const int s = l.a[i];
        // length[s] may already hold the cut value here: the smaller of the two is the same.
        const int len = accepted ? accepted[i] : max(0, min(l.b[i], c.length[s]));
        if (len < 0) continue;
        int* at = &c.table[(size_t)s * c.max_pages + j];
        if (j >= (int)(((long long)len + c.page - 1) >> c.page_shift)) {
            const int id = *at;
            if (id >= c.n_pages) atomicCAS(c.err, 0, ERR_CACHE_STATE);
            if (id >= 0 && id < c.n_pages) atomicSub(&c.ref[id], 1);
            if (id != -1) *at = -1;
        }
        if (j == 0) {
            c.length[s] = len;
            c.base[s] = accepted ? len : min(c.base[s], len);
        }
    }
}

// Moves the accepted drafts to the front.  dh / 8 lanes take the rows of one
// (sequence, layer, K or V, head), each lane its own 16 bytes of every row, in
// the order of the path: row e is written after rows e .. e + 3 were read, and
// later rows come from behind (path[e] >= e), so rows may overlap.
template <int N>
__global__ void __launch_bounds__(256) cache_accept_kernel(const __grid_constant__ CacheDev c,
                                                           const __grid_constant__ CacheList<N> l, const int* n_acc,
                                                           const int* path, int ld_path, int* accepted) {
    pdl_wait();
    pdl_trigger();
    const int lanes = c.dh >> 3;                 // 8 or 16, a divisor of the warp
    const int lane = threadIdx.x & 31, sub = lane & (lanes - 1);
    const uint32_t mask = (lanes == 16 ? 0xffffu : 0xffu) << (lane & ~(lanes - 1));
    const long long units = (long long)l.n * c.layers * 2 * c.Hkv;
    const long long per = 256 / lanes;
    const size_t page_elems = (size_t)c.Hkv * c.page * c.dh;
    for (long long u0 = blockIdx.x * per; u0 < units; u0 += gridDim.x * per) {
        const long long u = u0 + threadIdx.x / lanes;
        bool ok = true;
        int i = 0, h = 0, kv = 0, layer = 0, seq = 0, base = 0, n = 0;
        const int* mine = path;
        if (u < units) {
            h = (int)(u % c.Hkv);
            const long long v = u / c.Hkv;
            kv = (int)(v & 1);
            layer = (int)((v >> 1) % c.layers);
            i = (int)((v >> 1) / c.layers);
            seq = l.a[i];
            base = c.base[seq];
            const int drafts = c.length[seq] - base;
            n = n_acc[i];
            mine = path + (size_t)i * ld_path;
            if (base < 0 || drafts < 0 || (long long)base + drafts > (long long)c.max_pages * c.page || n < 0 ||
                n > min(min(drafts, kTreeMax), ld_path)) {
                ok = false;
                n = 0;
            }
            for (int e = sub; e < n; e += lanes) {
                const int from = mine[e];
                ok &= from >= 0 && from < drafts && (e == 0 || from > mine[e - 1]);
                const int to_id = c.table[(size_t)seq * c.max_pages + ((base + e) >> c.page_shift)];
                ok &= to_id >= 0 && to_id < c.n_pages && c.ref[to_id] == 1;
                if (ok) {
                    const int id = c.table[(size_t)seq * c.max_pages + ((base + from) >> c.page_shift)];
                    ok &= id >= 0 && id < c.n_pages;
                }
            }
        }
        ok = (__ballot_sync(0xffffffffu, !ok) & mask) == 0;
        if (u >= units) continue;
        if (layer == 0 && kv == 0 && h == 0 && sub == 0) {
            accepted[i] = ok ? base + n : -1;
            if (!ok) atomicCAS(c.err, 0, ERR_CACHE_PATH);
        }
        if (!ok) continue;
        __nv_bfloat16* pool = (kv ? c.v : c.k) + ((size_t)layer * c.n_pages) * page_elems + (size_t)h * c.page * c.dh;
        auto row = [&](int p) {
            const int id = c.table[(size_t)seq * c.max_pages + (p >> c.page_shift)];
            return reinterpret_cast<uint4*>(pool + (size_t)id * page_elems + (size_t)(p & (c.page - 1)) * c.dh) + sub;
        };
        for (int e0 = 0; e0 < n; e0 += 4) {
            uint4 r[4];
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if (e0 + w < n && mine[e0 + w] != e0 + w) r[w] = *row(base + mine[e0 + w]);
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if (e0 + w < n && mine[e0 + w] != e0 + w) *row(base + e0 + w) = r[w];
        }
    }
}

// One block: pairs the pages in use past the number in use with the free ones
// below it, both ascending; plan->total is that number, fresh[] the new places.
__global__ void __launch_bounds__(kStepThreads) cache_compact_kernel(const __grid_constant__ CacheDev c) {
    __shared__ int s_ws[33];
    pdl_wait();
    pdl_trigger();
    int mine = 0, live;
    for (int p = threadIdx.x; p < c.n_pages; p += kStepThreads) mine += c.ref[p] > 0;
    block_scan(mine, s_ws, live);
    const int holes = collect_pages(c.ref, 0, live, false, live, &c.copies[0].y, 2, s_ws);
    const int movers = collect_pages(c.ref, live, c.n_pages, true, holes, &c.copies[0].x, 2, s_ws);
    __syncthreads();
    for (int k = threadIdx.x; k < movers; k += kStepThreads) c.fresh[c.copies[k].x] = c.copies[k].y;
    if (threadIdx.x == 0) *c.plan = CachePlan{live, 0, 0, movers, 0, 0, 0};
}

// Tables and counts follow the moved pages.
__global__ void __launch_bounds__(256) cache_remap_kernel(const __grid_constant__ CacheDev c) {
    pdl_wait();
    pdl_trigger();
    const int live = (int)c.plan->total;
    const long long entries = (long long)c.max_seqs * c.max_pages;
    const long long at = blockIdx.x * 256LL + threadIdx.x, step = gridDim.x * 256LL;
    for (long long e = at; e < entries; e += step) {
        const int id = c.table[e];
        if (id >= live && id < c.n_pages) {
            if (c.ref[id] > 0) c.table[e] = c.fresh[id];
            else atomicCAS(c.err, 0, ERR_CACHE_STATE);
        }
    }
}

__global__ void __launch_bounds__(256) cache_recount_kernel(const __grid_constant__ CacheDev c) {
    pdl_wait();
    pdl_trigger();
    const int moved = c.plan->copies;
    for (int k = blockIdx.x * 256 + threadIdx.x; k < moved; k += gridDim.x * 256) {
        const int2 cp = c.copies[k];
        c.ref[cp.y] = c.ref[cp.x];
        c.ref[cp.x] = 0;
    }
}

template <int N>
CacheList<N> list_of(int n, const int* a, const int* b) {
    CacheList<N> l;
    l.n = n;
    std::copy(a, a + n, l.a);
    if (b) std::copy(b, b + n, l.b);
    return l;
}

unsigned entry_blocks(const CacheDev& c, long long entries) {
    return (unsigned)std::max<long long>(1, std::min<long long>((entries + 255) / 256, c.num_sms * 8));
}

// Small lists travel in small parameter blocks (a launch copies them).
constexpr int kShortList = 64;

template <int N>
cudaError_t step_launch(const CacheDev& c, int n, const int* seq, const int* q_len, cudaStream_t st) {
    return launch_pdl(cache_step_kernel<N>, dim3(1), dim3(kStepThreads), 0, st, c, list_of<N>(n, seq, q_len));
}

}  // namespace

cudaError_t launch_cache_step(const CacheDev& c, int n, const int* seq, const int* q_len, int T, cudaStream_t st) {
    cudaError_t e = n <= kShortList ? step_launch<kShortList>(c, n, seq, q_len, st)
                                    : step_launch<kCacheMaxSeqs>(c, n, seq, q_len, st);
    if (e != cudaSuccess) return e;
    return launch_pdl(cache_fill_kernel, dim3(c.num_sms * 6), dim3(kCopyThreads), 0, st, c, n, T);
}

cudaError_t launch_cache_fork(const CacheDev& c, int n, const int* src, const int* dst, cudaStream_t st) {
    const dim3 grid(entry_blocks(c, (long long)n * c.max_pages));
    if (n <= kShortList)
        return launch_pdl(cache_fork_kernel<kShortList>, grid, dim3(256), 0, st, c, list_of<kShortList>(n, src, dst));
    return launch_pdl(cache_fork_kernel<kCacheMaxSeqs>, grid, dim3(256), 0, st, c, list_of<kCacheMaxSeqs>(n, src, dst));
}

cudaError_t launch_cache_truncate(const CacheDev& c, int n, const int* seq, const int* length, cudaStream_t st) {
    const dim3 grid(entry_blocks(c, (long long)n * c.max_pages));
    const int* none = nullptr;
    if (n <= kShortList)
        return launch_pdl(cache_cut_kernel<kShortList>, grid, dim3(256), 0, st, c,
                          list_of<kShortList>(n, seq, length), none);
    return launch_pdl(cache_cut_kernel<kCacheMaxSeqs>, grid, dim3(256), 0, st, c,
                      list_of<kCacheMaxSeqs>(n, seq, length), none);
}

namespace {
template <int N>
cudaError_t accept_launch(const CacheDev& c, int n, const int* seq, const int* n_acc, const int* path, int ld_path,
                          cudaStream_t st) {
    int* accepted = reinterpret_cast<int*>(c.copies);
    const CacheList<N> l = list_of<N>(n, seq, nullptr);
    const long long per = 256 / (c.dh / 8), units = (long long)n * c.layers * 2 * c.Hkv;
    const dim3 grid((unsigned)std::min<long long>((units + per - 1) / per, c.num_sms * 16));
    cudaError_t e = launch_pdl(cache_accept_kernel<N>, grid, dim3(256), 0, st, c, l, n_acc, path, ld_path, accepted);
    if (e != cudaSuccess) return e;
    return launch_pdl(cache_cut_kernel<N>, dim3(entry_blocks(c, (long long)n * c.max_pages)), dim3(256), 0, st, c, l,
                      (const int*)accepted);
}
}  // namespace

cudaError_t launch_cache_accept(const CacheDev& c, int n, const int* seq, const int* n_acc, const int* path,
                                int ld_path, cudaStream_t st) {
    return n <= kShortList ? accept_launch<kShortList>(c, n, seq, n_acc, path, ld_path, st)
                           : accept_launch<kCacheMaxSeqs>(c, n, seq, n_acc, path, ld_path, st);
}

cudaError_t launch_cache_compact(const CacheDev& c, cudaStream_t st) {
    cudaError_t e = launch_pdl(cache_compact_kernel, dim3(1), dim3(kStepThreads), 0, st, c);
    if (e == cudaSuccess) e = launch_pdl(cache_fill_kernel, dim3(c.num_sms * 6), dim3(kCopyThreads), 0, st, c, 0, 0);
    if (e == cudaSuccess)
        e = launch_pdl(cache_remap_kernel, dim3(entry_blocks(c, (long long)c.max_seqs * c.max_pages)), dim3(256), 0,
                       st, c);
    if (e == cudaSuccess)
        e = launch_pdl(cache_recount_kernel, dim3(entry_blocks(c, c.n_pages)), dim3(256), 0, st, c);
    return e;
}

}  // namespace tmoe
