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
// Bounds: the bookkeeping reads a few kB and is a chain of dependent reads and block-wide
// scans in one block (a step of 24 to 40 sequences 7 to 9 us, launched apart and cold);
// page copies move 2 x layers x kv_heads x page_size x head_dim x 2 bytes each way per page
// and are bound by HBM (24 pages of 64 tokens in 32 layers, 8 heads of 128: 201 MB written
// in 36 us, 5.6 TB/s).  Moving accepted drafts is a chain too: path, table, rows (40
// sequences, 24 layers, 16 heads: 13 us, cold).
#include <algorithm>

#include "cache.cuh"

namespace tmoe {

namespace {

constexpr int kStepThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kCopyVecs = 4;           // 16-byte vectors in flight per thread
// Smallest share of a CTA, in key tiles: below it, fewer CTAs take part.  Two tiles
// keep both slots busy at once (one sequence of 1500 positions took 11.5 us so, 15.7 with
// three and more CTAs idle).
constexpr int kMinTiles = 2;

__device__ __forceinline__ int from_below(int v, int o) { return __shfl_up_sync(0xffffffffu, v, o); }
__device__ __forceinline__ long long from_below(long long v, int o) { return __shfl_up_sync(0xffffffffu, v, o); }

// Four sums scanned together.
struct Sums {
    int fresh, tok, group, cow;
    Sums() = default;
    __device__ explicit Sums(int v) : fresh(v), tok(v), group(v), cow(v) {}
    __device__ Sums(int a, int b, int c, int d) : fresh(a), tok(b), group(c), cow(d) {}
    __device__ Sums operator+(const Sums& o) const {
        return Sums(fresh + o.fresh, tok + o.tok, group + o.group, cow + o.cow);
    }
    __device__ Sums operator-(const Sums& o) const {
        return Sums(fresh - o.fresh, tok - o.tok, group - o.group, cow - o.cow);
    }
};
__device__ __forceinline__ Sums from_below(const Sums& v, int o) {
    return Sums(__shfl_up_sync(0xffffffffu, v.fresh, o), __shfl_up_sync(0xffffffffu, v.tok, o),
                __shfl_up_sync(0xffffffffu, v.group, o), __shfl_up_sync(0xffffffffu, v.cow, o));
}

// Exclusive prefix sum over the block; every thread gets the total.  ws: 33 entries.
template <class V>
__device__ V block_scan(V v, V* ws, V& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    V x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V y = from_below(x, o);
        if (lane >= o) x = x + y;
    }
    if (lane == 31) ws[warp] = x;
    __syncthreads();
    if (warp == 0) {
        V s = lane < (int)(blockDim.x >> 5) ? ws[lane] : V(0);
        const V own = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const V y = from_below(s, o);
            if (lane >= o) s = s + y;
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

// A page that compaction may move: in use, and by sequences alone (holders: its entries in
// the table).  Who holds it besides knows it by its index.
__device__ __forceinline__ bool movable(int ref, int holders) { return ref > 0 && ref <= holders; }

// Which of a thread's four pages p0 .. p0 + 3 below `to` are free (holders: movable
// instead), a bit each.
__device__ __forceinline__ uint32_t four_pages(const int* ref, const int* holders, int p0, int to) {
    uint32_t f = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (p0 + u < to && (holders ? movable(ref[p0 + u], holders[p0 + u]) : ref[p0 + u] <= 0)) f |= 1u << u;
    return f;
}

// Free (holders: movable) pages in [from, to), ascending: put(k, page) for the first
// `want` of them; returns how many there were, up to that.  first: this thread's
// four_pages() at from + 4 threadIdx.x, which the caller may read early.
template <class Put>
__device__ int collect_pages(const int* ref, const int* holders, int from, int to, int want, uint32_t first, int* ws,
                             Put put) {
    int found = 0;
    for (int b = from; b < to && found < want; b += kStepThreads * 4) {
        const int p0 = b + threadIdx.x * 4;
        const uint32_t f = b == from ? first : four_pages(ref, holders, p0, to);
        int total;
        int at = found + block_scan(__popc(f), ws, total);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (f >> u & 1u) {
                if (at < want) put(at, p0 + u);
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
    __shared__ int s_seq[kCacheMaxSeqs], s_q[kCacheMaxSeqs], s_len[kCacheMaxSeqs], s_last[kCacheMaxSeqs];
    __shared__ int s_pages[kCacheMaxSeqs], s_tok[kCacheMaxSeqs], s_groups[kCacheMaxSeqs], s_cow[kCacheMaxSeqs];
    __shared__ int s_fresh[kStepThreads];
    __shared__ long long s_pre[kStepThreads], s_wsl[33];
    __shared__ Sums s_wss[33];
    __shared__ int s_ws[33], s_bad, s_most;
    const int i = threadIdx.x, n = l.n, TT = c.tile_tokens;
    int q = 0, seq = 0;
    if (i < n) {
        s_seq[i] = seq = l.a[i];
        s_q[i] = q = l.b[i];
    }
    if (i == 0) s_bad = s_most = 0;
    pdl_wait();
    pdl_trigger();
    const uint32_t free4 = four_pages(c.ref, nullptr, i * 4, c.n_pages);      // (on its way beside the lengths)
    const int serial = c.plan->serial;
    int len = i < n ? c.length[seq] : 0;
    __syncthreads();
    int had = 0, last = -1, cow = 0, fresh = 0;
    if (i < n) {
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
    Sums sum;
    const Sums at = block_scan(Sums(fresh, q, (q + 2 * TT - 1) / (2 * TT), cow), s_wss, sum);
    const int n_fresh = sum.fresh, n_groups = sum.group;
    if (i < n) {
        s_pages[i] = at.fresh;
        s_tok[i] = at.tok;
        s_groups[i] = at.group;
        s_len[i] = len;
        s_last[i] = last;
        s_cow[i] = cow ? at.cow : -1;
    }
    __syncthreads();
    if (!s_bad && n_fresh > 0) {
        // (Shared memory holds as many as it has room for.)
        const int found = collect_pages(c.ref, nullptr, 0, c.n_pages, n_fresh, free4, s_ws, [&](int k, int page) {
            (k < kStepThreads ? s_fresh : c.fresh)[k] = page;
        });
        if (found < n_fresh && i == 0) s_bad = ERR_CACHE_FULL;
        __syncthreads();
    }
    if (s_bad) {
        if (i == 0) {
            CachePlan none{};
            none.serial = serial + 1;
            *c.plan = none;
            atomicCAS(c.err, 0, s_bad);
            *c.refused = 1;
        }
        return;
    }
    // Pages: the k-th taken page belongs to the sequence whose range holds k.
    for (int k = i; k < n_fresh; k += kStepThreads) {
        const int s = find_le(s_pages, n, k);
        const int id = (k < kStepThreads ? s_fresh : c.fresh)[k];
        const int copied = s_cow[s] >= 0;
        const int first = (int)(((long long)s_len[s] + c.page - 1) >> c.page_shift) - copied;
        const int j = first + k - s_pages[s];
        if (copied && k == s_pages[s]) {
            c.copies[s_cow[s]] = make_int2(s_last[s], id);
            atomicSub(&c.ref[s_last[s]], 1);
        }
        c.table[(size_t)s_seq[s] * c.max_pages + j] = id;
        c.ref[id] = 1;
    }
    if (i < n) {
        c.length[seq] = len + q;
        c.base[seq] = len;
        c.seqs[i] = CacheSeq{seq, at.tok, q, len + q};
    }
    // The work list.  Groups are numbered in the order of the sequences; when whole
    // items will be drawn (below), they are stored longest first.
    auto group_of = [&](int r) {
        CacheGroup g;
        const int s = find_le(s_groups, n, r);
        const int q_len = s_q[s], tok = (r - s_groups[s]) * 2 * TT;
        g.seq = s_seq[s];
        g.kv_len = s_len[s] + q_len;
        g.row = s_tok[s] + tok;
        g.ntok = min(2 * TT, q_len - tok);
        g.first = s_len[s] + tok;
        g.base = s_len[s];
        g.cost = (cache_group_tiles(q_len, g.kv_len, g.first, g.ntok) + 1) << cache_two_tiles(g.ntok, TT);
        g.pre = 0;
        return g;
    };
    const bool few = n_groups <= kStepThreads;           // a thread has one group at most
    CacheGroup mine;
    long long cost = 0, total;
    int most = 0, two = 0;
    for (int r = i; r < n_groups; r += kStepThreads) {
        mine = group_of(r);
        cost += mine.cost;
        most = max(most, mine.cost);
        two |= cache_two_tiles(mine.ntok, TT);
    }
    if (i < n_groups) atomicMax(&s_most, most);
    const long long before_mine = block_scan(cost, s_wsl, total);
    two = __syncthreads_or(two);
    const long long W = total * c.Hkv;
    // Whole items from two of the largest per CTA on.  Neither side is better throughout: with
    // equal items a last turn that few CTAs have costs more than cutting them, with the
    // mixed ones of prompts it does not.  Factor 1 / 2 / 4 / never whole: 20 equal contexts
    // of 4000 (160 items) 83 / 59 / 59 / 59 us, 39 of them 125 / 125 / 104 / 104, 40 of 900
    // at 12 heads 46 / 46 / 54 / 54; 5 prompts of 1000 61 / 61 / 93 / 93, one of 4096
    // 118 / 165 / 165 / 165, chunks behind prefixes 207 / 219 / 219 / 219.
    const bool whole = 2LL * s_most * c.num_sms <= W;
    const int n_ctas = !W || whole ? 0 : (int)max(1LL, min((long long)c.num_sms, W / (kMinTiles << (two ? 1 : 0))));
    if (whole) {
        // Counting sort by cost, costs past the last bucket together in the first one.
        auto bucket = [](int cost) { return max(0, kStepThreads - 1 - cost); };
        int* s_bucket = s_fresh;                         // (the pages have been given out)
        s_bucket[i] = 0;
        __syncthreads();
        for (int r = i; r < n_groups; r += kStepThreads) atomicAdd(&s_bucket[bucket(few ? mine.cost : group_of(r).cost)], 1);
        __syncthreads();
        int all;
        const int start = block_scan(s_bucket[i], s_ws, all);
        s_bucket[i] = start;
        __syncthreads();
        for (int r = i; r < n_groups; r += kStepThreads) {
            const CacheGroup g = few ? mine : group_of(r);
            c.groups[atomicAdd(&s_bucket[bucket(g.cost)], 1)] = g;
        }
    } else if (few) {
        if (i < n_groups) {
            mine.pre = s_pre[i] = before_mine;
            c.groups[i] = mine;
        }
    } else {
        long long before = 0;
        for (int b = 0; b < n_groups; b += kStepThreads) {
            const int r = b + i;
            CacheGroup g;
            if (r < n_groups) g = group_of(r);
            long long part;
            const long long pre = before + block_scan(r < n_groups ? (long long)g.cost : 0LL, s_wsl, part);
            if (r < n_groups) {
                g.pre = pre;
                c.groups[r] = g;
            }
            before += part;
        }
    }
    if (i == 0) {
        *c.plan = CachePlan{W, n_groups, n_ctas, sum.cow, 1, 0, 0, 0, serial + 1};
        *c.refused = 0;
    }
    __syncthreads();
    for (int b = i; b < n_ctas; b += kStepThreads) {
        CacheShare sh;
        sh.begin = W * b / n_ctas;
        sh.end = W * (b + 1) / n_ctas;
        const long long x = sh.begin / c.Hkv;
        if (few) {
            sh.group = find_le(s_pre, n_groups, x);
            sh.g = group_of(sh.group);
            sh.g.pre = s_pre[sh.group];
        } else {
            int lo = 0, hi = n_groups;
            while (hi - lo > 1) {
                const int m = (lo + hi) >> 1;
                if (c.groups[m].pre <= x) lo = m;
                else hi = m;
            }
            sh.group = lo;
            sh.g = c.groups[lo];
        }
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
        int slot = -1, pos = 0, owner = 0;
        if (ok) {
            int lo = 0, hi = n;
            while (hi - lo > 1) {
                const int m = (lo + hi) >> 1;
                if (c.seqs[m].q_off <= t) lo = m;
                else hi = m;
            }
            const CacheSeq s = c.seqs[owner = lo];
            pos = s.kv_len - s.q_len + (t - s.q_off);
            slot = (c.table[(size_t)s.seq * c.max_pages + (pos >> c.page_shift)] << c.page_shift) +
                   (pos & (c.page - 1));
            c.tokens[t] = CacheToken{s.seq, s.kv_len, s.kv_len - s.q_len, pos};
        }
        c.slot[t] = slot;
        c.pos[t] = pos;
        c.owner[t] = owner;
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
    if (!c.codes) return;
    // The pages' bounds (a page that a step copies is not full and has none yet).
    const size_t words = (size_t)c.Hkv * c.dh / 2;              // 4-byte words of a page's codes in one layer
    for (long long u = blockIdx.x; u < (long long)copies * c.layers; u += gridDim.x) {
        const int2 cp = c.copies[u / c.layers];
        const size_t first = (size_t)(u % c.layers) * c.n_pages;
        uint32_t* codes = reinterpret_cast<uint32_t*>(c.codes);
        for (size_t w = threadIdx.x; w < words; w += kCopyThreads)
            codes[(first + cp.y) * words + w] = codes[(first + cp.x) * words + w];
        for (int h = threadIdx.x; h < c.Hkv; h += kCopyThreads)
            c.scales[(first + cp.y) * c.Hkv + h] = c.scales[(first + cp.x) * c.Hkv + h];
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

// Moves the accepted drafts to the front.  dh / 8 lanes take the K and V rows of one
// (sequence, layer, head), each lane its own 16 bytes of every row, in the order of the
// path: row e is written after rows e .. e + 3 were read, and later rows come from
// behind (path[e] >= e), so rows may overlap.  Lane e looks up the e-th row's pages once,
// for the check and for the move (and again for paths longer than the lanes).  Behind a
// refused step nothing fits: base is that of the step before, whose tokens are no drafts.
template <int N>
__global__ void __launch_bounds__(256) cache_accept_kernel(const __grid_constant__ CacheDev c,
                                                           const __grid_constant__ CacheList<N> l, const int* n_acc,
                                                           const int* path, int ld_path, int* accepted) {
    pdl_wait();
    pdl_trigger();
    const int lanes = c.dh >> 3;                 // 8 or 16, a divisor of the warp
    const int lane = threadIdx.x & 31, sub = lane & (lanes - 1);
    const uint32_t mask = (lanes == 16 ? 0xffffu : 0xffu) << (lane & ~(lanes - 1));
    const long long units = (long long)l.n * c.layers * c.Hkv;
    const long long per = 256 / lanes;
    const size_t page_elems = (size_t)c.Hkv * c.page * c.dh;
    for (long long u0 = blockIdx.x * per; u0 < units; u0 += gridDim.x * per) {
        const long long u = u0 + threadIdx.x / lanes;
        bool ok = true;
        int i = 0, h = 0, layer = 0, base = 0, n = 0;
        const int *mine = path, *table = c.table;
        int from = 0, from_id = 0, to_id = 0;    // of row e0 + sub
        if (u < units) {
            h = (int)(u % c.Hkv);
            layer = (int)(u / c.Hkv % c.layers);
            i = (int)(u / c.Hkv / c.layers);
            const int seq = l.a[i];
            base = c.base[seq];
            const int drafts = c.length[seq] - base;
            n = n_acc[i];
            mine = path + (size_t)i * ld_path;
            table = c.table + (size_t)seq * c.max_pages;
            if (*c.refused || base < 0 || drafts < 0 || (long long)base + drafts > (long long)c.max_pages * c.page || n < 0 ||
                n > min(min(drafts, kTreeMax), ld_path)) {
                ok = false;
                n = 0;
            }
            for (int e = sub; e < n; e += lanes) {
                const int f = mine[e], before = e ? mine[e - 1] : -1;
                const int t = table[(base + e) >> c.page_shift];
                bool fits = f > before && f < drafts && t >= 0 && t < c.n_pages;
                if (fits) {
                    const int id = table[(base + f) >> c.page_shift];
                    fits = id >= 0 && id < c.n_pages && c.ref[t] == 1;
                    if (e == sub) {
                        from = f;
                        from_id = id;
                        to_id = t;
                    }
                }
                ok &= fits;
            }
        }
        ok = (__ballot_sync(0xffffffffu, !ok) & mask) == 0;
        if (u < units && layer == 0 && h == 0 && sub == 0) {
            accepted[i] = ok ? base + n : -1;
            if (!ok) atomicCAS(c.err, 0, ERR_CACHE_PATH);
        }
        if (!ok) n = 0;
        const size_t off = (size_t)layer * c.n_pages * page_elems + (size_t)h * c.page * c.dh + sub * 8;
        for (int e0 = 0; e0 < n; e0 += lanes) {    // (n is the same for the unit's lanes)
            if (e0 && e0 + sub < n) {
                from = mine[e0 + sub];
                from_id = table[(base + from) >> c.page_shift];
                to_id = table[(base + e0 + sub) >> c.page_shift];
            }
            for (int e1 = 0; e1 < lanes && e0 + e1 < n; e1 += 4) {
                uint4 rk[4], rv[4];
                size_t to[4];
                bool moves[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int e = e0 + e1 + w, at = e1 + w;
                    const int f = __shfl_sync(mask, from, at, lanes);
                    const size_t src = __shfl_sync(mask, from_id, at, lanes) * page_elems +
                                       (size_t)((base + f) & (c.page - 1)) * c.dh;
                    to[w] = off + __shfl_sync(mask, to_id, at, lanes) * page_elems +
                            (size_t)((base + e) & (c.page - 1)) * c.dh;
                    moves[w] = e < n && f != e;
                    if (moves[w]) {
                        rk[w] = *reinterpret_cast<const uint4*>(c.k + off + src);
                        rv[w] = *reinterpret_cast<const uint4*>(c.v + off + src);
                    }
                }
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    if (moves[w]) {
                        *reinterpret_cast<uint4*>(c.k + to[w]) = rk[w];
                        *reinterpret_cast<uint4*>(c.v + to[w]) = rv[w];
                    }
            }
        }
    }
}

// Compaction counts a page's entries in the table first: holders[] is 0 before, and again
// behind cache_recount_kernel.
__global__ void __launch_bounds__(256) cache_holders_kernel(const __grid_constant__ CacheDev c) {
    pdl_wait();
    pdl_trigger();
    const long long entries = (long long)c.max_seqs * c.max_pages, step = gridDim.x * 256LL;
    for (long long e = blockIdx.x * 256LL + threadIdx.x; e < entries; e += step) {
        const int id = c.table[e];
        if (id >= 0 && id < c.n_pages) atomicAdd(&c.holders[id], 1);
    }
}

// One block: pairs the movable pages past the number in use with the free ones below it,
// both ascending; plan->total is that number, fresh[] the new places.  (There are as many
// free ones below as pages in use past it, movable or not.)
__global__ void __launch_bounds__(kStepThreads) cache_compact_kernel(const __grid_constant__ CacheDev c) {
    __shared__ int s_ws[33];
    pdl_wait();
    pdl_trigger();
    int mine = 0, live;
    for (int p = threadIdx.x; p < c.n_pages; p += kStepThreads) mine += c.ref[p] > 0;
    block_scan(mine, s_ws, live);
    const int mine4 = threadIdx.x * 4;
    const int holes = collect_pages(c.ref, nullptr, 0, live, live, four_pages(c.ref, nullptr, mine4, live), s_ws,
                                    [&](int k, int page) { c.copies[k].y = page; });
    const int movers = collect_pages(c.ref, c.holders, live, c.n_pages, holes,
                                     four_pages(c.ref, c.holders, live + mine4, c.n_pages), s_ws,
                                     [&](int k, int page) { c.copies[k].x = page; });
    __syncthreads();
    for (int k = threadIdx.x; k < movers; k += kStepThreads) c.fresh[c.copies[k].x] = c.copies[k].y;
    if (threadIdx.x == 0) *c.plan = CachePlan{live, 0, 0, movers, 0, 0, 0, 0, c.plan->serial + 1};
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
            const int ref = c.ref[id];
            if (movable(ref, c.holders[id])) c.table[e] = c.fresh[id];
            else if (ref <= 0) atomicCAS(c.err, 0, ERR_CACHE_STATE);
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
    for (int p = blockIdx.x * 256 + threadIdx.x; p < c.n_pages; p += gridDim.x * 256) c.holders[p] = 0;
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
    const long long per = 256 / (c.dh / 8), units = (long long)n * c.layers * c.Hkv;
    const dim3 grid((unsigned)std::min<long long>((units + per - 1) / per, c.num_sms * 16));
    cudaError_t e = launch_pdl(cache_accept_kernel<N>, grid, dim3(256), 0, st, c, l, n_acc, path, ld_path, accepted);
    if (e != cudaSuccess) return e;
    e = launch_pdl(cache_cut_kernel<N>, dim3(entry_blocks(c, (long long)n * c.max_pages)), dim3(256), 0, st, c, l,
                   (const int*)accepted);
    if (e != cudaSuccess || !c.codes) return e;
    return launch_cache_bounds_accepted(c, n, seq, n_acc, accepted, st);
}
}  // namespace

cudaError_t launch_cache_accept(const CacheDev& c, int n, const int* seq, const int* n_acc, const int* path,
                                int ld_path, cudaStream_t st) {
    return n <= kShortList ? accept_launch<kShortList>(c, n, seq, n_acc, path, ld_path, st)
                           : accept_launch<kCacheMaxSeqs>(c, n, seq, n_acc, path, ld_path, st);
}

cudaError_t launch_cache_compact(const CacheDev& c, cudaStream_t st) {
    const dim3 entries(entry_blocks(c, (long long)c.max_seqs * c.max_pages));
    cudaError_t e = launch_pdl(cache_holders_kernel, entries, dim3(256), 0, st, c);
    if (e == cudaSuccess) e = launch_pdl(cache_compact_kernel, dim3(1), dim3(kStepThreads), 0, st, c);
    if (e == cudaSuccess) e = launch_pdl(cache_fill_kernel, dim3(c.num_sms * 6), dim3(kCopyThreads), 0, st, c, 0, 0);
    if (e == cudaSuccess) e = launch_pdl(cache_remap_kernel, entries, dim3(256), 0, st, c);
    if (e == cudaSuccess)
        e = launch_pdl(cache_recount_kernel, dim3(entry_blocks(c, c.n_pages)), dim3(256), 0, st, c);
    return e;
}

}  // namespace tmoe
