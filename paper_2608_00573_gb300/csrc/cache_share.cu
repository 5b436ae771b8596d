// The list of attention items of a step whose sequences come in groups with a common
// prompt (trimmoe_cache_share).
//
// A group's common positions are those of the pages that all of its sequences with new tokens
// hold at their front, in whole key tiles.  An item is a group of query rows and a
// key/value head, as in other steps; here there are two kinds: common items, all new
// tokens of a group of sequences over its common tiles, without any mask, and own
// items, the tokens of one sequence over its other tiles.  Every item's sums go to parts,
// which cache_join_shared_kernel adds per token: the common item's in the order of the keys, then
// its own.
//
//   o = sum_i e^(m_i - m) o_i / sum_i e^(m_i - m) l_i,  m = max m_i   over the parts i of a row
//
// Single tokens' own pages, and the common ones of groups of up to 32 rows, are pieces that a second kernel
// reads beside the attention kernel (cache_blocks_attention.cu): a 128-row tile would hold few rows of
// them, and HBM is what they wait for.
//
// Bound: HBM for single tokens, each common K and V row once a group; the chain of a key tile for drafted trees.
// Measured, 32 heads on 8, D = 128: 64 samples of a prompt of 8200 positions with up to 900 of their own 41.5 us (23 at
// the copy rate; the attention kernel's last CTA, the pieces and the join take 30, 31 and 8 alone); 4 samples of
// 700 positions 11.9 us, latency; 24 trees of 16 drafts behind 5000 positions 67 us; 16
// heads on 16, five groups of up to 24 behind 300 to 6000 positions 58 us.
//
// Single tokens are always taken up.  An attend without groups / with them, us, 32 heads on 8, pages of 64, up to 128 positions of
// their own, behind 300, 1000, 3000, 8000 and 30000 common ones:
//   one group of 2    10.9 / 10.1   12.0 / 10.3   17.8 / 12.8   21.8 / 17.8   40.2 / 33.1
//   of 4              11.1 / 11.7   16.2 / 12.4   20.9 / 17.5   27.8 / 20.1   61.3 / 35.1
//   of 16             18.2 / 14.4   24.5 / 16.2   35.2 / 16.3   64.0 / 27.0    195 / 41.6
//   of 64             30.1 / 19.1   50.7 / 20.5    106 / 22.8    244 / 34.5    854 / 55.8
//   16 groups of 2    25.3 / 17.3   36.8 / 22.8   61.5 / 45.5    159 / 89.8    553 / 288
//   64 groups of 1    30.9 / 26.9   56.8 / 55.2    134 / 126     320 / 306    1147 / 1094
// (the last share nothing: pieces of equal size).  16 heads on 16, pages of 16, one group of 4: 12.5 / 10.3, 19.3 / 11.5, 27.6 / 15.9,
// 51.7 / 22.4, 161 / 59.4.  Of 100 such pairs two lose, the group of 4 behind 300 and, on 16 heads, one sequence alone
// behind 30000, 49.9 / 57.0.  The list itself (two launches, once a step for all its layers) takes 9 to 16 us in a row of
// launches, 25 behind 30000 positions for 64 sequences, 56 where their pages are of 16.  Several tokens per sequence:
// trimmoe_cache_share.
#include <algorithm>

#include "cache.cuh"

namespace tmoe {

namespace {

constexpr int kCommonThreads = 256;
constexpr int kPlanThreads = 1024;
constexpr int kMinTiles = 2;           // as for other steps (cache_pages.cu)

// A block takes one group: the front pages that its sequences share, and how many whole key
// tiles these fill.
template <int N>
__global__ void __launch_bounds__(kCommonThreads) cache_common_kernel(const __grid_constant__ CacheDev c,
                                                                      const __grid_constant__ CacheList<N> l) {
    __shared__ int s_pages, s_lead, s_members;
    const int g = blockIdx.x, from = l.a[g], to = from + l.b[g];
    if (threadIdx.x == 0) {
        s_pages = 0x7fffffff;
        s_lead = 0x7fffffff;
        s_members = 0;
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    if (!c.step_plan->ok) return;
    for (int i = from + threadIdx.x; i < to; i += kCommonThreads) {
        const CacheSeq s = c.seqs[i];
        if (s.q_len > 0) {
            atomicMin(&s_pages, (s.kv_len - s.q_len) >> c.page_shift);
            atomicMin(&s_lead, i);
            atomicAdd(&s_members, 1);
        }
    }
    __syncthreads();
    if (s_members < 2) {
        if (threadIdx.x == 0) c.common[g] = 0;
        return;
    }
    // A warp takes one sequence at a time; the first difference ends it for all.
    const int lane = threadIdx.x & 31;
    const int* lead = c.table + (size_t)c.seqs[s_lead].seq * c.max_pages;
    for (int i = s_lead + 1 + (threadIdx.x >> 5); i < to; i += kCommonThreads / 32) {
        const CacheSeq s = c.seqs[i];
        if (s.q_len == 0) continue;
        const int* mine = c.table + (size_t)s.seq * c.max_pages;
        for (int j0 = 0;; j0 += 128) {
            const int end = __shfl_sync(0xffffffffu, *(volatile int*)&s_pages, 0);
            if (j0 >= end) break;
            int a[4], b[4], first = 0x7fffffff;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int j = j0 + u * 32 + lane;
                a[u] = j < end ? lead[j] : 0;
                b[u] = j < end ? mine[j] : 0;
            }
#pragma unroll
            for (int u = 3; u >= 0; --u)
                if (a[u] != b[u] || a[u] < 0) first = j0 + u * 32 + lane;
            first = __reduce_min_sync(0xffffffffu, first);
            if (lane == 0 && first != 0x7fffffff) atomicMin(&s_pages, first);
            __syncwarp();
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) c.common[g] = (s_pages << c.page_shift) / kCacheTile;
}

template <class V>
__device__ __forceinline__ V up(V v, int o) {
    return __shfl_up_sync(0xffffffffu, v, o);
}

// Exclusive prefix sum over the block; every thread gets the total.
template <class V>
__device__ V block_sum(V v, V* ws, V& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    V x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V y = up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) ws[warp] = x;
    __syncthreads();
    if (warp == 0) {
        V s = ws[lane];
        const V own = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const V y = up(s, o);
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

// One block: the items of the step, their shares of the line, where their parts lie and which
// items hold each token.  A thread takes one group of sequences, one sequence, then one
// item's row of heads at a time.
template <int N>
__global__ void __launch_bounds__(kPlanThreads) cache_share_kernel(const __grid_constant__ CacheDev c,
                                                                   const __grid_constant__ CacheList<N> l, int n_seqs, int T,
                                                                   int single) {
    __shared__ int s_common[kCacheMaxSeqs], s_begin[kCacheMaxSeqs + 1], s_own[kCacheMaxSeqs + 1];   // first items of groups, sequences
    __shared__ int s_of[kCacheMaxSeqs];                // a sequence's group
    __shared__ int s_row[kCacheMaxSeqs], s_cuts[kCacheMaxSeqs];        // pieces of small groups: parts' first row, cuts
    __shared__ int s_wi[33];
    __shared__ long long s_wl[33];
    const int i = threadIdx.x, n = l.n, TT = c.tile_tokens;
    pdl_wait();
    pdl_trigger();
    if (!c.step_plan->ok) {
        if (i == 0) {
            CachePlan none{};
            none.serial = c.step_plan->serial;
            *c.plan = none;
        }
        return;
    }
    int tiles = 0, count = 0;
    if (i < n) {
        tiles = c.common[i];
        for (int k = l.a[i]; k < l.a[i] + l.b[i]; ++k) s_of[k] = i;
    }
    int tok = 0;                                       // the group's tokens
    if (i < n) {
        const CacheSeq a = c.seqs[l.a[i]], z = c.seqs[l.a[i] + l.b[i] - 1];
        tok = z.q_off + z.q_len - a.q_off;
    }
    CacheSeq mine = {};
    if (i < n_seqs) mine = c.seqs[i];
    int pieces = 0;
    float piece_bytes = 0.f;
    if (single) {
        // Small groups' common pages are read in pieces, as sequences' own pages are; for
        // larger ones the 128-row tiles of the attention kernel read common pages.  (Short ones too: left to
        // their sequences where that cost less than 40 MB, 40 samples of 300 positions took 21.7 us instead of 17.2,
        // 20 of 300 18.2 instead of 13.7, 12 of 700 18.7 instead of 17.2; 32 heads on 8.)
        const int per = 16 / c.rep, row_tiles = small_tiles(tok, c.rep);
        const bool small = row_tiles <= kSmallTiles;
        if (i < n) s_common[i] = tiles;
        __syncthreads();
        // Stages of 64 positions of one head; a piece has as many as give each of two CTAs an SM three pieces,
        // but few enough not to be a long wait, and a sequence not more than kPieceCuts of them.
        const int common = small ? tiles * (kCacheTile / 64) : 0;
        const int own = mine.q_len ? (mine.kv_len - s_common[s_of[i]] * kCacheTile + 63) / 64 : 0;
        long long all;
        block_sum((long long)common * row_tiles + own, s_wl, all);
        piece_bytes = (float)all * c.Hkv * (64 * 4) * c.dh;
        const int share = (int)(all * c.Hkv / (2 * c.num_sms)) + 1;
        const int most = share < 6 ? max(2, share) : max(4, (share + 2) / 3);
        auto cuts_of = [&](int stages) { return min(kPieceCuts, (stages + most - 1) / most); };
        const int common_cuts = cuts_of(common), own_cuts = cuts_of(own);
        int n_group, n_own;
        const int first_group = block_sum(common_cuts * row_tiles, s_wi, n_group);
        const int first_own = n_group + block_sum(own_cuts, s_wi, n_own);
        pieces = n_group + n_own;
        int row, rows = common_cuts * c.Hkv * tok * c.rep, all_rows;
        row = block_sum(rows + own_cuts * c.Hkv * c.rep, s_wi, all_rows) + (int)cache_piece_rows(c);
        if (i < n) {
            s_row[i] = row;
            s_cuts[i] = common_cuts;
        }
        if (common_cuts) {
            // (Any of the group's sequences with new tokens; their table rows agree.)
            int lead = l.a[i];
            while (c.seqs[lead].q_len == 0) ++lead;
            const CacheSeq s = c.seqs[lead];
            for (int x = 0; x < common_cuts * row_tiles; ++x) {
                const int cut = x % common_cuts, tile = x / common_cuts;
                c.pieces[first_group + x] = CachePiece{s.seq, s.q_off + tile * per, min(per, tok - tile * per) * c.rep, 1,
                                                       common * cut / common_cuts, common * (cut + 1) / common_cuts, 0, tiles * kCacheTile,
                                                       row + (cut * tok + tile * per) * c.rep, common_cuts * tok * c.rep, {0, 0}};
            }
        }
        __syncthreads();
        if (own_cuts) {
            const int g = s_of[i], from = s_common[g] * kCacheTile >> c.page_shift;
            const int first = row + rows;
            const bool direct = own_cuts == 1 && !s_common[g];
            for (int x = 0; x < own_cuts; ++x)
                c.pieces[first_own + x] = CachePiece{mine.seq, mine.q_off, c.rep, 0, (int)((long long)own * x / own_cuts),
                                                     (int)((long long)own * (x + 1) / own_cuts), from, mine.kv_len,
                                                     direct ? -1 : first + x * c.rep, own_cuts * c.rep, {0, 0}};
            TokenParts p = {};
            p.own_row = first;
            p.own_n = own_cuts;
            p.own_item = p.common_item = -1;
            if (s_cuts[g]) {
                p.common_row = s_row[g] + (mine.q_off - c.seqs[l.a[g]].q_off) * c.rep;
                p.common_n = s_cuts[g];
                p.common_step = (c.seqs[l.a[g] + l.b[g] - 1].q_off + c.seqs[l.a[g] + l.b[g] - 1].q_len - c.seqs[l.a[g]].q_off) * c.rep;
            }
            c.parts_of[mine.q_off] = p;
        }
        __syncthreads();
        if (small) tiles = 0;                          // (from here on: what is on the line)
    }
    if (i < n) s_common[i] = tiles;
    __syncthreads();
    if (tiles) count = (tok + 2 * TT - 1) / (2 * TT);
    int n_common, n_own;
    const int at = block_sum(count, s_wi, n_common);
    const int own = block_sum(single ? 0 : (mine.q_len + 2 * TT - 1) / (2 * TT), s_wi, n_own);
    if (i < n) {
        s_begin[i] = at;
    }
    if (i < n_seqs) s_own[i] = n_common + own;
    if (i == 0) {
        s_begin[n] = n_common;
        s_own[n_seqs] = n_common + n_own;
    }
    __syncthreads();
    const int items = n_common + n_own;
    // Largest k with off[k] <= x: the one whose range is not empty.
    auto find = [](const int* off, int m, int x) {
        int lo = 0, hi = m;
        while (hi - lo > 1) {
            const int k = (lo + hi) >> 1;
            if (off[k] <= x) lo = k;
            else hi = k;
        }
        return lo;
    };
    long long W = 0;
    int two = 0;
    for (int e0 = 0; e0 < items; e0 += kPlanThreads) {
        const int e = e0 + i;
        CacheGroup g = {};
        if (e < n_common) {
            const int k = find(s_begin, n, e);
            const CacheSeq a = c.seqs[l.a[k]], z = c.seqs[l.a[k] + l.b[k] - 1];
            const int tok = (e - s_begin[k]) * 2 * TT, all = z.q_off + z.q_len - a.q_off;
            // (Any of the group's sequences with new tokens; their table rows agree.)
            int lead = l.a[k];
            while (c.seqs[lead].q_len == 0) ++lead;
            g.seq = c.seqs[lead].seq;
            g.kv_len = g.base = g.first = s_common[k] * kCacheTile;
            g.row = a.q_off + tok;
            g.ntok = min(2 * TT, all - tok);
            g.t0 = 0;
            g.common = 1;
            g.cost = s_common[k] * share_tile(cache_two_tiles(g.ntok, TT)) + kShareEnds;
        } else if (e < items) {
            const int k = find(s_own, n_seqs, e);
            const CacheSeq s = c.seqs[k];
            const int tok = (e - s_own[k]) * 2 * TT;
            g.seq = s.seq;
            g.kv_len = s.kv_len;
            g.base = s.kv_len - s.q_len;
            g.first = g.base + tok;
            g.row = s.q_off + tok;
            g.ntok = min(2 * TT, s.q_len - tok);
            g.t0 = s_common[s_of[k]];
            g.cost = (cache_group_tiles(s.q_len, s.kv_len, g.first, g.ntok) - g.t0) * share_tile(cache_two_tiles(g.ntok, TT)) + kShareEnds;
        }
        long long sum;
        g.pre = W + block_sum((long long)g.cost, s_wl, sum);
        W += sum;
        two |= e < items && cache_two_tiles(g.ntok, TT);
        if (e < items) c.groups[e] = g;
    }
    two = __syncthreads_or(two);
    W *= c.Hkv;
    int n_ctas = !W ? 0 : (int)max(1LL, min((long long)c.num_sms, W / (kMinTiles * share_tile(two ? 1 : 0))));
    if (single && n_ctas) {
        // The second kernel's CTAs read pieces beside this one's: as many SMs as let both end together, in us (a CTA
        // begins and ends in 6, and its tiles take 1.6 times as long beside the other kernel's
        // traffic; pieces at HBM's rate).  Measured, as here and with other constants: 64 samples of 8200 positions with up
        // to 900 of their own, 32 heads on 8: 41.3 us; 1.2 or 2.0 times 41.8, 43.4; at 5.5 or 7.5 TB/s 42.1, 43.5.  32 of 12000, up
        // to 150: 33.0; 30.2, 33.9; 30.2, 33.9; ends of 4 or 8 us 27.3, 34.7.  64 of 8000, up to 100, 16 heads on 16: 37.8;
        // 40.6, 43.6; 37.8, 37.8; 37.8, 43.6; + 2 or 6 instead of + 4 43.8, 37.8.  12 of 700, 32 on 8: 15.8; at least 8 or 16 us
        // instead of 12 14.3, 17.7; 16 of 3000 16.8; 18.1, 18.9.
        const float a = W * (1.6f * kShareUnit), b = piece_bytes / 6.5e6f * c.num_sms;
        const float t = max(12.f, (a + b) / c.num_sms + 4.f);
        n_ctas = min(n_ctas, (int)(a / (t - 6.f)) + 1);
        // A whole number of CTAs to an item, where there are as many, the nearest one: a CTA that begins a second item
        // ends 6 us later.  (Nearest, the next below, as it comes: 64 of 8000, up to 1000 of their own, 16 heads on 16, 71.5 us,
        // 118, 75.4; 40 of 20000 52.8, 52.8, 55.8; 64 of 8200, 32 on 8, 41.2, 42.0, 41.0; 12 of 700 15.8, 17.2, 16.1; but 4 times 16 of
        // 1000 25.2, 22.7, 24.5, and 16 of 8000 27.0 instead of the next below's 24.3.)
        const int all = items * c.Hkv;
        if (n_ctas > all) n_ctas = min(c.num_sms, (n_ctas + all / 2) / all * all);
    }
    // Where parts lie: an item's pieces are as many as heads and cuts.
    long long rows = 0;
    for (int e0 = 0; e0 < items; e0 += kPlanThreads) {
        const int e = e0 + i;
        int mine = 0, r = 0, first = 0;
        CacheGroup g = {};
        if (e < items) {
            g = c.groups[e];
            r = cache_part_rows(g.ntok, TT, c.rep);
            first = cache_cta_of(g.pre * c.Hkv, W, n_ctas);
            const int last = cache_cta_of((g.pre + g.cost) * c.Hkv - 1, W, n_ctas);
            mine = ((c.Hkv + last - first) * r + 31) & ~31;
        }
        long long sum;
        const long long before = rows + block_sum((long long)mine, s_wl, sum);
        rows += sum;
        if (e < items) c.groups[e].part_row = (int)(before - (long long)first * r);
    }
    __syncthreads();
    for (int k = i; k < items * c.Hkv; k += kPlanThreads) {
        const int e = k / c.Hkv;
        const int cost = c.groups[e].cost, two_tiles = cache_two_tiles(c.groups[e].ntok, TT), step = share_tile(two_tiles);
        const long long start = c.groups[e].pre * c.Hkv + (long long)(k - e * c.Hkv) * cost;
        const int first = cache_cta_of(start, W, n_ctas);
        const int tiles = share_tiles(cost, two_tiles);
        c.cut[k] = make_int2(first, cache_cta_of(start + (long long)(tiles - 1) * step, W, n_ctas) - first + 1);
    }
    if (i == 0) *c.plan = CachePlan{W, items, n_ctas, 0, 1, 0, 0, pieces, c.step_plan->serial, T, single};
    for (int t = i; t < T; t += kPlanThreads) {
        const int k = c.owner[t], g = s_of[k], from = c.seqs[l.a[g]].q_off;
        const int item = s_common[g] ? s_begin[g] + (t - from) / (2 * TT) : -1;
        if (single) c.parts_of[t].common_item = item;
        else c.parts_of[t] = TokenParts{0, 0, s_own[k] + (t - c.seqs[k].q_off) / (2 * TT), 0, 0, 0, item, 0};
    }
    __syncthreads();
    for (int k = i; k < T * c.Hkv; k += kPlanThreads) {
        const int t = k / c.Hkv, head = k - t * c.Hkv;
        const TokenParts of = c.parts_of[t];
        c.lists[2 * (size_t)k] = common_parts(c, of, head, t);
        c.lists[2 * (size_t)k + 1] = own_parts(c, of, head, t);
    }
    for (int b = i; b < n_ctas; b += kPlanThreads) {
        CacheShare sh;
        sh.begin = W * b / n_ctas;
        sh.end = W * (b + 1) / n_ctas;
        const long long x = sh.begin / c.Hkv;
        int lo = 0, hi = items;
        while (hi - lo > 1) {
            const int m = (lo + hi) >> 1;
            if (c.groups[m].pre <= x) lo = m;
            else hi = m;
        }
        sh.group = lo;
        sh.g = c.groups[lo];
        sh.within = sh.begin - sh.g.pre * c.Hkv;
        sh.head = (int)(sh.within / sh.g.cost);
        sh.within -= (long long)sh.head * sh.g.cost;
        sh.first = sh.last = b;                        // (not used here)
        c.shares[b] = sh;
    }
}

// Adds the parts of a step with groups of sequences.  A block takes a token and some key/value heads
// (about as many columns as threads, by four), whose lists of parts it looks up first; a thread then takes four columns of a query
// head at a time, the common item's parts first, in the order of the keys.  Neighbouring
// threads take the heads that share a key/value head: their rows of a part lie side by side (with
// neighbouring columns instead the join of 12 trees took 27 us).  Bound: L2.
constexpr int kJoinHeads = 16;
inline __host__ __device__ int join_heads(const CacheDev& c) {
    const int n = 1024 / (c.rep * c.dh);
    return n < 1 ? 1 : n < kJoinHeads ? n : kJoinHeads;
}
// B: parts that a thread reads at a time.  With few blocks of threads their latency is what counts (64 samples, 12 at a
// time 42 us, 6 at a time 44); with many, how many threads an SM holds (12 trees 3 at a time with 6 blocks an SM 92.5 us, 4 with
// 5 93.5, 6 with 4 95, 2 with 8 94, 12 with 2 102; 6 prompts of 200 to 400 tokens behind a common 6000 212 / 216 / 228 / 216 / 259).
template <int DH, int B>
__global__ void __launch_bounds__(256, B > 3 ? 2 : 6) cache_join_shared_kernel(const __grid_constant__ CacheDev c,
                                                                   const __grid_constant__ AttendParams p) {
    __shared__ PartList s_parts[kJoinHeads * 2];
    const int most = join_heads(c), blocks = (c.Hkv + most - 1) / most;
    const int t = blockIdx.x / blocks, head0 = blockIdx.x % blocks * most, heads = min(most, c.Hkv - head0);
    pdl_wait();
    pdl_trigger();
    const CachePlan pl = *c.plan;
    if (threadIdx.x < 2 * heads) s_parts[threadIdx.x] = c.lists[((size_t)t * c.Hkv + head0) * 2 + threadIdx.x];
    __syncthreads();
    if (!pl.ok || share_stale(c, pl, p.T, p.single, p.alone)) return;     // (a refused step has written no lists)
    // A token whose only part is one piece has its result already.
    if (pl.pieces && s_parts[0].count == 0 && s_parts[1].count == 1) return;
    for (int e = threadIdx.x; e < heads * c.rep * (DH / 4); e += 256) {
        const int x = e / c.rep, k = x / (DH / 4), col = x % (DH / 4) * 4, row = e - x * c.rep;
        float top = -INFINITY, l = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
        add_parts<DH, B>(c, s_parts[2 * k], s_parts[2 * k + 1], row, col, top, l, a);
        const float il = l == 0.f ? 0.f : 1.f / l;
        *reinterpret_cast<uint2*>(p.out + (size_t)t * p.ld_out + (size_t)((head0 + k) * c.rep + row) * DH + col) =
            make_uint2(pack_bf16x2(a[0] * il, a[1] * il), pack_bf16x2(a[2] * il, a[3] * il));
    }
}

template <int N>
cudaError_t share_launch(const CacheDev& c, int n, const int* counts, int n_seqs, int T, int single, cudaStream_t st) {
    CacheList<N> l;
    l.n = n;
    int at = 0;
    for (int i = 0; i < n; ++i) {
        l.a[i] = at;
        l.b[i] = counts[i];
        at += counts[i];
    }
    const cudaError_t e = launch_pdl(cache_common_kernel<N>, dim3((unsigned)n), dim3(kCommonThreads), 0, st, c, l);
    if (e != cudaSuccess) return e;
    return launch_pdl(cache_share_kernel<N>, dim3(1), dim3(kPlanThreads), 0, st, c, l, n_seqs, T, single);
}

}  // namespace

cudaError_t launch_cache_share(const CacheDev& c, int n, const int* counts, int n_seqs, int T, int single, cudaStream_t st) {
    return n <= 64 ? share_launch<64>(c, n, counts, n_seqs, T, single, st)
                   : share_launch<kCacheMaxSeqs>(c, n, counts, n_seqs, T, single, st);
}

cudaError_t launch_cache_join(const CacheDev& c, const AttendParams& p, cudaStream_t st) {
    const dim3 grid((unsigned)(p.T * ((c.Hkv + join_heads(c) - 1) / join_heads(c))));
    const bool few = grid.x <= 2u * c.num_sms;
    if (c.dh == 64)
        return few ? launch_pdl(cache_join_shared_kernel<64, 12>, grid, dim3(256), 0, st, c, p)
                   : launch_pdl(cache_join_shared_kernel<64, 3>, grid, dim3(256), 0, st, c, p);
    return few ? launch_pdl(cache_join_shared_kernel<128, 12>, grid, dim3(256), 0, st, c, p)
               : launch_pdl(cache_join_shared_kernel<128, 3>, grid, dim3(256), 0, st, c, p);
}

}  // namespace tmoe
