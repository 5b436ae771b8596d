// Attention of each new token over pages that it is told to read (a list per key/value
// head) and over the positions from its step's first page on; and, for single tokens of
// sequences with a common prompt (cache_share.cu), over each sequence's own pages.
//
// An item is a token, a key/value head and up to 16 of the query heads that share it.
// No two items have a list in common, so that a tile of the tensor cores has the item's 1
// to 16 rows alone and the operator is bound by what the lists bring in: HBM for single tokens
// (each listed K and V row once), L2 for chunks whose tokens list the same pages.  The
// products are therefore mma.sync with 16 rows, fed from shared memory; a 128-row tile of
// TMEM would hold the same rows.  Measured: 48 single tokens, 16 heads on 16, 96 pages of 16 each, 102 us,
// 5.95 TB/s, 0.87 of the copy rate; one token, 32 heads on 8, 32 pages of 64, 8.4 us, latencies; 800
// tokens' chunks, 24 pages of 64, 430 us, 5.6 GB out of L2 at 13 TB/s.  Prompts whose lists name much of what
// their sequences hold are therefore left to the attention kernel, with the lists as masks (lists_dense:
// those chunks take 168 us), and this kernel computes what that one marks.
//
// A stage is 64 listed positions: pages, or halves of pages of 128, as boxes of the cache's
// tensor maps, with their values.  One warp draws items, finds their pages and keeps the
// copies going, into the next item while this one is computed.  Four warps take 16 positions of every
// stage each, with sums of their own:
//
//   S = Q K^T (16 x 16);  m' = max(m, max s);  p = 2^(scale' s - m');  l += sum p;  O = O 2^(m - m') + P V
//
// (m moves only when a score is more than 2^8 above it; P is rounded to bf16, the
// type of the product's operand, l sums p before that rounding; the first key's p is 1.)
// At an item's end the warps' sums are added in shared memory.  (With columns instead of
// positions shared out for P V, and maxima and P handed on at every stage, no sums would have to be
// added, but two barriers a stage cost more: 800 tokens' chunks 593 us against 446.)  When there are
// few items, an item's stages are cut among the CTAs of a cluster, whose sums meet in
// distributed shared memory.  Sums are always added in the same order.
//
// Masked positions (of the last pages: later tokens, other branches of a tree, places
// that no position uses yet) never reach a result: scores are replaced and value
// operands zeroed, not multiplied by 0.
#include <algorithm>

#include "cache.cuh"

namespace tmoe {

namespace {

constexpr int kReaders = 4;                            // warps that multiply; one more loads
constexpr int kThreads = (kReaders + 1) * 32;
constexpr int kStageKeys = 64;
constexpr int kHidden = -1, kWhole = -2;               // what a stage's pages are, else their first position

// What the loading warp says of an item.
struct Item {
    int valid;
    int t, head, row0, rows;   // token, key/value head, query heads of it
    int base, kv_len, pos;
    int g0, g1;                // stages
    int part;                  // OWN: row of its part, -1: it is the result
};

template <int DH>
struct Stage {
    static constexpr int KB = DH / 64;
    static constexpr int SLAB = kStageKeys * 128;      // 64 rows of 64 columns
    static constexpr int TILE = KB * SLAB;             // K or V
    static constexpr int BYTES = 2 * TILE;
    static constexpr int COUNT = 96 * 1024 / BYTES;    // two CTAs to an SM
};

template <int DH>
struct __align__(128) Shared {
    uint8_t stage[Stage<DH>::COUNT][Stage<DH>::BYTES]; // (first: swizzled tiles start at multiples of 1024)
    __nv_bfloat16 q[16][DH];   // the item's queries
    float2 swap[2][DH / 8][32];   // sums of eight rows that one warp gives another, as the lanes hold them
    float2 ml[kReaders][16];   // the warps' maxima and sums of p
    float2 mine[16];           // the CTA's (clusters)
    uint64_t full[8], empty[8], q_full, q_empty;
    int first[8][4];           // of the stage's pages: first position, kHidden or kWhole
    Item item;
    CachePlan plan;
    int first_item;
    int abort_flag, never;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

// Barriers of the four multiplying warps.
__device__ __forceinline__ void readers_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool readers_any(bool x) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r)
                 : "r"((uint32_t)x)
                 : "memory");
    return r != 0;
}

// Entries of a list, 32 at a time, a lane each, in turn: which of them count.  In order is a column of a whole page before
// the step (below `own`) that is larger than the entry before it.  What is not, or stands behind a -1, is left out and
// flagged.  A list that goes on in order behind such an entry may name a page again, which counts once: masks see to that
// by themselves, a list that is followed is searched up to there, and so is cut to kRepeats entries from then on (4096 entries
// by one CTA, the 101st out of order, take 4.0 ms; in order 0.6).
constexpr int kRepeats = 4096;
constexpr int kLeftOut = 0, kCounts = 1, kMayRepeat = 2;
__device__ __forceinline__ bool in_order(int j, int col, int before, int own) {
    return col >= 0 && col < own && (j == 0 || (before >= 0 && col > before));
}
struct ListReader {
    bool ended = false, broken = false;                // by an entry before these: a -1, one that is out of order
    // there: the lane has an entry, its j-th.
    __device__ __forceinline__ int read(const CacheDev& c, bool there, int j, int col, int before, int own) {
        const bool end = there && col == -1, bad = there && !end && !in_order(j, col, before, own);
        const uint32_t e = __ballot_sync(0xffffffffu, end), w = __ballot_sync(0xffffffffu, bad);
        const uint32_t below = (1u << (threadIdx.x & 31)) - 1u;
        const bool late = ended || (e & below), again = broken || (w & below);
        if (there && !end && (bad || late)) atomicCAS(c.err, 0, ERR_CACHE_BLOCKS);
        ended |= e != 0;
        broken |= w != 0;
        if (!there || end || bad || late || (again && j >= kRepeats)) return kLeftOut;
        return again ? kMayRepeat : kCounts;
    }
};
// A page that counts is one of the list's j entries before it.
__device__ __noinline__ bool named_before(const int* list, int j, int col) {
    int before = -1;
    bool found = false;
#pragma unroll 8
    for (int k = 0; k < j; ++k) {
        const int x = list[k];
        found |= x == col && (k == 0 || (before >= 0 && before < x));
        before = x;
    }
    return found;
}

// OWN: no lists; an item is a piece (cache_share.cu) of a key/value head, whose sums are a part, or the result when it
// is its token's only one.  This kernel runs beside the attention kernel before it, which lets it start
// when all that comes before has ended, and waits for that kernel only at its own end (alone: all groups are
// small, and there is no such kernel).
template <int DH, bool OWN>
__global__ void __launch_bounds__(kThreads)
cache_blocks_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ CacheDev c, const __grid_constant__ BlocksParams p) {
    using S = Stage<DH>;
    constexpr int ST = S::COUNT;
    extern __shared__ __align__(1024) uint8_t smem[];
    Shared<DH>& sh = *reinterpret_cast<Shared<DH>*>(smem);
    const uint32_t sb = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int splits = p.splits, rank = blockIdx.x % splits;
    if (threadIdx.x == 0) {
        for (int s = 0; s < ST; ++s) {
            mbar_init(smem_u32(&sh.full[s]), 1);
            mbar_init(smem_u32(&sh.empty[s]), kReaders);
        }
        mbar_init(smem_u32(&sh.q_full), 1);
        mbar_init(smem_u32(&sh.q_empty), kReaders);
        sh.abort_flag = sh.never = 0;
        sh.item.rows = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
        if (!OWN || p.alone) pdl_wait();
        // (All have to agree on the plan, whose counters change, and on the first item, so they are read once.)
        sh.first_item = OWN ? atomicAdd(&c.plan->drawn, 1) : 0;
        sh.plan = from_l2(c.plan);
    }
    __syncthreads();
    if (!OWN || p.alone) pdl_wait();
    pdl_trigger();
    const CachePlan pl = sh.plan;
    // Lists that have been masks of an attention over all pages: the items that it marked.
    const bool again = !OWN && lists_dense(c, p.lists, pl);
    const int items = OWN ? pl.pieces * c.Hkv : again ? pl.pieces * p.row_tiles : p.T * c.Hkv * p.row_tiles;
    // The last CTA to finish drawing leaves the counter at zero for the next call.
    auto drawn_all = [&] {
        __threadfence();
        if (atomicAdd(&c.plan->done, 1) == (int)gridDim.x - 1) {
            c.plan->drawn = 0;
            c.plan->done = 0;
        }
    };
    if (!pl.ok || (OWN && share_stale(c, pl, p.T, 1, p.alone))) {       // (all CTAs)
        if (OWN) {                                     // (the list may be the next call's: what was drawn goes back)
            if (threadIdx.x == 0) drawn_all();
            pdl_wait();
        }
        return;
    }
    if (OWN && sh.first_item >= items) {               // (a CTA that began late)
        if (threadIdx.x == 0) drawn_all();
        pdl_wait();
        return;
    }
    if (sb & 1023u) {
        if (threadIdx.x == 0) atomicCAS(c.err, 0, ERR_TIMEOUT_CACHE_ATTN);
        return;
    }
    const uint32_t abort_at = smem_u32(&sh.abort_flag);
    auto wait = [&](uint64_t* b, uint32_t parity) {
        return __any_sync(0xffffffffu, wait_probes(smem_u32(b), parity & 1u, abort_at, c.err)) != 0;
    };
    const int box_shift = max(0, c.page_shift - 6), page_boxes = 1 << box_shift;   // boxes of a page's rows (pages of 128: two)
    const int per_stage = max(1, kStageKeys >> c.page_shift), box_rows = kStageKeys / per_stage;
    // Four columns of a row: its sums (ml: maximum and sum of p) as a part, or the result.
    auto put = [&](const Item& it, __nv_bfloat16* out, int row, int col, float2 ml, float4 x) {
        if (OWN && it.part >= 0) {
            const long long at = it.part + row;
            *reinterpret_cast<float4*>(c.part_o + at * DH + col) = x;
            if (col == 0) c.part_ml[at] = ml;
        } else {
            const float il = ml.y == 0.f ? 0.f : 1.f / ml.y;
            *reinterpret_cast<uint2*>(out + (size_t)row * DH + col) = make_uint2(pack_bf16x2(x.x * il, x.y * il), pack_bf16x2(x.z * il, x.w * il));
        }
    };

    if (warp == kReaders) {
        // ------------------------------------------------------------ items and loads
        uint32_t issued = 0, n_items = 0;
        const long long piece_end = cache_share_part_rows(c) - 16;
        bool ok = true;
        // OWN: all items are drawn (CTAs on the attention kernel's SMs begin when it has ended), else each CTA has
        // its first one.
        int index = blockIdx.x / splits;
        const int given = OWN ? 0 : (int)gridDim.x;
        if (OWN) index = sh.first_item;
        while (ok && index < items) {
            // The next item (single CTAs; clusters have one each).
            int drawn = items;
            if (splits == 1 && lane == 0) drawn = given + atomicAdd(&c.plan->drawn, 1);
            Item it;
            it.valid = 1;
            int listed = 0, first_own = 0;             // entries of the list that count, first page of the step's own (OWN: of the piece)
            int seq;
            bool all_seen = false;
            if (OWN) {
                const CachePiece pc = from_l2(c.pieces + index / c.Hkv);
                it.head = index % c.Hkv;
                it.t = pc.tok;
                it.row0 = 0;
                it.rows = pc.rows;
                it.kv_len = pc.kv_len;
                it.base = it.pos = pc.kv_len - 1;
                it.g0 = pc.g0;
                it.g1 = pc.g1;
                it.part = pc.part_row < 0 ? -1 : pc.part_row + it.head * pc.head_step;
                first_own = pc.first_page;
                seq = pc.seq;
                all_seen = pc.whole;
                // (Whatever it is, it names nothing that is not there.)
                if (it.rows < 1 || it.rows > 16 || it.t < 0 || it.t + (it.rows - 1) / c.rep >= p.T || it.g0 < 0 ||
                    it.g1 > (c.max_pages << c.page_shift) / kStageKeys + 1 || seq < 0 || seq >= c.max_seqs || first_own < 0 ||
                    pc.part_row < -1 || it.part >= piece_end) {
                    if (lane == 0) atomicCAS(c.err, 0, ERR_CACHE_STATE);
                    index = __shfl_sync(0xffffffffu, drawn, 0);
                    continue;
                }
            } else {
                const int tile = index % p.row_tiles, which = index / p.row_tiles, x = again ? (int)__ldcg(p.lists.marked(which)) : which;
                it.t = x / c.Hkv;
                it.head = x - it.t * c.Hkv;
                it.row0 = tile * 16;
                it.rows = min(16, c.rep - it.row0);
                const CacheToken tok = c.tokens[it.t];
                it.base = tok.base;
                it.kv_len = tok.kv_len;
                it.pos = tok.pos;
                it.part = -1;
                seq = tok.seq;
                first_own = it.base >> c.page_shift;
                listed = min(p.n, first_own);
                const int last = p.tree ? it.kv_len - 1 : it.pos;
                const int boxes = (listed + (last >> c.page_shift) - first_own + 1) * page_boxes;
                const int stages = (boxes + per_stage - 1) / per_stage;
                it.g0 = (int)((long long)stages * rank / splits);
                it.g1 = (int)((long long)stages * (rank + 1) / splits);
            }
            // Lane i looks up box i of 32, the next 32 while these are copied.
            ListReader reader;
            const int* list = p.blocks + ((size_t)it.t * c.Hkv + it.head) * p.n;
            const int* row = c.table + (size_t)seq * c.max_pages;
            const int boxes_end = it.g1 * per_stage;
            struct Box {
                int id, first;                         // page, first position (kWhole, kHidden)
            };
            auto entry_of = [&](int b) {
                const int j = b >> box_shift;
                const bool there = !OWN && b < boxes_end && j < listed;
                return make_int2(there ? list[j] : -1, there && j ? list[j - 1] : -1);
            };
            auto look_up = [&](int b, int2 entry) {
                Box x{0, kHidden};
                const int j = b >> box_shift, sub = b & (page_boxes - 1);
                const bool mine = b < boxes_end, in_list = !OWN && j < listed;
                int col = first_own + j - listed;
                bool fits = mine && !in_list && col < c.max_pages && (col << c.page_shift) < it.kv_len;
                if (!OWN && (b - lane) >> box_shift < listed) {            // (some lanes' boxes are listed)
                    const int says = reader.read(c, mine && in_list, j, entry.x, entry.y, first_own);
                    if (says != kLeftOut) {
                        col = entry.x;
                        fits = says == kCounts || !named_before(list, j, col);
                    }
                }
                if (!fits) return x;
                x.id = OWN ? __ldcg(row + col) : row[col];
                if (x.id < 0 || x.id >= c.n_pages) {
                    atomicCAS(c.err, 0, ERR_CACHE_STATE);
                    return x;
                }
                x.first = j < listed || all_seen ? kWhole : (col << c.page_shift) + sub * box_rows;
                return x;
            };
            int b0 = it.g0 * per_stage;
            const int2 entry0 = entry_of(b0 + lane), entry1 = entry_of(b0 + 32 + lane);
            if (!OWN && b0 > 0) {                      // (what the entries before this CTA's say)
                bool e = false, w = false;
                for (int k = lane; k < min(listed, b0 >> box_shift); k += 32) {
                    const int col = list[k], before = k ? list[k - 1] : -1;
                    e |= col == -1;
                    w |= col != -1 && !in_order(k, col, before, first_own);
                }
                reader.ended = __any_sync(0xffffffffu, e) != 0;
                reader.broken = __any_sync(0xffffffffu, w) != 0;
            }
            Box now = look_up(b0 + lane, entry0), next = look_up(b0 + 32 + lane, entry1);
            // The readers have taken what was said of the item before, and its queries.
            if (n_items) ok = !wait(&sh.q_empty, n_items - 1);
            if (!ok) break;
            // (A piece of common pages has several tokens' queries.)
            const int q_rows = OWN ? c.rep : it.rows;
            if (lane == 0) {
                sh.item = it;
                mbar_arrive_expect_tx(smem_u32(&sh.q_full), (uint32_t)it.rows * DH * 2);
            }
            __syncwarp();
            if (lane * q_rows < it.rows)
                bulk_load(smem_u32(sh.q[lane * q_rows]), p.q + (size_t)(it.t + lane) * p.ld_q + (size_t)(it.head * c.rep + it.row0) * DH,
                          (uint32_t)q_rows * DH * 2, smem_u32(&sh.q_full));
            __syncwarp();
            ++n_items;
            for (int g = it.g0; g < it.g1; ++g) {
                const int at = g * per_stage - b0;     // (per_stage divides 32)
                const int s = (int)(issued % ST);
                if (issued >= (uint32_t)ST) ok = !wait(&sh.empty[s], issued / ST - 1);
                if (!ok) break;
                const int i = lane / (2 * S::KB), kb = lane % S::KB, is_v = lane / S::KB & 1;
                const int id = __shfl_sync(0xffffffffu, now.id, (at + i) & 31), first = __shfl_sync(0xffffffffu, now.first, (at + i) & 31);
                const bool mine = i < per_stage, there = mine && first != kHidden;
                const uint32_t n = __popc(__ballot_sync(0xffffffffu, there));
                if (mine && kb == 0 && !is_v) sh.first[s][i] = first;
                __syncwarp();
                const uint32_t fb = smem_u32(&sh.full[s]);
                if (lane == 0) mbar_arrive_expect_tx(fb, n * box_rows * 128);
                __syncwarp();
                if (there) {
                    const int sub = (g * per_stage + i) & (page_boxes - 1);
                    tma_load_2d(sb + s * S::BYTES + is_v * S::TILE + kb * S::SLAB + i * box_rows * 128, is_v ? &tm_v : &tm_k, kb * 64,
                                (int)((((size_t)id * c.Hkv + it.head) << c.page_shift) + sub * box_rows), fb);
                }
                __syncwarp();
                ++issued;
                if (at + per_stage == 32) {
                    b0 += 32;
                    now = next;
                    next = look_up(b0 + 32 + lane, entry_of(b0 + 32 + lane));
                }
            }
            if (!OWN && rank == 0) {                   // nothing is behind the columns that a list can have
                bool more = false;
                for (long long k = listed + lane; k < p.n; k += 32) more |= list[k] != -1;
                if (more) atomicCAS(c.err, 0, ERR_CACHE_BLOCKS);
            }
            index = __shfl_sync(0xffffffffu, drawn, 0);
        }
        if (splits == 1 && lane == 0) drawn_all();
        if (ok && n_items) ok = !wait(&sh.q_empty, n_items - 1);
        if (ok && lane == 0) {
            sh.item.valid = 0;
            mbar_arrive(smem_u32(&sh.q_full));
        }
        // The copies have landed before the CTA ends, also one that gave up.
        const uint32_t never = smem_u32(&sh.never), tail = min(issued, (uint32_t)ST);
        for (uint32_t k = issued - tail; k < issued; ++k) wait_probes(smem_u32(&sh.full[k % ST]), (k / ST) & 1, never, c.err);
        if (n_items && !ok) wait_probes(smem_u32(&sh.q_full), (n_items - 1) & 1, never, c.err);
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ products
        const int r = lane >> 2, q2 = (lane & 3) * 2;
        const int k16 = warp * 16, box = k16 / box_rows;
        // ldmatrix rows: keys of K by halves of 8 columns, keys of V by halves of 8 keys.
        const int krow = k16 + (lane >> 4) * 8 + (lane & 7), kcol = (lane >> 3) & 1;
        const int vrow = k16 + ((lane >> 3) & 1) * 8 + (lane & 7), vcol = lane >> 4;
        uint32_t at = 0;
        bool lost = false;                             // lost: a wait ran out; all go on to the next barrier
        for (uint32_t n = 0;; ++n) {
            lost |= wait(&sh.q_full, n);
            if (readers_any(lost) || !sh.item.valid) break;
            const Item it = sh.item;
            uint32_t qa[DH / 16][4];
            {
                auto word = [&](int row, int col) {
                    return row < it.rows ? *reinterpret_cast<const uint32_t*>(&sh.q[row][col + q2]) : 0u;
                };
#pragma unroll
                for (int k = 0; k < DH / 16; ++k) {
                    qa[k][0] = word(r, k * 16);
                    qa[k][1] = word(r + 8, k * 16);
                    qa[k][2] = word(r, k * 16 + 8);
                    qa[k][3] = word(r + 8, k * 16 + 8);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.q_empty));
            const uint64_t tree = p.tree ? __ldcg(p.tree + it.t) : 0;
            const bool two = it.rows > 8;              // the tile's lower half has rows
            float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};   // rows lane / 4 and lane / 4 + 8
            float o[DH / 8][4];
#pragma unroll
            for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
            for (int g = it.g0; g < it.g1 && !lost; ++g, ++at) {
                const int s = (int)(at % ST);
                lost |= wait(&sh.full[s], at / ST);
                const int first = sh.first[s][box];
                uint32_t see = 0;                      // keys of the 16 that the token sees
                if (first == kWhole) {
                    see = 0xffffu;
                } else if (first != kHidden) {
                    const int key = first + (k16 & (box_rows - 1));
                    const int all = p.tree ? it.base : it.pos + 1, k = all - key;
                    see = k >= 16 ? 0xffffu : k > 0 ? (1u << k) - 1u : 0u;
                    if (p.tree) {
                        const int d = key - it.base, end = it.kv_len - key;
                        if (d >= 0) {
                            if (d < 64) see |= (uint32_t)(tree >> d) & 0xffffu;
                        } else if (d > -16) {
                            see |= (uint32_t)(tree << -d) & 0xffffu;
                        }
                        see &= end >= 16 ? 0xffffu : end > 0 ? (1u << end) - 1u : 0u;
                    }
                }
                if (see) {
                    const uint32_t kt = sb + s * S::BYTES, vt = kt + S::TILE;
                    float sc[2][4] = {};
#pragma unroll
                    for (int k = 0; k < DH / 16; ++k) {
                        uint32_t b[4];
                        ldmatrix_x4(b, kt + (k >> 2) * S::SLAB + krow * 128 + ((((k & 3) * 2 + kcol) ^ (krow & 7)) << 4));
                        const uint32_t b0[2] = {b[0], b[1]}, b1[2] = {b[2], b[3]};
                        mma_bf16_16816(sc[0], qa[k], b0);
                        mma_bf16_16816(sc[1], qa[k], b1);
                    }
                    uint32_t pa[4] = {0, 0, 0, 0};
                    float f[2] = {1.f, 1.f};
                    bool moved = false;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (i && !two) break;
                        float x[4] = {sc[0][2 * i] * p.scale_log2, sc[0][2 * i + 1] * p.scale_log2,
                                      sc[1][2 * i] * p.scale_log2, sc[1][2 * i + 1] * p.scale_log2};
                        if (see != 0xffffu) {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (!(see >> (q2 + (j & 1) + (j >> 1) * 8) & 1u)) x[j] = -INFINITY;
                        }
                        float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                        if (mx > m[i] + 8.f || m[i] == -INFINITY) {
                            f[i] = m[i] == -INFINITY ? 0.f : ex2(m[i] - mx);
                            m[i] = mx;
                            moved = true;
                        }
                        const float ref = m[i] == -INFINITY ? 0.f : m[i];
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[j] = ex2(x[j] - ref);
                        l[i] = l[i] * f[i] + ((x[0] + x[1]) + (x[2] + x[3]));
                        pa[i] = pack_bf16x2(x[0], x[1]);
                        pa[2 + i] = pack_bf16x2(x[2], x[3]);
                    }
                    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                        for (int i = 0; i < DH / 8; ++i) {
                            o[i][0] *= f[0];
                            o[i][1] *= f[0];
                            o[i][2] *= f[1];
                            o[i][3] *= f[1];
                        }
                    }
                    const uint32_t z0 = (see >> q2 & 1u ? 0xffffu : 0u) | (see >> (q2 + 1) & 1u ? 0xffff0000u : 0u);
                    const uint32_t z1 = (see >> (q2 + 8) & 1u ? 0xffffu : 0u) | (see >> (q2 + 9) & 1u ? 0xffff0000u : 0u);
#pragma unroll
                    for (int k = 0; k < DH / 16; ++k) {
                        uint32_t b[4];
                        ldmatrix_x4_trans(b, vt + (k >> 2) * S::SLAB + vrow * 128 + ((((k & 3) * 2 + vcol) ^ (vrow & 7)) << 4));
                        const uint32_t b0[2] = {b[0] & z0, b[1] & z1}, b1[2] = {b[2] & z0, b[3] & z1};
                        mma_bf16_16816(o[2 * k], pa, b0);
                        mma_bf16_16816(o[2 * k + 1], pa, b1);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sh.empty[s]));
            }
            // -------------------------------------------------------------- the item's result
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
                if ((lane & 3) == 0) sh.ml[warp][r + 8 * i] = make_float2(m[i], l[i]);
            }
            readers_sync();
            // All warps' sums relative to the largest maximum; those of a warp that saw nothing, or no score above
            // -inf, are times 0.  (Not left out: where its scores are NaN its maximum is -inf and its sums are NaN.)
            float top[2], sum[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                top[i] = -INFINITY;
                sum[i] = 0.f;
#pragma unroll
                for (int w = 0; w < kReaders; ++w) top[i] = fmaxf(top[i], sh.ml[w][r + 8 * i].x);
                const float ref = top[i] == -INFINITY ? 0.f : top[i];
#pragma unroll
                for (int w = 0; w < kReaders; ++w) {
                    const float2 ml = sh.ml[w][r + 8 * i];
                    sum[i] += __fmul_rn(ml.y, ex2(ml.x - ref));
                }
                const float f = ex2(m[i] - ref);
#pragma unroll
                for (int k = 0; k < DH / 8; ++k) {
                    o[k][2 * i] *= f;
                    o[k][2 * i + 1] *= f;
                }
            }
            __nv_bfloat16* out = p.out + (size_t)it.t * p.ld_out + (size_t)(it.head * c.rep + it.row0) * DH;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (i && !two) break;
                // Warps 2 and 3 give theirs to 0 and 1, warp 1 gives the sum to 0.
                if (warp >= 2)
#pragma unroll
                    for (int k = 0; k < DH / 8; ++k) sh.swap[warp - 2][k][lane] = make_float2(o[k][2 * i], o[k][2 * i + 1]);
                readers_sync();
                if (warp < 2)
#pragma unroll
                    for (int k = 0; k < DH / 8; ++k) {
                        const float2 x = sh.swap[warp][k][lane];
                        o[k][2 * i] += x.x;
                        o[k][2 * i + 1] += x.y;
                        if (warp == 1) sh.swap[1][k][lane] = make_float2(o[k][2 * i], o[k][2 * i + 1]);
                    }
                readers_sync();
                // The rows' result: in a cluster where the stages were (its item is the CTA's last).
                float* own = splits > 1 ? reinterpret_cast<float*>(smem) + 8 * i * DH : reinterpret_cast<float*>(sh.swap[0]);
                if (warp == 0) {
#pragma unroll
                    for (int k = 0; k < DH / 8; ++k) {
                        const float2 x = sh.swap[1][k][lane];
                        *reinterpret_cast<float2*>(own + r * DH + k * 8 + q2) = make_float2(o[k][2 * i] + x.x, o[k][2 * i + 1] + x.y);
                    }
                    if ((lane & 3) == 0) sh.mine[r + 8 * i] = make_float2(top[i], sum[i]);
                }
                readers_sync();
                if (splits > 1) continue;
                for (int e = threadIdx.x; e < min(8, it.rows - 8 * i) * (DH / 4); e += kReaders * 32) {
                    const int row = e / (DH / 4), col = e % (DH / 4) * 4;
                    put(it, out, 8 * i + row, col, sh.mine[8 * i + row], *reinterpret_cast<const float4*>(own + row * DH + col));
                }
                readers_sync();
            }
            if (splits > 1) break;                     // (a cluster has one item)
        }
    }
    if (splits == 1) {
        if (OWN) pdl_wait();
        return;
    }
    // ------------------------------------------------------------------- clusters
    cluster_sync();
    const Item& it = sh.item;                          // (kept: the loading warp says no more than that there are no more)
    const uint32_t own_at = sb, ml_at = smem_u32(sh.mine);
    auto peer2 = [](uint32_t at, uint32_t cta) {
        float2 v;
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(mapa_shared(at, cta)) : "memory");
        return v;
    };
    auto peer4 = [](uint32_t at, uint32_t cta) {
        float4 v;
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(mapa_shared(at, cta)) : "memory");
        return v;
    };
    __nv_bfloat16* out = p.out + (size_t)it.t * p.ld_out + (size_t)(it.head * c.rep + it.row0) * DH;
    for (int e = rank * kThreads + threadIdx.x; e < it.rows * (DH / 4); e += splits * kThreads) {
        const int row = e / (DH / 4), col = e % (DH / 4) * 4;
        float top = -INFINITY, sum = 0.f, a[4] = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < splits; ++w) add_source(peer2(ml_at + row * 8, w), peer4(own_at + (row * DH + col) * 4, w), true, top, sum, a);
        put(it, out, row, col, make_float2(top, sum), make_float4(a[0], a[1], a[2], a[3]));
    }
    cluster_sync();                                    // nobody ends while others read its sums
    if (OWN) pdl_wait();
}

// Lists as bits, for the attention kernel: a warp takes a token and key/value head, a window of pages at a time.  Pages from the step's
// first one on are seen as far as positions are.  Entries that do not fit are left out and flagged.
constexpr int kMaskWarps = 8, kMaskWords = 128;
__global__ void __launch_bounds__(kMaskWarps * 32) cache_masks_kernel(const __grid_constant__ CacheDev c,
                                                                      const __grid_constant__ BlocksParams p) {
    __shared__ uint32_t s_bits[kMaskWarps][kMaskWords];
    const int lane = threadIdx.x & 31;
    uint32_t* bits = s_bits[threadIdx.x >> 5];
    pdl_wait();
    pdl_trigger();
    const CachePlan pl = *c.plan;
    if (!pl.ok || !lists_dense(c, p.lists, pl)) return;
    if (blockIdx.x == 0 && threadIdx.x == 0) c.plan->pieces = 0;
    for (long long i = (long long)blockIdx.x * kMaskWarps + (threadIdx.x >> 5); i < (long long)p.T * c.Hkv;
         i += (long long)gridDim.x * kMaskWarps) {
        const CacheToken tok = c.tokens[i / c.Hkv];
        const int own = tok.base >> c.page_shift, listed = min(p.n, own), end = (tok.kv_len - 1 >> c.page_shift) / 32 + 1;
        const int* list = p.blocks + (size_t)i * p.n;
        if (lane == 0) *p.lists.mark(i) = 0;
        for (int w0 = 0; w0 < end; w0 += kMaskWords) {
            for (int w = lane; w < kMaskWords; w += 32) {
                const int n = own - (w0 + w) * 32;     // pages of the word before the step's own
                bits[w] = n >= 32 ? 0u : n > 0 ? ~0u << n : ~0u;
            }
            __syncwarp();
            ListReader reader;
            for (int j0 = 0; j0 < listed; j0 += 32) {
                const int j = j0 + lane;
                const bool there = j < listed;
                const int col = there ? list[j] : -1, before = there && j ? list[j - 1] : -1;
                const bool counts = reader.read(c, there, j, col, before, own) != kLeftOut;
                const int w = (col >> 5) - w0;
                if (counts && w >= 0 && w < kMaskWords) atomicOr(&bits[w], 1u << (col & 31));
            }
            if (w0 == 0)
                for (long long j = listed + lane; j < p.n; j += 32)
                    if (list[j] != -1) atomicCAS(c.err, 0, ERR_CACHE_BLOCKS);
            __syncwarp();
            for (int w = lane; w < min(kMaskWords, end - w0); w += 32) p.lists.bits(i)[w0 + w] = bits[w];
            __syncwarp();
        }
    }
}

template <int DH, bool OWN>
cudaError_t blocks_launch(const CacheDev& c, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const BlocksParams& p,
                          cudaStream_t st) {
    constexpr size_t smem = sizeof(Shared<DH>);
    static_assert(smem + 1024 <= 228 * 1024 / 2, "two CTAs to an SM");
    static_assert(Stage<DH>::COUNT <= 8, "barriers");
    static PerDevice attr;
    cudaError_t e = (cudaError_t)attr.get([] {
        return (int)cudaFuncSetAttribute(cache_blocks_kernel<DH, OWN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    }, true);
    if (e != cudaSuccess) return e;
    const long long items = (long long)p.T * c.Hkv * p.row_tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(OWN              ? 2LL * c.num_sms
                                  : p.splits == 1 ? std::min<long long>(items, 2LL * c.num_sms)
                                                  : items * p.splits));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute a[2];
    a[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    a[0].val.programmaticStreamSerializationAllowed = 1;
    a[1].id = cudaLaunchAttributeClusterDimension;
    a[1].val.clusterDim.x = (unsigned)p.splits;
    a[1].val.clusterDim.y = a[1].val.clusterDim.z = 1;
    cfg.attrs = a;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, cache_blocks_kernel<DH, OWN>, tm_k, tm_v, c, p);
}

}  // namespace

cudaError_t launch_cache_blocks(const CacheDev& c, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const BlocksParams& p,
                                cudaStream_t st) {
    return c.dh == 64 ? blocks_launch<64, false>(c, tm_k, tm_v, p, st) : blocks_launch<128, false>(c, tm_k, tm_v, p, st);
}

cudaError_t launch_cache_masks(const CacheDev& c, const BlocksParams& p, cudaStream_t st) {
    const long long blocks = ((long long)p.T * c.Hkv + kMaskWarps - 1) / kMaskWarps;
    return launch_pdl(cache_masks_kernel, dim3((unsigned)std::min<long long>(blocks, 8LL * c.num_sms)), dim3(kMaskWarps * 32), 0, st, c, p);
}

cudaError_t launch_cache_own(const CacheDev& c, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const BlocksParams& p,
                             cudaStream_t st) {
    return c.dh == 64 ? blocks_launch<64, true>(c, tm_k, tm_v, p, st) : blocks_launch<128, true>(c, tm_k, tm_v, p, st);
}

// As many CTAs to an item as fill the GPU twice, with a stage each at least.
int cache_blocks_splits(const CacheDev& c, long long items, int stages) {
    int splits = 1;
    while (splits < 8 && items * splits * 2 <= 2LL * c.num_sms && splits * 2 <= stages + 1) splits *= 2;
    return splits;
}

}  // namespace tmoe
