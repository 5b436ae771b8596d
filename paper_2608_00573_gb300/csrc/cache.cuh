// Internal declarations of the paged key/value cache: device records, kernel
// parameters and launchers.
#pragma once

#include <algorithm>

#include "internal.cuh"

namespace tmoe {

constexpr int kCacheMaxSeqs = 1024;
constexpr int kCacheTile = 128;        // rows of a query tile, keys of a key tile
constexpr int kTreeMax = 64;           // drafted tokens of a sequence (mask bits)
// Up to this many rows of an item, the CTA that writes a cut item's last part joins
// them, and a step is one launch; above, a second kernel does, with a CTA per 32 rows.
// Here against there, 32 heads on 8, one sequence of 6000 positions: 8 rows 17.4 us
// against 25.6, 16 rows 21.4 / 25.7, 24 rows 25.6 / 25.7, 32 rows 30.7 / 25.5, 128 rows
// 86 / 26; 8 sequences of 1000 to 8000: 8 rows 37.7 / 39.2, 16 rows 39.9 / 39.0, 24 rows
// 42.6 / 39.7, 32 rows 45.2 / 39.4.
constexpr int kJoinHereRows = 16;

// One listed sequence of the current step.
struct CacheSeq {
    int seq, q_off, q_len, kv_len;     // kv_len: its length with the new tokens
};

// One new token of the current step: its sequence, the sequence's lengths with the step's tokens
// and without, its position.
struct __align__(16) CacheToken {
    int seq, kv_len, base, pos;
};

// A group: up to two query tiles of one sequence, that is ntok consecutive new
// tokens (a tile holds tile_tokens = 128 / (q_heads / kv_heads) tokens, all query
// heads of one key/value head).  One item of attention work is a group and a
// key/value head; items are ordered by group, then head.
struct __align__(16) CacheGroup {
    long long pre;                     // cost of one head's items before this group
    int cost;                          // of one item: (key tiles + 1) << two query tiles
    int seq, kv_len;
    int row, ntok;                     // first packed token, tokens
    int first;                         // position of the first token
    int base;                          // positions before the step
    // Steps with groups of sequences (trimmoe_cache_share):
    int t0;                            // first key tile: those before it are the group of sequences' common ones
    int common;                        // the item is of those tiles, for all tokens of the group: kv_len and base end them
    int part_row;                      // its parts' first row, see cache_part_rows
};

// A CTA's share of the line on which the items' costs are laid end to end.
struct __align__(16) CacheShare {
    long long begin, end;
    long long within;                  // begin, from the start of the item that holds it
    int group, head;                   // that item
    int first, last;                   // CTAs that hold key tiles of it
    int pad[2];
    CacheGroup g;                      // its group
};

struct __align__(16) CachePlan {
    long long total;                   // cost of all items
    int n_groups;
    int n_ctas;                        // CTAs that share the line; 0: whole items, drawn from a counter
    int copies;                        // pages to copy (shared last pages)
    int ok;                            // 0: the step was refused
    int drawn, done;                   // items drawn beyond the first round, CTAs that have finished
    int pieces;                        // with groups of sequences and single tokens: what is not on the line; lists as
                                       // masks: items to be computed again
    int serial;                        // of the step (a list with groups is of the step with its number)
    // Lists with groups: what the attend that reads them has to be made for.
    int tokens, single;                // of the step; of single tokens (pieces and common items, see launch_cache_own)
};

__host__ __device__ inline int cache_two_tiles(int ntok, int tile_tokens) { return ntok > tile_tokens ? 1 : 0; }

// Key tiles of a group.  Short steps count to the sequence's end, because a draft
// mask may show any new token to any other.
__host__ __device__ inline int cache_group_tiles(int q_len, int kv_len, int first, int ntok) {
    const int keys = q_len <= kTreeMax ? kv_len : first + ntok;
    return (keys + kCacheTile - 1) / kCacheTile;
}

// Key tiles of an item of this cost (two: it has two query tiles), and how many of
// them the first x of its cost cover.
__host__ __device__ inline int cache_item_tiles(int cost, int two) { return (cost >> two) - 1; }
__host__ __device__ inline int cache_tiles_before(long long x, int cost, int two) {
    const long long n = cache_item_tiles(cost, two), t = x <= 0 ? 0 : (x + two) >> two;
    return (int)(x >= cost || t > n ? n : t);
}

// Steps of single tokens with groups of sequences: a piece of a sequence's own pages, for its token, or of a
// small group's common ones, for up to 16 rows (tokens by query heads of a key/value head).
struct __align__(16) CachePiece {
    int seq, tok, rows, whole;         // first token; whole: every position is seen
    int g0, g1, first_page, kv_len;    // stages of 64 positions from that page on; end of what is seen
    int part_row, head_step;           // part: row of the first key/value head, rows from head to head; -1: the result
    int pad[2];
};
constexpr int kPieceCuts = 24;         // of one sequence's or group's pages at most
constexpr int kPieces = 8192;          // 1024 tokens' and 512 groups' two, a piece more of each when they are cut, and 5 times
                                       // two CTAs an SM more, with room to spare

// Parts that hold a token: rows row + i * step, i < count, of query head 0 of a key/value head; warps: stored
// 32 rows of 4 columns side by side.
struct __align__(16) PartList {
    int row, step, count, warps;
};

// Where a token's parts are: pieces of its own pages and of common ones (rows of the first query head of the
// first key/value head, and how many), or items of the line (-1: none).
struct __align__(16) TokenParts {
    int own_row, own_n, own_item;
    int common_row, common_n, common_step, common_item;
    int pad;
};

// Rows of a part of an item, in a step with groups of sequences.  From 32 on they are whole
// warps, stored 32 rows of 4 columns side by side; fewer are stored row by row.
__host__ __device__ inline int cache_part_rows(int ntok, int tile_tokens, int rep) {
    if (ntok > tile_tokens) return kCacheTile + (((ntok - tile_tokens) * rep + 31) & ~31);
    return ntok * rep < 32 ? ntok * rep : (ntok * rep + 31) & ~31;
}
// The part of the group's item of key/value head `head` that CTA `cta` computes begins at row
// g.part_row + (head + cta) * cache_part_rows(g): along the line of items head and CTA both
// grow, so their sum names the pieces.

// With groups of sequences: cost of a key tile (both query tiles', when an item has two) and of an
// item's beginning and end, in kShareUnit us.  (Measured: 0.9 to 1.5, 1.4 to 1.9 and 3.2 to 4.4 us;
// sequences' own items are short, so this matters more than in other steps: with a tile and an end
// alike, the last CTA of 12 drafted trees ended at 97 us, the others at 63.  As 7, 4 and 16 here: those trees 94.0 us,
// 4 groups of 2 to 9 trees of 29, 16 heads on 16, 104; as 7, 5, 16 95.5 and 107, 8, 5, 16 94.8 and 104, 6, 5, 16 97
// and 111, 7, 6, 16 98 and 110, 7, 5, 12 95.7 and 106, 7, 5, 28 97.6 and 110.)
constexpr float kShareUnit = 0.25f;
__host__ __device__ inline int share_tile(int two) { return two ? 7 : 4; }
constexpr int kShareEnds = 16;
__host__ __device__ inline int share_tiles(int cost, int two) { return (cost - kShareEnds) / share_tile(two); }
// Key tiles that the first x of an item's cost cover.
__host__ __device__ inline int share_tiles_before(long long x, int cost, int two) {
    const long long n = share_tiles(cost, two), t = x <= 0 ? 0 : (x + share_tile(two) - 1) / share_tile(two);
    return (int)(t > n ? n : t);
}

// The CTA whose share of a line of cost W holds x: shares are [W b / n, W (b + 1) / n).
__host__ __device__ inline int cache_cta_of(long long x, long long W, int n) {
    return (int)(((x + 1) * n + W - 1) / W) - 1;
}

// The handle's device state, passed to every kernel by value.
struct CacheDev {
    int layers, Hq, Hkv, rep, dh, page, page_shift, n_pages, max_seqs, max_pages, T_max;
    int tile_tokens, num_sms;
    __nv_bfloat16 *k, *v;
    int *table, *length, *ref;
    // workspaces
    CachePlan* plan;
    CacheSeq* seqs;                    // [kCacheMaxSeqs]
    CacheGroup* groups;                // [T_max / (2 tile_tokens) + max_seqs + 1]
    CacheShare* shares;                // [num_sms]
    int* slot;                         // [T_max] page row (page * page_size + place) of each new token, -1 none
    int* pos;                          // [T_max] its position in its sequence
    int* owner;                        // [T_max] its sequence's place in seqs
    CacheToken* tokens;                // [T_max] valid behind a step that was not refused
    int2* copies;                      // [max(n_pages, max_seqs)] (from, to) pages
    int* fresh;                        // [n_pages] free pages taken by a step; new place of each page (compact)
    int* base;                         // [max_seqs] length before the sequence's last step
    int* holders;                      // [n_pages] a page's entries in table, counted by compact, 0 between calls
    // Parts of cut items: two buffers per CTA, for the item that its share begins in and
    // the one that it ends in; rows 0..127 and 128..255 from the two slots.
    float* part_o;                     // [2 num_sms][256][dh] sums of p v (order within: cache_attention.cu)
    float2* part_ml;                   // [2 num_sms][256] row maxima and sums of p
    int* arrived;                      // [num_sms] parts written of the item that a CTA began, 0 between calls
    // Bounds of the keys of whole pages (trimmoe_cache_set_bounds), or NULL.
    int8_t* codes;                     // [layers][n_pages][Hkv][2][dh]
    float* scales;                     // [layers][n_pages][Hkv]
    uint32_t* scores;                  // [cache_score_keys] of a choice, as ordered whole numbers
    // Steps with groups of sequences: the list of items is in plan, shares and groups and the parts in
    // part_o and part_ml as for other steps, but these are other buffers (the host side chooses).
    int shared;
    const CachePlan* step_plan;        // the step's own plan
    TokenParts* parts_of;              // [T]
    PartList* lists;                   // [T][Hkv][2] where a token's parts are: common ones, own ones
    CachePiece* pieces;                // [kPieces]
    int* common;                       // [max_seqs] key tiles that a group of sequences has in common
    int2* cut;                         // [groups][Hkv] first CTA that holds tiles of an item, how many do
    int* err;
    int* refused;                      // behind err: the last step was refused and stats has not reset that yet
};

// Host arrays of a call travel as kernel parameters (no staging buffer whose
// lifetime would have to be tracked; a capture keeps them).
template <int N>
struct CacheList {
    int n;
    int a[N], b[N];
};

struct AppendParams {
    const __nv_bfloat16* qkv;
    __nv_bfloat16* q_out;
    int ld_qkv, ld_q, T, norm, rope, split;
    long long layer_off;               // elements before the layer in k and v
    const __nv_bfloat16 *gamma_q, *gamma_k;
    float eps;
    const int* pos;
    uint64_t turn[64];                 // turns per position of each pair, in units of 2^-64
};

// Lists of pages as bits, for the attention kernel to mask with (cache_attend_blocks).
struct PageLists {
    uint32_t* mask;                    // [T][Hkv][words + 2], or NULL: lists are followed instead
    int words;
    long long stages;                  // of 64 listed positions, all tokens and heads (and 16 of their rows)
    __host__ __device__ uint32_t* bits(long long item) const { return mask + item * (words + 2); }
    __device__ uint32_t* mark(long long item) const { return bits(item) + words; }        // the item is computed again
    __device__ uint32_t* marked(long long i) const { return bits(i) + words + 1; }        // i-th such item
};

struct AttendParams {
    const uint64_t* tree;
    __nv_bfloat16* out;
    int ld_out;
    int join_here;                     // the attention kernel joins cut items itself
    float scale_log2;
    int T;
    PageLists lists;
    int single, alone;                 // with groups: of single tokens; all of them small (no attention kernel)
};

// attend_blocks: q and out as for attend.
struct BlocksParams {
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    const int* blocks;                 // [T][Hkv][n]
    const uint64_t* tree;
    int ld_q, ld_out, T, n;
    int row_tiles;                     // of 16 query heads of a key/value head
    int splits;                        // CTAs of an item
    int alone;                         // pieces: there is no attention kernel to run beside
    float scale_log2;
    PageLists lists;
};

struct SelectParams {
    const __nv_bfloat16* q;
    int* blocks;                       // [T][Hkv][n]
    int ld_q, T, n, first, last, layer, max_q;
};

// Room for the scores of a choice: 8 M blocks (32 MB), fewer when no step has as many, one token's
// at least.
inline size_t cache_score_keys(const CacheDev& c) {
    const size_t row = (((size_t)c.max_pages + 3) & ~size_t(3)) * c.Hkv;
    return std::max(row, std::min(row * c.T_max, (size_t)8 << 20));
}

// Steps of single tokens with groups of sequences: groups with at most this many tiles of 16 rows are small.
constexpr int kSmallTiles = 2;
__host__ __device__ inline int small_tiles(int tokens, int rep) { return (tokens + 16 / rep - 1) / (16 / rep); }

// Steps with groups of sequences: rows (tokens times query heads) at most, and what that allows in a cache whose steps
// have T_max tokens.
constexpr int kShareRows = 65536;
__host__ __device__ inline int cache_share_tokens(const CacheDev& c) {
    const int most = kShareRows / c.Hq;
    return c.T_max < most ? c.T_max : most;
}
// Every token has its own and at most one common part, a part's rows are at most twice its
// tokens' (whole warps, tiles that rep does not divide), a cut adds one part of 256 rows, and
// an item's rows begin at a multiple of 32.  Of single tokens common parts alone are on the line; pieces' parts lie row by
// row behind those: one for each token and of each kind, and 16 rows more for a cut and head, of which there
// are fewer than 6 an SM (cache_share_kernel).
__host__ __device__ inline long long cache_share_groups(const CacheDev& c) {
    const long long T = cache_share_tokens(c), n = T / (2 * c.tile_tokens) + c.max_seqs + 1;
    return 2 * (T < n ? T : n);
}
__host__ __device__ inline long long cache_piece_rows(const CacheDev& c) {
    return 2LL * cache_share_tokens(c) * c.Hq + 256LL * c.num_sms + 32 * cache_share_groups(c);
}
__host__ __device__ inline long long cache_share_part_rows(const CacheDev& c) {
    return cache_piece_rows(c) + 2LL * cache_share_tokens(c) * c.Hq + 128LL * c.num_sms;
}

cudaError_t launch_cache_step(const CacheDev& c, int n, const int* seq, const int* q_len, int T, cudaStream_t st);
cudaError_t launch_cache_fork(const CacheDev& c, int n, const int* src, const int* dst, cudaStream_t st);
cudaError_t launch_cache_truncate(const CacheDev& c, int n, const int* seq, const int* length, cudaStream_t st);
cudaError_t launch_cache_accept(const CacheDev& c, int n, const int* seq, const int* n_acc, const int* path,
                                int ld_path, cudaStream_t st);
cudaError_t launch_cache_compact(const CacheDev& c, cudaStream_t st);
cudaError_t launch_cache_append(const CacheDev& c, const AppendParams& p, cudaStream_t st);
// Bounds of the pages that the step filled (whole: of all full pages of its sequences) in one
// layer; n listed sequences with at most max_q new tokens.
cudaError_t launch_cache_bounds(const CacheDev& c, int layer, int n, int max_q, int whole, cudaStream_t st);
// Of those that accepted drafts filled, in all layers (accepted: the accept kernel's new lengths, -1: none).
cudaError_t launch_cache_bounds_accepted(const CacheDev& c, int n, const int* seq, const int* n_acc, const int* accepted,
                                         cudaStream_t st);
cudaError_t launch_cache_select(const CacheDev& c, const SelectParams& p, cudaStream_t st, int& launches);
cudaError_t launch_cache_blocks(const CacheDev& c, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                                const BlocksParams& p, cudaStream_t st);
// Its lists as bits (p.lists).
cudaError_t launch_cache_masks(const CacheDev& c, const BlocksParams& p, cudaStream_t st);
// A step of single tokens with groups of sequences, beside the attention kernel: the pieces.
cudaError_t launch_cache_own(const CacheDev& c, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const BlocksParams& p,
                             cudaStream_t st);
// Behind both: the sums of a step's parts.
cudaError_t launch_cache_join(const CacheDev& c, const AttendParams& p, cudaStream_t st);
// CTAs of one of `items` items with about as many stages of 64 positions.
int cache_blocks_splits(const CacheDev& c, long long items, int stages);
// A record as it is in L2.  A kernel that runs beside the one before it, and reads what kernels before that
// one have written without a wait of its own, may find older contents in L1.
template <class R>
__device__ __forceinline__ R from_l2(const R* at) {
    static_assert(sizeof(R) % 16 == 0, "whole 16-byte words");
    union {
        R r;
        int4 w[sizeof(R) / 16];
    } u;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(R) / 16); ++i) u.w[i] = __ldcg(reinterpret_cast<const int4*>(at) + i);
    return u.r;
}

// Whether the step's lists are masks of an attention over all pages (else each is followed), in ns of an SM:
// that attention takes kDenseEnds, with its launches, and kDenseCost for a key tile and a query tile; a followed stage
// kStageCost.  Measured, 800 tokens of 3 chunks, masks against lists, 32 heads on 8, 24 pages of 64: behind 6000 to
// 15000 positions 168 us / 436, 15000 to 30000 308 / 432, 30000 to 60000 582 / 447; 16 heads on 16, 96 pages of
// 16: 148 / 1174, 280 / 1184; 12 heads of 64 columns, 40 pages of 32: 84 / 458, 141 / 456; 20 times 17 tokens behind
// 2000 to 9000, 32 heads on 8: 93 / 177; 64 tokens behind 16000, 32 pages: 47 / 53.
constexpr int kDenseEnds = 33000, kDenseCost = 1050, kStageCost = 420;
__device__ __forceinline__ bool lists_dense(const CacheDev& c, const PageLists& l, const CachePlan& pl) {
    return l.mask && (long long)kDenseEnds * c.num_sms + pl.total * kDenseCost <= l.stages * kStageCost;
}

// A list with groups is not one that this attend's launches compute: it is not of the last step (a captured attend
// replayed without its share), of another number of tokens, of single tokens and the launches are not, or the other way
// round, or has common items and there is no attention kernel for them (alone).
__device__ __forceinline__ bool share_stale(const CacheDev& c, const CachePlan& pl, int tokens, int single, int alone) {
    const bool stale = pl.serial != __ldcg(&c.step_plan->serial) || pl.tokens != tokens || pl.single != single ||
                       (alone && pl.n_groups);
    if (stale && blockIdx.x == 0 && threadIdx.x == 0) atomicCAS(c.err, 0, ERR_CACHE_STATE);
    return stale;
}

// The list of items of a step whose listed sequences form n groups.  single: each has one new token at most,
// and launch_cache_own runs too.
cudaError_t launch_cache_share(const CacheDev& c, int n, const int* counts, int n_seqs, int T, int single, cudaStream_t st);
cudaError_t launch_cache_attend(const CacheDev& c, const CUtensorMap& tm_q, const CUtensorMap& tm_k,
                                const CUtensorMap& tm_v, const AttendParams& p, int max_rows, cudaStream_t st);

// Device helpers of the attention kernels.

__device__ __forceinline__ PartList item_parts(const CacheDev& c, int item, int head, int t) {
    if (item < 0) return PartList{0, 0, 0, 0};
    const int2 cut = c.cut[(size_t)item * c.Hkv + head];
    const CacheGroup g = c.groups[item];
    const int rows = cache_part_rows(g.ntok, c.tile_tokens, c.rep), in = t - g.row;
    return PartList{g.part_row + (head + cut.x) * rows +
                        (in >= c.tile_tokens ? 128 + (in - c.tile_tokens) * c.rep : in * c.rep),
                    rows, cut.y, rows >= 32};
}
__device__ __forceinline__ PartList own_parts(const CacheDev& c, const TokenParts& p, int head, int t) {
    if (p.own_n) return PartList{p.own_row + head * p.own_n * c.rep, c.rep, p.own_n, 0};
    return item_parts(c, p.own_item, head, t);
}
__device__ __forceinline__ PartList common_parts(const CacheDev& c, const TokenParts& p, int head, int t) {
    if (p.common_n) return PartList{p.common_row + head * p.common_n * p.common_step, p.common_step, p.common_n, 0};
    return item_parts(c, p.common_item, head, t);
}

__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// One more source of a row (there: it is one): its maximum and sum (x), added to top and l; fa and fb are the
// factors of what was summed before and of the source.  A source that saw nothing is (-inf, 0) and adds 0.  The
// maximum says nothing of NaN, which fmaxf leaves out: (-inf, NaN) is a source of NaN scores, and they stay.
__device__ __forceinline__ void join_source(float2 x, bool there, float& top, float& l, float& fa, float& fb) {
    const float m = there ? fmaxf(top, x.x) : top, ref = m == -INFINITY ? 0.f : m;
    fa = ex2(top - ref);
    fb = ex2(x.x - ref);
    top = m;
    l = there ? l * fa + x.y * fb : l;
}

// Adds a source's four columns of a row.  (Without a branch: loads would be moved behind it, one by one.)
__device__ __forceinline__ void add_source(float2 ml, float4 x, bool there, float& top, float& l, float (&a)[4]) {
    float fa, fb;
    join_source(ml, there, top, l, fa, fb);
    a[0] = there ? a[0] * fa + x.x * fb : a[0];
    a[1] = there ? a[1] * fa + x.y * fb : a[1];
    a[2] = there ? a[2] * fa + x.z * fb : a[2];
    a[3] = there ? a[3] * fa + x.w * fb : a[3];
}
// Adds four columns of query head `row` from two lists of parts, the first one's first; B are read at a time.
template <int DH, int B>
__device__ __forceinline__ void add_parts(const CacheDev& c, const PartList& p0, const PartList& p1, int row, int col, float& top,
                                          float& l, float (&a)[4]) {
    const int n = p0.count + p1.count;
    for (int k0 = 0; k0 < n; k0 += B) {
        float2 ml[B];
        float4 x[B];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int k = min(k0 + i, n - 1);
            const bool second = k >= p0.count;
            const long long at = (second ? p1.row + (k - p0.count) * p1.step : p0.row + k * p0.step) + row;
            const bool warps = second ? p1.warps : p0.warps;
            const float* src = c.part_o + (warps ? (at & ~31LL) * DH + (at & 31) * 4 + col * 32 : at * DH + col);
            ml[i] = __ldcg(c.part_ml + at);
            x[i] = __ldcg(reinterpret_cast<const float4*>(src));
        }
#pragma unroll
        for (int i = 0; i < B; ++i) add_source(ml[i], x[i], k0 + i < n, top, l, a);
    }
}

// Bounded wait by all lanes of a warp.  A probe sleeps until the phase ends or up to
// about a microsecond; after 2^22 of them, some seconds, the waiter raises the CTA's
// abort flag and the error word; it also gives up when another role has.  The loop is
// inside the asm so that control flow stays uniform for the compiler (see elect_one).
// Returns 0 when the phase ended, 1 when given up.
__device__ __forceinline__ uint32_t wait_probes(uint32_t bar, uint32_t parity, uint32_t abort_flag, int* err) {
    uint32_t gave_up;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b32 n, a;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "mov.b32 n, 0;\n\t"
        "mov.b32 %0, 0;\n\t"
        "@p bra DONE;\n\t"
        "PROBE:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 1000;\n\t"
        "@p bra DONE;\n\t"
        "ld.volatile.shared.b32 a, [%3];\n\t"
        "setp.ne.b32 p, a, 0;\n\t"
        "@p bra GONE;\n\t"
        "add.s32 n, n, 1;\n\t"
        "setp.lt.s32 p, n, 4194304;\n\t"
        "@p bra PROBE;\n\t"
        "st.volatile.shared.b32 [%3], 1;\n\t"
        "atom.global.cas.b32 a, [%4], 0, %5;\n\t"
        "GONE:\n\t"
        "mov.b32 %0, 1;\n\t"
        "DONE:\n\t}"
        : "=&r"(gave_up)
        : "r"(bar), "r"(parity), "r"(abort_flag), "l"(err), "n"((int)ERR_TIMEOUT_CACHE_ATTN)
        : "memory");
    return gave_up;
}

}  // namespace tmoe
