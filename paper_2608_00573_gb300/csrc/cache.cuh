// Internal declarations of the paged key/value cache: device records, kernel
// parameters and launchers.
#pragma once

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
    int pad[3];
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

struct CachePlan {
    long long total;                   // cost of all items
    int n_groups;
    int n_ctas;                        // CTAs that share the line; 0: whole items, drawn from a counter
    int copies;                        // pages to copy (shared last pages)
    int ok;                            // 0: the step was refused
    int drawn, done;                   // items drawn beyond the first round, CTAs that have finished
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
    int2* copies;                      // [max(n_pages, max_seqs)] (from, to) pages
    int* fresh;                        // [n_pages] free pages taken by a step; new place of each page (compact)
    int* base;                         // [max_seqs] length before the sequence's last step
    int* holders;                      // [n_pages] a page's entries in table, counted by compact, 0 between calls
    // Parts of cut items: two buffers per CTA, for the item that its share begins in and
    // the one that it ends in; rows 0..127 and 128..255 from the two slots.
    float* part_o;                     // [2 num_sms][256][dh] sums of p v (order within: cache_attention.cu)
    float2* part_ml;                   // [2 num_sms][256] row maxima and sums of p
    int* arrived;                      // [num_sms] parts written of the item that a CTA began, 0 between calls
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

struct AttendParams {
    const uint64_t* tree;
    __nv_bfloat16* out;
    int ld_out;
    int join_here;                     // the attention kernel joins cut items itself
    float scale_log2;
};

cudaError_t launch_cache_step(const CacheDev& c, int n, const int* seq, const int* q_len, int T, cudaStream_t st);
cudaError_t launch_cache_fork(const CacheDev& c, int n, const int* src, const int* dst, cudaStream_t st);
cudaError_t launch_cache_truncate(const CacheDev& c, int n, const int* seq, const int* length, cudaStream_t st);
cudaError_t launch_cache_accept(const CacheDev& c, int n, const int* seq, const int* n_acc, const int* path,
                                int ld_path, cudaStream_t st);
cudaError_t launch_cache_compact(const CacheDev& c, cudaStream_t st);
cudaError_t launch_cache_append(const CacheDev& c, const AppendParams& p, cudaStream_t st);
cudaError_t launch_cache_attend(const CacheDev& c, const CUtensorMap& tm_q, const CUtensorMap& tm_k,
                                const CUtensorMap& tm_v, const AttendParams& p, int max_rows, cudaStream_t st);

}  // namespace tmoe
