// Attention over the paged cache: prompts, single tokens and drafted trees.
//
// A query tile is 128 rows: tile_tokens = 128 / rep consecutive new tokens of one
// sequence, each with the rep = q_heads / kv_heads query heads of one key/value
// head, so that a key tile read once serves all heads that share it.  For a tile and
// key tiles of 128 positions (FlashAttention's running softmax, in base 2):
//
//   S = Q K^T                       tcgen05.mma, M = 128, N = 128, K = D -> TMEM
//   m' = max(m, max_j s_j);  p_j = 2^(scale' (s_j - m'))   fp32, one row per thread
//   O = O 2^(scale' (m - m')) + P V  tcgen05.mma, A = P from TMEM (bf16), B = V from
//                                   shared memory with its D axis contiguous
//   l = l 2^(...) + sum_j p_j;      out = O / l
//
// O is rescaled only when some row's maximum grew by more than 2^8: until then p
// stays below 2^8, which costs no precision in floating point, and the extra
// pass over O in TMEM is rare.
//
// A CTA holds two query tiles in flight ("slots", each with its own S and O in
// TMEM and its own group of four softmax warps), so that one slot's products run
// under the other's softmax.  In a group of more than tile_tokens tokens the
// slots are its two query tiles and share every key tile; in a smaller group
// (single tokens, short drafts) both slots hold the same tile and take the even and
// the odd key tiles, and their results are joined at the end.
//
// Work is split evenly whatever the lengths: the items' costs are laid end to
// end and each CTA takes the same share of the line, cutting items at key tiles
// (cache_pages.cu makes the list).  A cut item's parts go to a buffer, at most two per
// CTA, and cache_join_kernel adds them in the order of the keys, so results do
// not depend on timing.
//
// Masked places never reach a result: scores are replaced, not added to; value
// rows that no row of the item sees are zeroed in shared memory (0 * NaN would
// be NaN), and a tile whose partly masked value rows hold an infinity or a NaN is
// multiplied by the softmax warps themselves, skipping masked keys.
//
// Bounds: prompts the tensor cores (and the exponentials: 128 x 128 per 4 x 128 x
// 128 x D multiply-adds); decoding HBM, each K and V row once per query tile.
#include <algorithm>

#include "cache.cuh"

namespace tmoe {

namespace {

constexpr int kThreads = 384;       // load, MMA and two guard warps; two groups of four softmax warps
constexpr int kSegSlots = 4;
constexpr uint32_t kTmemCols = 512; // S in two 128-column buffers (P over S), O in two D-column buffers
constexpr int kBox = 128 * 128;     // bytes of 128 rows x 64 columns

template <int DH>
struct Layout {
    static constexpr int KB = DH / 64;
    static constexpr int TILE = KB * kBox;
    static constexpr int STAGES = 160 * 1024 / TILE;     // ring of K and V tiles
    static constexpr int Q = 0;                          // two query tiles; joins odd and even key tiles' O
    static constexpr int RING = 2 * TILE;
    static constexpr int BYTES = RING + STAGES * TILE;
};

// A CTA's piece of an item.
struct Seg {
    int valid;
    int seq, kv_len, row, ntok, first, base, head;
    int t0, t1;          // key tiles
    int part;            // part buffer, -1: the whole item
    int pad;
};

struct __align__(8) Bars {
    uint64_t kv_full[10], kv_empty[10];
    uint64_t go[10], guard[10];   // masked value tile has landed / has been guarded, in the order of such tiles
    uint64_t q_full, q_empty;
    uint64_t s_full[2], p_full[2], o_full[2];
    uint64_t x_full[4];
    uint64_t seg_full[kSegSlots], seg_empty[kSegSlots];
    Seg seg[kSegSlots];
    int bad[10][2];      // guard warps' finding per ring stage
    float2 xml[128];     // odd slot's maximum and sum per row
    uint32_t tmem_base;
    int abort_flag;
};
constexpr int kSegReaders = 1 + 2 + 8;   // warps that read a segment

template <int DH>
constexpr size_t smem_bytes() {
    return 1024 + (size_t)Layout<DH>::BYTES + sizeof(Bars);
}

// What every role derives from a segment.
struct SegInfo {
    bool dual;
    int n0, n1;          // slot s works on key tiles below n_s
    int kmax;            // positions that some row sees
    int kall;            // positions that every row sees
};

__device__ __forceinline__ SegInfo seg_info(const Seg& g, int tile_tokens, bool tree) {
    SegInfo s;
    s.dual = g.ntok > tile_tokens;
    s.kmax = tree ? g.kv_len : g.first + g.ntok;
    s.kall = tree ? g.base : g.first + 1;
    s.n1 = min(g.t1, (s.kmax + kCacheTile - 1) / kCacheTile);
    s.n0 = s.n1;
    if (s.dual && !tree) s.n0 = min(s.n1, (g.first + tile_tokens + kCacheTile - 1) / kCacheTile);
    return s;
}

// Share of one CTA on the line of items, in the cost units of the plan.
__device__ __forceinline__ long long share_begin(const CachePlan& pl, int b) { return pl.total * b / pl.n_ctas; }

// Key tiles [t0, t1) of an item (n of them, `a` products each) that the stretch
// [x0, x1) of its cost covers; stretches that meet cover meeting ranges.
__device__ __forceinline__ void stretch_tiles(long long x0, long long x1, long long cost, int a, int n, int* t0, int* t1) {
    *t0 = (int)min((long long)n, (x0 + a - 1) / a);
    *t1 = x1 >= cost ? n : (int)min((long long)n, (x1 + a - 1) / a);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 1)
cache_attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                       const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CacheDev c,
                       const __grid_constant__ AttendParams p) {
    using L = Layout<DH>;
    constexpr int ST = L::STAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    uint8_t* smem = smem_raw + (((raw + 1023u) & ~1023u) - raw);
    const uint32_t sb = smem_u32(smem);
    Bars* bars = reinterpret_cast<Bars*>(smem + L::BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool tree = p.tree != nullptr;
    const int TT = c.tile_tokens, rep = c.rep;

    if (threadIdx.x == 0) {
        for (int s = 0; s < ST; ++s) {
            mbar_init(smem_u32(&bars->kv_full[s]), 1);
            mbar_init(smem_u32(&bars->kv_empty[s]), 1);
            mbar_init(smem_u32(&bars->go[s]), 1);
            mbar_init(smem_u32(&bars->guard[s]), 2);
        }
        mbar_init(smem_u32(&bars->q_full), 1);
        mbar_init(smem_u32(&bars->q_empty), 8);
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&bars->s_full[s]), 1);
            mbar_init(smem_u32(&bars->p_full[s]), 4);
            mbar_init(smem_u32(&bars->o_full[s]), 1);
        }
        for (int s = 0; s < 4; ++s) mbar_init(smem_u32(&bars->x_full[s]), 1);
        for (int s = 0; s < kSegSlots; ++s) {
            mbar_init(smem_u32(&bars->seg_full[s]), 1);
            mbar_init(smem_u32(&bars->seg_empty[s]), kSegReaders);
        }
        bars->abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_q);
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
    }
    if (warp == 0) tmem_alloc(smem_u32(&bars->tmem_base), kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = bars->tmem_base;
    volatile int* abort_flag = &bars->abort_flag;
    pdl_wait();
    pdl_trigger();

    auto wait1 = [&](uint64_t* bar, uint32_t parity) {
        return mbar_wait_bounded(smem_u32(bar), parity & 1u, abort_flag, c.err, ERR_TIMEOUT_CACHE_ATTN);
    };
    auto wait_warp = [&](uint64_t* bar, uint32_t parity) {      // lane 0 waits for the warp
        int ok = 1;
        if (lane == 0) ok = wait1(bar, parity);
        return __shfl_sync(0xffffffffu, ok, 0) != 0;
    };
    // The it-th segment of this CTA (false: none left, or aborted).
    auto next_seg = [&](int it, Seg& g) {
        const int s = it % kSegSlots;
        if (!wait_warp(&bars->seg_full[s], it / kSegSlots)) return false;
        g = bars->seg[s];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->seg_empty[s]));
        return g.valid != 0;
    };

    // Registers go from the first four warps to the softmax warps (80 x 128 + 208 x 256 of the
    // 168 x 384 at launch).  The branches do not meet again before the roles end:
    // where they meet, the compiler takes the smaller number.
    if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 0) {
        // ------------------------------------------------ segments and loads
        const CachePlan pl = *c.plan;
        const int b = blockIdx.x;
        int it = 0;
        uint32_t cnt = 0;                       // ring entries issued
        bool ok = true;
        auto give_seg = [&](const Seg& g) {
            const int s = it % kSegSlots;
            if (it >= kSegSlots && !wait_warp(&bars->seg_empty[s], it / kSegSlots - 1)) return false;
            if (lane == 0) {
                bars->seg[s] = g;
                mbar_arrive(smem_u32(&bars->seg_full[s]));
            }
            ++it;
            return true;
        };
        const int pages_per_tile = kCacheTile >> c.page_shift;
        const int my_page = lane / L::KB, my_kb = lane % L::KB;
        int nseg = 0;
        if (pl.ok && b < pl.n_ctas) {
            long long x = share_begin(pl, b);
            const long long x_end = share_begin(pl, b + 1);
            int r = c.cta_group[b];
            CacheGroup g = c.groups[r];
            long long g_next = c.groups[r + 1].pre;
            while (ok && x < x_end) {
                const long long cost = g_next - g.pre, within = x - g.pre * c.Hkv;
                const int head = (int)(within / cost);
                const long long x0 = within - head * cost, x1 = min(cost, x0 + (x_end - x));
                const int a = cache_tile_cost(g.ntok, TT);
                const int n = (int)(cost / a) - 1;
                Seg sg;
                sg.valid = 1;
                sg.seq = g.seq;
                sg.kv_len = g.kv_len;
                sg.row = g.row;
                sg.ntok = g.ntok;
                sg.first = g.first;
                sg.base = g.base;
                sg.head = head;
                stretch_tiles(x0, x1, cost, a, n, &sg.t0, &sg.t1);
                sg.part = (sg.t0 == 0 && sg.t1 == n) ? -1 : (sg.t0 > 0 ? 2 * b : 2 * b + 1);
                sg.pad = 0;
                x += x1 - x0;
                if (x >= g_next * c.Hkv && x < x_end) {
                    ++r;
                    g = c.groups[r];
                    g_next = c.groups[r + 1].pre;
                }
                if (sg.t0 >= sg.t1) continue;
                if (!give_seg(sg)) break;
                const SegInfo si = seg_info(sg, TT, tree);
                // Queries, once the previous segment's products have read theirs.
                if (nseg > 0 && !wait_warp(&bars->q_empty, nseg - 1)) break;
                if (lane == 0) {
                    const uint32_t qb = smem_u32(&bars->q_full);
                    const uint32_t bytes = (uint32_t)L::KB * TT * rep * 128;
                    mbar_arrive_expect_tx(qb, si.dual ? 2 * bytes : bytes);
                    for (int s = 0; s < (si.dual ? 2 : 1); ++s)
                        for (int kb = 0; kb < L::KB; ++kb)
                            tma_load_3d(sb + L::Q + s * L::TILE + kb * kBox, &tm_q, kb * 64, sg.head * rep,
                                        sg.row + s * TT, qb);
                }
                __syncwarp();
                ++nseg;
                // Keys and values: page indices of the tiles ahead travel in registers.
                const int n_pages = (si.kmax + c.page - 1) >> c.page_shift;
                const int* row = c.table + (size_t)sg.seq * c.max_pages;
                auto page_of = [&](int t) {
                    const int j = t * pages_per_tile + my_page;
                    return (lane < pages_per_tile * L::KB && t < sg.t1 && j < n_pages) ? row[j] : -1;
                };
                auto load = [&](const CUtensorMap* tm, int t, int id) {
                    const int s = (int)(cnt % ST);
                    if (cnt >= (uint32_t)ST && !wait_warp(&bars->kv_empty[s], cnt / ST - 1)) return false;
                    const int have = max(0, min(pages_per_tile, n_pages - t * pages_per_tile));
                    const uint32_t fb = smem_u32(&bars->kv_full[s]);
                    if (lane == 0) mbar_arrive_expect_tx(fb, (uint32_t)have * c.page * 128 * L::KB);
                    __syncwarp();
                    if (lane < pages_per_tile * L::KB && my_page < have)
                        tma_load_2d(sb + L::RING + s * L::TILE + my_kb * kBox + my_page * c.page * 128, tm, my_kb * 64,
                                    (id * c.Hkv + sg.head) << c.page_shift, fb);
                    __syncwarp();
                    ++cnt;
                    return true;
                };
                int id0 = page_of(sg.t0), id1 = page_of(sg.t0 + 1), id2 = page_of(sg.t0 + 2);
                ok = load(&tm_k, sg.t0, id0);
                if (ok && !si.dual && sg.t0 + 1 < sg.t1) ok = load(&tm_k, sg.t0 + 1, id1);
                for (int t = sg.t0; ok && t < sg.t1; ++t) {
                    const int id3 = page_of(t + 3);
                    ok = load(&tm_v, t, id0);
                    const int tk = t + (si.dual ? 1 : 2);
                    if (ok && tk < sg.t1) ok = load(&tm_k, tk, si.dual ? id1 : id2);
                    id0 = id1;
                    id1 = id2;
                    id2 = id3;
                }
            }
        }
        if (ok && !*abort_flag) {
            Seg end = {};
            give_seg(end);
        }
        // The last copies have landed, and been read unless the CTA gave up, before
        // it ends.
        const uint32_t tail = min(cnt, (uint32_t)ST);
        if (lane == 0) {
            int never = 0;
            for (uint32_t k = cnt - tail; k < cnt; ++k)
                mbar_wait_bounded(smem_u32(&bars->kv_full[k % ST]), (k / ST) & 1, &never, c.err, ERR_TIMEOUT_CACHE_ATTN);
            if (nseg > 0)
                mbar_wait_bounded(smem_u32(&bars->q_full), (nseg - 1) & 1, &never, c.err, ERR_TIMEOUT_CACHE_ATTN);
        }
        __syncwarp();
        for (uint32_t k = cnt - tail; k < cnt; ++k)
            if (!wait_warp(&bars->kv_empty[k % ST], k / ST)) break;
    } else if (warp == 1) {
        // -------------------------------------------------------------- MMAs
        constexpr uint32_t idS = idesc_bf16_f32(128, 128);
        constexpr uint32_t idO = idesc_bf16_f32(128, DH) | kIdescBMn;
        uint32_t cnt = 0, masked = 0, np[2] = {0, 0};     // ring entries, masked tiles, P tiles of each slot
        Seg g;
        bool ok = true;
        for (int it = 0; ok && next_seg(it, g); ++it) {
            if (lane == 0) {
                const SegInfo si = seg_info(g, TT, tree);
                const int lead = si.dual ? 1 : 2, nt = g.t1 - g.t0;
                const int lim[2] = {si.n0, si.n1};
                bool began[2] = {false, false};
                auto k_entry = [&](int i) { return cnt + i + max(0, i - lead + 1); };
                auto v_entry = [&](int i) { return cnt + i + min(nt, i + lead); };
                auto mma_s = [&](int slot, uint32_t e) {
                    const uint32_t qa = sb + L::Q + (si.dual ? slot * L::TILE : 0);
                    const uint32_t ka = sb + L::RING + (e % ST) * L::TILE;
#pragma unroll
                    for (int kk = 0; kk < DH / 16; ++kk)
                        tc_mma_bf16(tbase + slot * 128, smem_desc_sw128(qa + (kk >> 2) * kBox + (kk & 3) * 32),
                                    smem_desc_sw128(ka + (kk >> 2) * kBox + (kk & 3) * 32), idS, kk ? 1u : 0u);
                    tc_commit(smem_u32(&bars->s_full[slot]));
                };
                ok = wait1(&bars->q_full, it);
                for (int i = 0; ok && i < min(lead, nt); ++i) {
                    const uint32_t e = k_entry(i);
                    ok = wait1(&bars->kv_full[e % ST], e / ST);
                    if (!ok) break;
                    tc_fence_after();
                    if ((si.dual || i == 0) && g.t0 + i < lim[0]) mma_s(0, e);
                    if ((si.dual || i == 1) && g.t0 + i < lim[1]) mma_s(1, e);
                    tc_commit(smem_u32(&bars->kv_empty[e % ST]));
                }
                for (int i = 0; ok && i < nt; ++i) {
                    const int t = g.t0 + i;
                    const uint32_t ev = v_entry(i), ek = k_entry(i + lead);
                    const bool more = i + lead < nt;
                    ok = wait1(&bars->kv_full[ev % ST], ev / ST);
                    if (!ok) break;
                    bool bad = false;
                    if ((t + 1) * kCacheTile > si.kall) {
                        const uint32_t gs = masked % ST;
                        mbar_arrive(smem_u32(&bars->go[gs]));
                        ok = wait1(&bars->guard[gs], masked / ST);
                        if (!ok) break;
                        bad = bars->bad[gs][0] | bars->bad[gs][1];
                        ++masked;
                    }
                    const int s0 = si.dual ? 0 : (i & 1), s1 = si.dual ? 1 : s0;
                    for (int s = s0; s <= s1; ++s) {
                        if (t < lim[s]) {
                            ok = wait1(&bars->p_full[s], np[s]);
                            if (!ok) break;
                            ++np[s];
                            tc_fence_after();
                            if (!bad) {
                                const uint32_t va = sb + L::RING + (ev % ST) * L::TILE;
#pragma unroll
                                for (int kk = 0; kk < 8; ++kk)
                                    tc_mma_bf16_ts(tbase + 256 + s * DH, tbase + s * 128 + kk * 8,
                                                   smem_desc_sw128_mn(va + kk * 2048, kBox), idO,
                                                   (began[s] || kk) ? 1u : 0u);
                            }
                            began[s] = true;
                        }
                        if (s == s1) tc_commit(smem_u32(&bars->kv_empty[ev % ST]));
                        if (more && s == s0) {
                            ok = wait1(&bars->kv_full[ek % ST], ek / ST);
                            if (!ok) break;
                            tc_fence_after();
                        }
                        if (t < lim[s]) {
                            if (more && t + lead < lim[s]) mma_s(s, ek);
                            else tc_commit(smem_u32(&bars->o_full[s]));
                        }
                    }
                    if (ok && more) tc_commit(smem_u32(&bars->kv_empty[ek % ST]));
                }
                cnt += 2 * nt;
            }
            ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
        }
    } else {
        // ------------------------------------------------------------ guards
        // Values of partly masked tiles: rows that nobody sees become zeros, rows
        // that some see are searched for infinities and NaN.
        const int me = threadIdx.x - 64;                   // 0..63
        uint32_t cnt = 0, masked = 0;
        Seg g;
        bool ok = true;
        for (int it = 0; ok && next_seg(it, g); ++it) {
            const SegInfo si = seg_info(g, TT, tree);
            const int lead = si.dual ? 1 : 2, nt = g.t1 - g.t0;
            for (int i = max(0, si.kall / kCacheTile - g.t0); ok && i < nt; ++i) {
                const int t = g.t0 + i;
                if ((t + 1) * kCacheTile <= si.kall) continue;
                const uint32_t e = cnt + i + min(nt, i + lead);
                // A parity names a phase only to who has seen the one before: the ring's
                // phases are followed by the MMA warp, which says when e is there.
                ok = wait_warp(&bars->go[masked % ST], masked / ST) && wait_warp(&bars->kv_full[e % ST], e / ST);
                if (!ok) break;
                uint8_t* v = smem + L::RING + (e % ST) * L::TILE;
                const int lo = max(0, si.kall - t * kCacheTile), hi = max(0, min(kCacheTile, si.kmax - t * kCacheTile));
                for (int x = hi * 8 + me; x < kCacheTile * 8; x += 64)
#pragma unroll
                    for (int kb = 0; kb < L::KB; ++kb)
                        *reinterpret_cast<uint4*>(v + kb * kBox + x * 16) = make_uint4(0, 0, 0, 0);
                bool found = false;
                for (int x = lo * 8 + me; x < hi * 8; x += 64)
#pragma unroll
                    for (int kb = 0; kb < L::KB; ++kb) {
                        const uint4 u = *reinterpret_cast<const uint4*>(v + kb * kBox + x * 16);
                        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            found |= (w[k] & 0x7F80u) == 0x7F80u || (w[k] & 0x7F800000u) == 0x7F800000u;
                    }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                found = __any_sync(0xffffffffu, found);
                if (lane == 0) {
                    bars->bad[masked % ST][warp - 2] = found;
                    mbar_arrive(smem_u32(&bars->guard[masked % ST]));
                }
                ++masked;
            }
            cnt += 2 * nt;
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        // -------------------------------------------------- softmax and output
        const int slot = (warp - 4) >> 2;
        const int qw = warp & 3;                           // TMEM lane quarter
        const int r = qw * 32 + lane;
        const uint32_t loff = (uint32_t)(qw * 32) << 16;
        const uint32_t tS = tbase + loff + slot * 128, tO = tbase + loff + 256 + slot * DH;
        const int tok_in_tile = r / rep, head_in_tile = r - tok_in_tile * rep;
        const float sl2 = p.scale_log2;
        uint32_t ns = 0, no = 0, nx = 0, masked = 0, cnt = 0;
        Seg g;
        bool ok = true;
        for (int it = 0; ok && next_seg(it, g); ++it) {
            const SegInfo si = seg_info(g, TT, tree);
            const int nt = g.t1 - g.t0, lead = si.dual ? 1 : 2;
            const int tok0 = si.dual ? slot * TT : 0;
            const int ntok = min(TT, g.ntok - tok0);       // tokens of this slot's tile
            const bool mine = tok_in_tile < ntok;          // (rows past tile_tokens * rep have no token)
            const bool live = (qw * 32) / rep < ntok;      // some row of the warp has one
            const int lim = slot ? si.n1 : si.n0;
            const int step = si.dual ? 1 : 2, begin = g.t0 + (si.dual ? 0 : slot);
            const bool work = begin < lim;
            const int token = g.row + tok0 + min(tok_in_tile, ntok - 1);
            const int seen = g.first + tok0 + min(tok_in_tile, ntok - 1) + 1;   // causal
            const uint64_t word = (tree && live) ? p.tree[token] : 0;
            float m = -INFINITY, l = 0.f;
            int left = work ? (lim - begin + step - 1) / step : 0;   // tiles still to come
            if (left == 0) {
                // Not before this segment's queries are there: an idle slot must not
                // count for an earlier segment.
                ok = wait_warp(&bars->q_full, it);
                if (!ok) break;
                if (lane == 0) mbar_arrive(smem_u32(&bars->q_empty));
            }
            for (int t = g.t0; ok && t < g.t1; ++t) {
                const bool part = (t + 1) * kCacheTile > si.kall;
                const uint32_t mi = masked;
                if (part) ++masked;
                if ((!si.dual && ((t - g.t0) & 1) != slot) || t >= lim) continue;
                ok = wait_warp(&bars->s_full[slot], ns);
                if (!ok) break;
                ++ns;
                tc_fence_after();
                --left;
                if (left == 0 && si.dual && lane == 0) mbar_arrive(smem_u32(&bars->q_empty));
                uint32_t see[4] = {~0u, ~0u, ~0u, ~0u};
                if (live) {
                    uint32_t u[4][32];
#pragma unroll
                    for (int q = 0; q < 4; ++q) tmem_ld_32x32(tS + q * 32, u[q]);
                    tmem_ld_wait();
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int j = 0; j < 32; ++j) asm volatile("" : "+r"(u[q][j]));
                    if (part) {
                        // Keys of the tile that this row sees, one bit each.
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int k0 = t * kCacheTile + q * 32;
                            const int n = (tree ? g.base : seen) - k0;             // the first n keys
                            see[q] = n >= 32 ? ~0u : n > 0 ? (1u << n) - 1u : 0u;
                            if (tree) {
                                const int d = k0 - g.base;                         // draft of the word's bit 0
                                if (d >= 0) {
                                    if (d < 64) see[q] |= (uint32_t)(word >> d);
                                } else if (d > -32) {
                                    see[q] |= (uint32_t)(word << -d);
                                }
                                const int end = g.kv_len - k0;                     // bits past the drafts
                                see[q] &= end >= 32 ? ~0u : end > 0 ? (1u << end) - 1u : 0u;
                            }
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (!(see[q] >> j & 1u)) u[q][j] = 0xff800000u;    // -inf
                        }
                    }
                    float mx[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        mx[q] = __uint_as_float(u[q][0]);
#pragma unroll
                        for (int j = 1; j < 31; j += 2)
                            mx[q] = max3(mx[q], __uint_as_float(u[q][j]), __uint_as_float(u[q][j + 1]));
                        mx[q] = fmaxf(mx[q], __uint_as_float(u[q][31]));
                    }
                    const float top = fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
                    if (t == begin) {
                        m = top;
                    } else {
                        const bool grow = (top - m) * sl2 > 8.f;                   // also from m = -inf
                        if (__any_sync(0xffffffffu, grow)) {
                            const float f = grow ? ex2((m - top) * sl2) : 1.f;
                            l *= f;
                            if (grow) m = top;
#pragma unroll 1
                            for (int k = 0; k < DH; k += 16) {
                                uint32_t o[16];
                                tmem_ld_32x16(tO + k, o);
                                tmem_ld_wait();
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                                tmem_st_32x16(tO + k, o);
                            }
                        }
                    }
                    const float ms = m == -INFINITY ? 0.f : m * sl2;               // a row without keys so far: p = 0
                    float ls[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t w[16];
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float e0 = ex2(fmaf(__uint_as_float(u[q][j]), sl2, -ms));
                            const float e1 = ex2(fmaf(__uint_as_float(u[q][j + 1]), sl2, -ms));
                            ls[q] += e0;
                            ls[q] += e1;
                            w[j >> 1] = pack_bf16x2(e0, e1);
                        }
                        tmem_st_32x16(tS + q * 16, w);
                    }
                    l += (ls[0] + ls[1]) + (ls[2] + ls[3]);
                    tmem_st_wait();
                }
                if (part) {
                    ok = wait_warp(&bars->guard[mi % ST], mi / ST);
                    if (!ok) break;
                    if (live && (bars->bad[mi % ST][0] | bars->bad[mi % ST][1])) {
                        // O += P V by this warp, seen keys only.
                        const int i = t - g.t0;
                        const uint32_t e = cnt + i + min(nt, i + lead);
                        ok = wait_warp(&bars->kv_full[e % ST], e / ST);
                        if (!ok) break;
                        const uint8_t* v = smem + L::RING + (e % ST) * L::TILE;
                        const int keys = min(kCacheTile, si.kmax - t * kCacheTile);
#pragma unroll 1
                        for (int k = 0; k < DH; k += 32) {
                            uint32_t o[32];
                            tmem_ld_32x32(tO + k, o);
                            tmem_ld_wait();
                            float acc[32];
#pragma unroll
                            for (int j = 0; j < 32; ++j) acc[j] = t == begin ? 0.f : __uint_as_float(o[j]);
#pragma unroll 1
                            for (int key = 0; key < keys; ++key) {
                                __syncwarp();
                                uint32_t pw;
                                tmem_ld_32x1(tS + (key >> 1), pw);
                                tmem_ld_wait();
                                const float pk = (key & 1) ? bf16_hi(pw) : bf16_lo(pw);
                                const uint32_t sq = key < 64 ? (key < 32 ? see[0] : see[1]) : (key < 96 ? see[2] : see[3]);
                                const bool sees = sq >> (key & 31) & 1u;
                                const uint8_t* vr = v + (k >> 6) * kBox + key * 128;
#pragma unroll
                                for (int ch = 0; ch < 4; ++ch) {
                                    const int c16 = ((k & 63) >> 3) + ch;
                                    const uint4 x = *reinterpret_cast<const uint4*>(vr + ((c16 ^ (key & 7)) << 4));
                                    const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                                    for (int y = 0; y < 4; ++y) {
                                        const int j = ch * 8 + 2 * y;
                                        acc[j] = sees ? fmaf(pk, bf16_lo(xw[y]), acc[j]) : acc[j];
                                        acc[j + 1] = sees ? fmaf(pk, bf16_hi(xw[y]), acc[j + 1]) : acc[j + 1];
                                    }
                                }
                            }
                            __syncwarp();
#pragma unroll
                            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(acc[j]);
                            tmem_st_32x32(tO + k, o);
                        }
                        tmem_st_wait();
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->p_full[slot]));
            }
            if (!ok) break;
            cnt += 2 * nt;
            // ---- the segment's result
            if (work) {
                ok = wait_warp(&bars->o_full[slot], no);
                if (!ok) break;
                ++no;
                tc_fence_after();
            }
            const bool joins = !si.dual && g.t0 + 1 < si.n1;   // both slots hold parts of the same rows
            if (!si.dual && slot == 1) {
                // All products of the segment are done: the query tiles' space takes this slot's O.
                if (joins) {
                    if (live) {
#pragma unroll 1
                        for (int k = 0; k < DH; k += 32) {
                            uint32_t o[32];
                            tmem_ld_32x32(tO + k, o);
                            tmem_ld_wait();
                            if (mine) {
                                uint8_t* dst = smem + L::Q + r * DH * 4;
#pragma unroll
                                for (int j = 0; j < 8; ++j)
                                    *reinterpret_cast<uint4*>(dst + ((((k >> 2) + j) ^ (r & (DH / 4 - 1))) << 4)) =
                                        make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                            }
                            __syncwarp();
                        }
                        bars->xml[r] = make_float2(m, l);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(smem_u32(&bars->x_full[qw]));
                        mbar_arrive(smem_u32(&bars->q_empty));
                    }
                }
                tc_fence_before();
                continue;
            }
            float fo = 1.f, fx = 0.f;
            if (joins) {
                ok = wait_warp(&bars->x_full[qw], nx);
                if (!ok) break;
                ++nx;
                if (live) {
                    const float2 x = bars->xml[r];
                    const float top = fmaxf(m, x.x), ms = top == -INFINITY ? 0.f : top;
                    fo = ex2((m - ms) * sl2);
                    fx = ex2((x.x - ms) * sl2);
                    l = l * fo + x.y * fx;
                    m = top;
                }
            }
            if (live) {
                float* po = nullptr;
                __nv_bfloat16* out = nullptr;
                if (g.part >= 0) {
                    const size_t row = (size_t)g.part * 256 + (si.dual ? slot * 128 : 0) + r;
                    po = c.part_o + row * DH;
                    if (mine) c.part_ml[row] = make_float2(work ? m : -INFINITY, l);
                } else {
                    out = p.out + (size_t)token * p.ld_out + (size_t)(g.head * rep + head_in_tile) * DH;
                }
                const float il = g.part >= 0 ? 1.f : l == 0.f ? 0.f : 1.f / l;
                fo *= il;
                fx *= il;
#pragma unroll 1
                for (int k = 0; k < DH; k += 32) {
                    uint32_t o[32];
                    if (work) {
                        tmem_ld_32x32(tO + k, o);
                        tmem_ld_wait();
                    }
                    if (mine) {
                        float f[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) f[j] = work && l != 0.f ? __uint_as_float(o[j]) * fo : 0.f;
                        if (joins) {
                            const uint8_t* src = smem + L::Q + r * DH * 4;
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const float4 x = *reinterpret_cast<const float4*>(
                                    src + ((((k >> 2) + j) ^ (r & (DH / 4 - 1))) << 4));
                                if (fx != 0.f) {
                                    f[4 * j] = fmaf(x.x, fx, f[4 * j]);
                                    f[4 * j + 1] = fmaf(x.y, fx, f[4 * j + 1]);
                                    f[4 * j + 2] = fmaf(x.z, fx, f[4 * j + 2]);
                                    f[4 * j + 3] = fmaf(x.w, fx, f[4 * j + 3]);
                                }
                            }
                        }
                        if (po) {
#pragma unroll
                            for (int j = 0; j < 32; j += 4)
                                *reinterpret_cast<float4*>(po + k + j) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; j += 8)
                                *reinterpret_cast<uint4*>(out + k + j) =
                                    make_uint4(pack_bf16x2(f[j], f[j + 1]), pack_bf16x2(f[j + 2], f[j + 3]),
                                               pack_bf16x2(f[j + 4], f[j + 5]), pack_bf16x2(f[j + 6], f[j + 7]));
                        }
                    }
                    __syncwarp();
                }
            }
            if (!si.dual && work) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars->q_empty));
            }
            tc_fence_before();
        }
    }
    __syncthreads();
    if (warp == 0) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tbase, kTmemCols);
    }
}

// Joins the parts of cut items.  Block (b, y) takes rows [16 y, 16 y + 16) of the
// item that CTA b of the attention began and did not finish; a warp takes a row:
// its lanes read the parts' maxima and sums, then D / 32 columns each of the parts'
// sums, added in the order of the keys.
template <int DH>
__global__ void __launch_bounds__(128) cache_join_kernel(const __grid_constant__ CacheDev c,
                                                         const __grid_constant__ AttendParams p) {
    pdl_wait();
    pdl_trigger();
    const CachePlan pl = *c.plan;
    const int b = blockIdx.x, TT = c.tile_tokens;
    if (!pl.ok || b + 1 >= pl.n_ctas) return;
    const long long x = share_begin(pl, b + 1);            // the cut
    const CacheGroup g = c.groups[c.cta_group[b + 1]];
    const long long cost = c.groups[c.cta_group[b + 1] + 1].pre - g.pre, within = x - g.pre * c.Hkv;
    const int head = (int)(within / cost);
    const long long start = g.pre * c.Hkv + head * cost;
    if (x == start || start < share_begin(pl, b)) return;  // cut between items; begun by an earlier CTA
    const int a = cache_tile_cost(g.ntok, TT), n = (int)(cost / a) - 1;
    int t0, t1;
    stretch_tiles(0, x - start, cost, a, n, &t0, &t1);
    if (t1 == n) return;                                   // only the item's end is on the other side
    // CTAs b + 1 .. last hold the other parts.
    int last = b + 1;
    while (last + 1 < pl.n_ctas && share_begin(pl, last + 1) < start + cost) ++last;
    const int rows_tile = TT * c.rep;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rows = g.ntok > TT ? 128 + (g.ntok - TT) * c.rep : g.ntok * c.rep;
    constexpr int V = DH / 32;
    for (int r = blockIdx.y * 16 + warp; r < min(rows, blockIdx.y * 16 + 16); r += 4) {
        const int tile = r >> 7, in = r & 127;
        if (in >= rows_tile) continue;
        const int token = g.row + tile * TT + in / c.rep, h = head * c.rep + in % c.rep;
        // Part k of the item is in buffer part(k), or none when its stretch holds no tile.
        auto part = [&](int k) {
            if (k == 0) return 2 * b + 1;
            int u0, u1;
            stretch_tiles(share_begin(pl, b + k) - start, min(cost, share_begin(pl, b + k + 1) - start), cost, a, n, &u0,
                          &u1);
            return u0 < u1 ? 2 * (b + k) : -1;
        };
        const int parts = last - b + 1;
        float top = -INFINITY;
        for (int k = lane; k < parts; k += 32) {
            const int s = part(k);
            if (s >= 0) top = fmaxf(top, c.part_ml[(size_t)s * 256 + r].x);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float ms = top == -INFINITY ? 0.f : top;
        float l = 0.f, acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.f;
        for (int k0 = 0; k0 < parts; k0 += 32) {
            const int k = k0 + lane, s = k < parts ? part(k) : -1;
            float f = 0.f, lk = 0.f;
            if (s >= 0) {
                const float2 ml = c.part_ml[(size_t)s * 256 + r];
                f = ex2((ml.x - ms) * p.scale_log2);
                lk = ml.y * f;
            }
            const int cnt = min(32, parts - k0);
            for (int i = 0; i < cnt; ++i) {
                const int si = __shfl_sync(0xffffffffu, s, i);
                const float fi = __shfl_sync(0xffffffffu, f, i);
                l += __shfl_sync(0xffffffffu, lk, i);
                if (si < 0 || fi == 0.f) continue;
                const float* src = c.part_o + ((size_t)si * 256 + r) * DH + lane * V;
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] = fmaf(src[j], fi, acc[j]);
            }
        }
        const float il = l == 0.f ? 0.f : 1.f / l;
        __nv_bfloat16* out = p.out + (size_t)token * p.ld_out + (size_t)h * DH + lane * V;
#pragma unroll
        for (int j = 0; j < V; j += 2)
            *reinterpret_cast<uint32_t*>(out + j) = pack_bf16x2(acc[j] * il, acc[j + 1] * il);
    }
}

static_assert(smem_bytes<128>() <= 227 * 1024 && smem_bytes<64>() <= 227 * 1024, "shared memory of a block");

template <int DH>
cudaError_t attend(const CacheDev& c, const CUtensorMap& tm_q, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                   const AttendParams& p, int max_rows, cudaStream_t st) {
    static PerDevice attr;
    cudaError_t e = (cudaError_t)attr.get([] {
        return (int)cudaFuncSetAttribute(cache_attention_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         (int)smem_bytes<DH>());
    }, true);
    if (e != cudaSuccess) return e;
    // The kernel moves registers between its warpgroups: what they ask for (80 x 128 +
    // 208 x 256) must be within what the block is launched with, or they would wait.
    static PerDevice regs;
    const int nreg = regs.get([] {
        cudaFuncAttributes fa = {};
        return cudaFuncGetAttributes(&fa, cache_attention_kernel<DH>) == cudaSuccess ? fa.numRegs : 0;
    });
    if (nreg * kThreads < 80 * 128 + 208 * 256) return cudaErrorInvalidConfiguration;
    e = launch_pdl(cache_attention_kernel<DH>, dim3(c.num_sms), dim3(kThreads), smem_bytes<DH>(), st, tm_q, tm_k, tm_v,
                   c, p);
    if (e != cudaSuccess) return e;
    return launch_pdl(cache_join_kernel<DH>, dim3(c.num_sms, (max_rows + 15) / 16), dim3(128), 0, st, c, p);
}

}  // namespace

cudaError_t launch_cache_attend(const CacheDev& c, const CUtensorMap& tm_q, const CUtensorMap& tm_k,
                                const CUtensorMap& tm_v, const AttendParams& p, int max_rows, cudaStream_t st) {
    return c.dh == 64 ? attend<64>(c, tm_q, tm_k, tm_v, p, max_rows, st)
                      : attend<128>(c, tm_q, tm_k, tm_v, p, max_rows, st);
}

}  // namespace tmoe
