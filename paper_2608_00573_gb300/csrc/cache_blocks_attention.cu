// Attention of each new token over pages that it is told to read (a list per key/value
// head) and over the positions from its step's first page on.
//
// An item is a token, a key/value head and up to 16 of the query heads that share it.
// No two items have a list in common, so that a tile of the tensor cores has the item's 1
// to 16 rows alone and the operator is bound by what the lists bring in: HBM for single tokens
// (each listed K and V row once), L2 for chunks whose tokens list the same pages.  The
// products are therefore mma.sync with 16 rows, fed from shared memory; a 128-row tile of
// TMEM would hold the same rows.
//
// A stage is 64 listed positions: pages, or halves of pages of 128, as boxes of the cache's
// tensor maps, with their values.  One warp finds the pages and starts the copies; four
// warps take 16 positions of every stage each, with sums of their own:
//
//   S = Q K^T (16 x 16);  m' = max(m, max s);  p = 2^(scale' s - m');  l += sum p;  O = O 2^(m - m') + P V
//
// (m moves only when a score is more than 2^8 above it; P is rounded to bf16, the
// type of the product's operand, l sums p before that rounding; the first key's p is 1.)
// An item's stages are cut among the CTAs of a cluster, whose sums meet in distributed
// shared memory: first the four warps', then the CTAs', always in the same order.
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

template <int DH>
struct Stage {
    static constexpr int KB = DH / 64;
    static constexpr int SLAB = kStageKeys * 128;      // 64 rows of 64 columns
    static constexpr int TILE = KB * SLAB;             // K or V
    static constexpr int BYTES = 2 * TILE;
    static constexpr int COUNT = 96 * 1024 / BYTES;    // two CTAs to an SM
};

struct __align__(8) Bars {
    uint64_t full[8], empty[8];
    int first[8][4];           // of the stage's pages: first position, kHidden or kWhole
    float2 ml[kReaders][16];   // the warps' maxima and sums
    float2 mine[16];           // the CTA's
    PartList parts[2];         // OWN: the common item's parts, the sequence's own ones
    int abort_flag, never;
};

// What an item's item is about.
struct Item {
    int t, head, row0, rows;   // token, key/value head, query heads of it
    int seq, base, kv_len, pos;
    int listed, first_own;     // entries of the list that count, first page of the step's own
    int subs;                  // boxes of a page's rows (pages of 128: two)
    int stages;
};

// OWN: no lists; the token's sequence from its group's common tiles on, and then the common tiles'
// parts, which the attention kernel before this one has written.  Nothing but these is
// read behind that kernel's end: whatever comes before it has ended when it lets this one start.
template <int DH, bool OWN>
__global__ void __launch_bounds__(kThreads)
cache_blocks_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                    const __grid_constant__ CacheDev c, const __grid_constant__ BlocksParams p) {
    const int splits = p.splits;
    using S = Stage<DH>;
    constexpr int ST = S::COUNT;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sb = smem_u32(smem);
    Bars* bars = reinterpret_cast<Bars*>(smem + ST * S::BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % splits, index = blockIdx.x / splits;
    if (threadIdx.x == 0) {
        for (int s = 0; s < ST; ++s) {
            mbar_init(smem_u32(&bars->full[s]), 1);
            mbar_init(smem_u32(&bars->empty[s]), kReaders);
        }
        bars->abort_flag = bars->never = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
    }
    __syncthreads();
    if (!OWN) {
        pdl_wait();
        pdl_trigger();
    }
    const CachePlan pl = *c.plan;
    if (!pl.ok) return;                                // (all CTAs)
    if (sb & 1023u) {                                  // swizzled tiles start at multiples of 1024
        if (threadIdx.x == 0) atomicCAS(c.err, 0, ERR_TIMEOUT_CACHE_ATTN);
        return;
    }
    const uint32_t abort_at = smem_u32(&bars->abort_flag);
    auto wait = [&](uint64_t* b, uint32_t parity) {
        return __any_sync(0xffffffffu, wait_probes(smem_u32(b), parity & 1u, abort_at, c.err)) != 0;
    };

    Item it;
    {
        const int per = c.Hkv * p.row_tiles;
        it.t = index / per;
        it.head = index % per / p.row_tiles;
        it.row0 = index % p.row_tiles * 16;
        it.rows = min(16, c.rep - it.row0);
        const CacheToken s = c.tokens[it.t];
        it.seq = s.seq;
        it.kv_len = s.kv_len;
        it.base = s.base;
        it.pos = s.pos;
        int2 items = make_int2(-1, -1);
        if (OWN) {
            items = c.items_of[it.t];
            it.first_own = items.y < 0 ? 0 : c.groups[items.y].kv_len >> c.page_shift;
            it.listed = 0;
            if (threadIdx.x < 2) bars->parts[threadIdx.x] = part_list(c, pl, threadIdx.x ? items.x : items.y, it.head, it.t);
        } else {
            it.first_own = it.base >> c.page_shift;
            it.listed = min(p.n, it.first_own);
        }
        const int last = p.tree ? it.kv_len - 1 : it.pos;
        it.subs = c.page > kStageKeys ? c.page / kStageKeys : 1;
        const int boxes = (it.listed + (last >> c.page_shift) - it.first_own + 1) * it.subs;
        const int per_stage = max(1, kStageKeys >> c.page_shift);
        it.stages = OWN && !pl.own_apart ? 0 : (boxes + per_stage - 1) / per_stage;
    }
    const int per_stage = max(1, kStageKeys >> c.page_shift), box_rows = kStageKeys / per_stage;
    const int g0 = (int)((long long)it.stages * rank / splits), g1 = (int)((long long)it.stages * (rank + 1) / splits);

    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};   // rows lane / 4 and lane / 4 + 8
    float o[DH / 8][4];
#pragma unroll
    for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

    if (warp == kReaders) {
        // ------------------------------------------------------------------ loads
        // Lane i looks up box i of 32, the next 32 while these are copied.
        const int* list = p.blocks + ((size_t)it.t * c.Hkv + it.head) * p.n;
        const int* row = c.table + (size_t)it.seq * c.max_pages;
        const int boxes_end = g1 * per_stage;
        struct Box {
            int id, first;                             // page, first position (kWhole, kHidden)
        };
        auto look_up = [&](int b) {
            Box x{0, kHidden};
            const int j = b / it.subs, sub = b - j * it.subs;
            if (b >= boxes_end) return x;
            int col;
            bool fits = true;
            if (j < it.listed) {
                col = list[j];
                if (col == -1) {
                    fits = false;
                } else {
                    const int before = j ? list[j - 1] : -1;
                    fits = col >= 0 && col < it.first_own && (j == 0 || (before >= 0 && col > before));
                    if (!fits) atomicCAS(c.err, 0, ERR_CACHE_BLOCKS);
                }
            } else {
                col = it.first_own + j - it.listed;
                if (col >= c.max_pages || (col << c.page_shift) >= it.kv_len) fits = false;
            }
            if (!fits) return x;
            x.id = row[col];
            if (x.id < 0 || x.id >= c.n_pages) {
                atomicCAS(c.err, 0, ERR_CACHE_STATE);
                return x;
            }
            x.first = j < it.listed ? kWhole : (col << c.page_shift) + sub * box_rows;
            return x;
        };
        int b0 = g0 * per_stage;
        Box now = look_up(b0 + lane), next = look_up(b0 + 32 + lane);
        bool ok = true;
        uint32_t issued = 0;
        for (int g = g0; ok && g < g1; ++g) {
            const int at = g * per_stage - b0;         // (per_stage divides 32)
            const int s = (int)(issued % ST);
            if (issued >= (uint32_t)ST) ok = !wait(&bars->empty[s], issued / ST - 1);
            if (!ok) break;
            const int i = lane / (2 * S::KB), kb = lane % S::KB, is_v = lane / S::KB & 1;
            const int id = __shfl_sync(0xffffffffu, now.id, (at + i) & 31), first = __shfl_sync(0xffffffffu, now.first, (at + i) & 31);
            const bool mine = i < per_stage, there = mine && first != kHidden;
            const uint32_t boxes = __popc(__ballot_sync(0xffffffffu, there));
            if (mine && kb == 0 && !is_v) bars->first[s][i] = first;
            __syncwarp();
            const uint32_t fb = smem_u32(&bars->full[s]);
            if (lane == 0) mbar_arrive_expect_tx(fb, boxes * box_rows * 128);
            __syncwarp();
            if (there) {
                const int sub = (g * per_stage + i) % it.subs;
                tma_load_2d(sb + s * S::BYTES + is_v * S::TILE + kb * S::SLAB + i * box_rows * 128, is_v ? &tm_v : &tm_k, kb * 64,
                            (int)((((size_t)id * c.Hkv + it.head) << c.page_shift) + sub * box_rows), fb);
            }
            __syncwarp();
            ++issued;
            if (at + per_stage == 32) {
                b0 += 32;
                now = next;
                next = look_up(b0 + 32 + lane);
            }
        }
        // The copies have landed before the CTA ends, also one that gave up.
        const uint32_t never = smem_u32(&bars->never), tail = min(issued, (uint32_t)ST);
        for (uint32_t k = issued - tail; k < issued; ++k) wait_probes(smem_u32(&bars->full[k % ST]), (k / ST) & 1, never, c.err);
    } else {
        // --------------------------------------------------------------- products
        const int r = lane >> 2, q2 = (lane & 3) * 2;
        uint32_t qa[DH / 16][4];
        {
            const __nv_bfloat16* q = p.q + (size_t)it.t * p.ld_q + (size_t)(it.head * c.rep + it.row0) * DH + q2;
            auto word = [&](int row, int col) {
                return row < it.rows ? __ldg(reinterpret_cast<const uint32_t*>(q + (size_t)row * DH + col)) : 0u;
            };
#pragma unroll
            for (int k = 0; k < DH / 16; ++k) {
                qa[k][0] = word(r, k * 16);
                qa[k][1] = word(r + 8, k * 16);
                qa[k][2] = word(r, k * 16 + 8);
                qa[k][3] = word(r + 8, k * 16 + 8);
            }
        }
        const uint64_t tree = p.tree ? __ldg(p.tree + it.t) : 0;
        const bool two = it.rows > 8;                  // the tile's lower half has rows
        const int k16 = warp * 16, box = k16 / box_rows;
        // ldmatrix rows: keys of K by halves of 8 columns, keys of V by halves of 8 keys.
        const int krow = k16 + (lane >> 4) * 8 + (lane & 7), kcol = (lane >> 3) & 1;
        const int vrow = k16 + ((lane >> 3) & 1) * 8 + (lane & 7), vcol = lane >> 4;
        bool ok = true;
        uint32_t at = 0;
        for (int g = g0; ok && g < g1; ++g, ++at) {
            const int s = (int)(at % ST);
            ok = !wait(&bars->full[s], at / ST);
            if (!ok) break;
            const int first = bars->first[s][box];
            uint32_t see = 0;                          // keys of the 16 that the token sees
            if (first == kWhole) {
                see = 0xffffu;
            } else if (first != kHidden) {
                const int key = first + (k16 & (box_rows - 1));
                const int all = p.tree ? it.base : it.pos + 1, n = all - key;
                see = n >= 16 ? 0xffffu : n > 0 ? (1u << n) - 1u : 0u;
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
            if (lane == 0) mbar_arrive(smem_u32(&bars->empty[s]));
        }
        // Sums of the row's four lanes.
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        }
    }
    __syncthreads();                                   // the stages are free: all copies have landed and been read
    // ------------------------------------------------------------------- joins
    float* parts = reinterpret_cast<float*>(smem);     // [kReaders][16][DH], then the CTA's [16][DH]
    float* own = parts + kReaders * 16 * DH;
    if (warp < kReaders) {
        const int r = lane >> 2, q2 = (lane & 3) * 2;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (r + 8 * i < it.rows) {
                if ((lane & 3) == 0) bars->ml[warp][r + 8 * i] = make_float2(m[i], l[i]);
                float* to = parts + (warp * 16 + r + 8 * i) * DH + q2;
#pragma unroll
                for (int k = 0; k < DH / 8; ++k) *reinterpret_cast<float2*>(to + k * 8) = make_float2(o[k][2 * i], o[k][2 * i + 1]);
            }
    }
    __syncthreads();
    auto rescale = [](float part, float top) { return part == -INFINITY ? 0.f : ex2(part - top); };   // (no key seen: no part)
    __nv_bfloat16* out = p.out + (size_t)it.t * p.ld_out + (size_t)(it.head * c.rep + it.row0) * DH;
    if (OWN) {
        pdl_wait();
        pdl_trigger();
    }
    // Two columns of a row: the other parts first, in the order of the keys, then what is here; its output.
    auto put_out = [&](int r, int col, float top, float sum, float a, float b) {
        if (OWN) {
            float t0 = -INFINITY, s0 = 0.f, a0 = 0.f, b0 = 0.f, fa, fb;
            const int n0 = bars->parts[0].count, n = n0 + bars->parts[1].count;
            constexpr int SIDE = 8;
            for (int k0 = 0; k0 < n; k0 += SIDE) {
                float2 ml[SIDE], v[SIDE];
#pragma unroll
                for (int i = 0; i < SIDE; ++i) {
                    const int k = min(k0 + i, n - 1);
                    const PartList& l = bars->parts[k >= n0];
                    const long long row = l.row + (long long)(k >= n0 ? k - n0 : k) * l.step + r;
                    ml[i] = __ldcg(c.part_ml + row);
                    v[i] = __ldcg(reinterpret_cast<const float2*>(l.at<DH>(c.part_o, row) + (col >> 2) * l.next4() + (col & 3)));
                }
#pragma unroll
                for (int i = 0; i < SIDE; ++i)
                    if (join_source(ml[i], k0 + i < n, t0, s0, fa, fb)) {
                        a0 = a0 * fa + v[i].x * fb;
                        b0 = b0 * fa + v[i].y * fb;
                    }
            }
            if (join_source(make_float2(top, sum), true, t0, s0, fa, fb)) {
                a0 = a0 * fa + a * fb;
                b0 = b0 * fa + b * fb;
            }
            sum = s0;
            a = a0;
            b = b0;
        }
        const float il = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint32_t*>(out + (size_t)r * DH + col) = pack_bf16x2(a * il, b * il);
    };
    for (int x = threadIdx.x; x < it.rows * (DH / 2); x += kThreads) {
        const int r = x / (DH / 2), col = x % (DH / 2) * 2;
        float top = -INFINITY, sum = 0.f, a = 0.f, b = 0.f;
#pragma unroll
        for (int w = 0; w < kReaders; ++w) top = fmaxf(top, bars->ml[w][r].x);
#pragma unroll
        for (int w = 0; w < kReaders; ++w) {
            const float2 ml = bars->ml[w][r], v = *reinterpret_cast<const float2*>(parts + (w * 16 + r) * DH + col);
            const float f = rescale(ml.x, top);
            sum = ml.x == -INFINITY ? sum : fmaf(ml.y, f, sum);
            a = ml.x == -INFINITY ? a : fmaf(v.x, f, a);
            b = ml.x == -INFINITY ? b : fmaf(v.y, f, b);
        }
        if (splits == 1) {
            put_out(r, col, top, sum, a, b);
        } else {
            *reinterpret_cast<float2*>(own + r * DH + col) = make_float2(a, b);
            if (col == 0) bars->mine[r] = make_float2(top, sum);
        }
    }
    if (splits == 1) return;
    cluster_sync();
    const uint32_t own_at = smem_u32(own), ml_at = smem_u32(bars->mine);
    auto peer = [](uint32_t at, uint32_t cta) {
        float2 v;
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(mapa_shared(at, cta)) : "memory");
        return v;
    };
    for (int x = rank * kThreads + threadIdx.x; x < it.rows * (DH / 2); x += splits * kThreads) {
        const int r = x / (DH / 2), col = x % (DH / 2) * 2;
        float top = -INFINITY, sum = 0.f, a = 0.f, b = 0.f;
        for (int w = 0; w < splits; ++w) top = fmaxf(top, peer(ml_at + r * 8, w).x);
        for (int w = 0; w < splits; ++w) {
            const float2 ml = peer(ml_at + r * 8, w), v = peer(own_at + (r * DH + col) * 4, w);
            const float f = rescale(ml.x, top);
            sum = ml.x == -INFINITY ? sum : fmaf(ml.y, f, sum);
            a = ml.x == -INFINITY ? a : fmaf(v.x, f, a);
            b = ml.x == -INFINITY ? b : fmaf(v.y, f, b);
        }
        put_out(r, col, top, sum, a, b);
    }
    cluster_sync();                                    // nobody ends while others read its sums
}

template <int DH, bool OWN>
cudaError_t blocks_launch(const CacheDev& c, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const BlocksParams& p,
                          cudaStream_t st) {
    constexpr size_t smem = Stage<DH>::COUNT * Stage<DH>::BYTES + sizeof(Bars);
    static_assert((kReaders + 1) * 16 * DH * 4 <= Stage<DH>::COUNT * Stage<DH>::BYTES, "joins fit the stages");
    static_assert(Stage<DH>::COUNT <= 8, "barriers");
    static PerDevice attr;
    cudaError_t e = (cudaError_t)attr.get([] {
        return (int)cudaFuncSetAttribute(cache_blocks_kernel<DH, OWN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    }, true);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((long long)p.T * c.Hkv * p.row_tiles * p.splits));
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
