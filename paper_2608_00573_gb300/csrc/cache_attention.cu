// Attention over the paged cache: prompts, single tokens and drafted trees.
//
// A query tile is 128 rows: tile_tokens = 128 / rep consecutive new tokens of one
// sequence, each with the rep = q_heads / kv_heads query heads of one key/value
// head, so that a key tile read once serves all heads that share it.  For a tile and
// key tiles of 128 positions (a running softmax, in base 2):
//
//   S = Q K^T                       tcgen05.mma, M = 128, N = 128, K = D -> TMEM
//   m' = max(m, max_j s_j);  p_j = 2^(scale' (s_j - m'))   fp32, one row per thread
//   O = O 2^(scale' (m - m')) + P V  tcgen05.mma, A = P from TMEM (bf16), B = V from
//                                   shared memory with its D axis contiguous
//   l = l 2^(...) + sum_j p_j;      out = O / l
//
// The reference m need not be the maximum: O and l are rescaled only when a row's
// maximum is more than a factor 2^8 above m, so p stays below 2^8, which costs no
// precision in floating point, and the pass over O in TMEM is rare.  P is rounded to bf16,
// the type of the tensor cores' other operand; l sums p in fp32 before that rounding (sums
// of the rounded values cost 11 % of a long prompt).  m starts as the maximum of the first
// keys that the row sees, whose p then is 1 and rounds to itself: a row that sees one key
// gives its value exactly.  Over hundreds of keys the error against 64 bits is 0.0019 to
// 0.0024 of the result's size, 1.1 to 1.45 times that of the output's rounding alone
// (0.0016 to 0.0017, all that is left with P in 32 bits).
//
// A CTA holds two query tiles in flight ("slots", each with its own S and O in
// TMEM and its own group of four softmax warps), so that one slot's products run
// under the other's softmax.  In a group of more than tile_tokens tokens the
// slots are its two query tiles and share every key tile; in a smaller group
// (single tokens, short drafts) both slots hold the same tile and take the even and
// the odd key tiles, and their results are joined at the end, each slot reading the
// other's O in TMEM.  A thread has one row, so that maxima and sums need no exchange;
// P is handed over in two halves of 64 keys, the first half's product running under
// the second half's exponentials.  (Two threads to a row, sixteen softmax warps, spill
// and are slower: a 16384-token prompt took 2.27 ms against 1.56.)
//
// Work is split evenly whatever the lengths (cache_pages.cu makes the lists).  With many
// items each CTA draws whole items from a counter, the longest first.  Otherwise the
// items' costs are laid end to end and each CTA takes the same share of the line, cutting
// items at key tiles; a cut item's parts go to a buffer, at most two per CTA, and are
// added in the order of the keys, so results do not depend on timing.  With
// few rows the CTA that writes an item's last part joins it (join_row), else
// cache_join_kernel does (join_rows).
//
// Masked places never reach a result: scores are replaced, not added to; value
// rows that no row of the item sees are zeroed in shared memory (0 * NaN would
// be NaN), and a tile whose partly masked value rows hold an infinity or a NaN is
// multiplied by the softmax warps themselves, skipping masked keys.
//
// Bounds: prompts the tensor cores and, per key tile, the chain S -> exponentials -> P V
// of each slot; decoding HBM, each K and V row once per query tile.  Measured (32 query
// heads on 8, D = 128): a 16384-token prompt 1.46 to 1.53 ms (by the clock that the power
// cap leaves), 1.44 to 1.51 PFLOP/s, 0.75 to 0.78 of cuBLAS; 7 sequences of 30k to 65k
// positions, a token each, 199 us, 0.98 of the copy rate; one sequence of 1500 positions
// 11.7 to 14.2 us, launches and latencies.
#include <algorithm>
#include <cstddef>

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
    static constexpr int Q = 0;                          // two query tiles
    static constexpr int RING = 2 * TILE;
    static constexpr int BYTES = RING + STAGES * TILE;
};

// A CTA's piece of an item.
struct Seg {
    int valid;
    int seq, kv_len, row, ntok, first, base, head;
    int t0, t1;          // key tiles
    int part;            // part buffer, -1: the whole item
};

struct __align__(8) Bars {
    uint64_t kv_full[10], kv_empty[10];
    uint64_t go[10], guard[10];   // partly masked value tile is under way / has been guarded, in the order of such tiles
    uint64_t q_full, q_empty;
    uint64_t s_full[2], o_full[2];
    uint64_t p_half[2], p_full[2];   // P of a tile's first 64 keys, of all
    uint64_t half_done[2];           // O has the first 64 keys' part
    uint64_t x_full[2][4], x_done[2][4];   // a slot's maxima and sums are there, the other slot's O has been read
    uint64_t part_done, join_go;
    uint64_t seg_full[kSegSlots], seg_empty[kSegSlots];
    Seg seg[kSegSlots];
    int bad[10][2];      // guard warps' finding per ring stage
    float2 xml[2][128];  // each slot's maximum and sum per row
    uint32_t tmem_base;
    int last_part;       // this CTA wrote an item's last missing part
    int abort_flag, never;
};
constexpr int kSegReaders = 1 + 2 + 8;   // warps that read a segment

template <int DH>
constexpr size_t smem_bytes() {
    return (size_t)Layout<DH>::BYTES + sizeof(Bars);
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

// One lane of a converged warp.  Products and commits stand behind it: the compiler
// then knows that a single lane issues them and keeps their operands in uniform
// registers (behind lane == 0 each cost some thirty instructions, more than its 64
// cycles).
__device__ __forceinline__ bool elect_one() {
    uint32_t pred = 0;
    asm volatile("{\n\t.reg .b32 r;\n\t.reg .pred p;\n\telect.sync r|p, 0xffffffff;\n\t@p mov.s32 %0, 1;\n\t}"
                 : "+r"(pred));
    return pred != 0;
}

// Products with the descriptors' upper words as constants (the lower ones, address and
// leading offset, take no carry): less to issue per product than 64-bit sums, on the warp
// that all others wait for (16384-token prompt 1.50 -> 1.47 ms).
constexpr uint32_t kDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;   // of smem_desc_sw128 and smem_desc_sw128_mn
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "mov.b64 b, {%2, %5};\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHigh)
        : "memory");
}

// Waits for the TMEM loads in flight; x, one of their results, is not used before.
__device__ __forceinline__ void landed(uint32_t (&x)[32]) {
    tmem_ld_wait();
#pragma unroll
    for (int j = 0; j < 32; ++j) asm volatile("" : "+r"(x[j]));
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n\t.reg .b64 a, b, c, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// Seldom used, so a function of its own, out of the way of the code that runs for every
// tile.
//
// O += P V of keys [key0, key1) of a tile (of one half of it; see0, see1: those that the
// row sees) for this warp's rows.  v: the tile's value rows.
template <int DH>
__device__ __noinline__ void pv_by_hand(uint32_t tS, uint32_t tO, const uint8_t* v, int key0, int key1, uint32_t see0,
                                        uint32_t see1, bool first) {
#pragma unroll 1
    for (int k = 0; k < DH; k += 32) {
        uint32_t o[32];
        tmem_ld_32x32(tO + k, o);
        landed(o);
        float acc[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) acc[j] = first ? 0.f : __uint_as_float(o[j]);
#pragma unroll 1
        for (int key = key0; key < key1; ++key) {
            __syncwarp();
            uint32_t pw;
            tmem_ld_32x1(tS + (key >> 1), pw);
            tmem_ld_wait();
            const float pk = (key & 1) ? bf16_hi(pw) : bf16_lo(pw);
            const bool sees = ((key & 32) ? see1 : see0) >> (key & 31) & 1u;
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

// Parts that a second kernel joins hold 32 rows of 4 columns side by side, so that the
// threads of a warp, a row each, write whole lines (with a row's columns side by side a
// 777-token prompt took 18.0 us instead of 15.3, 24 drafted trees 96 instead of 91).  Those
// that the writing CTAs join have few rows: there a row's columns are side by side, and a
// warp reads a row at once (one sequence's token 11.9 us instead of 12.5).
template <int DH>
__device__ __forceinline__ size_t part_at(size_t buf, int row, int col) {
    return (buf * 256 + (row & ~31)) * DH + (size_t)(col >> 2) * 128 + (row & 31) * 4 + (col & 3);
}

// One more source of a row: its maximum and sum (x), added to top and l; fa and fb are the
// factors of what was summed before and of the source.  False: nothing was summed in it.
__device__ __forceinline__ bool join_source(float2 x, bool there, float& top, float& l, float& fa, float& fb) {
    there = there && x.x != -INFINITY;
    const float m = there ? fmaxf(top, x.x) : top, ref = m == -INFINITY ? 0.f : m;
    fa = ex2(top - ref);
    fb = ex2(x.x - ref);
    top = m;
    l = there ? l * fa + x.y * fb : l;
    return there;
}

// Joins row r of a cut item of one query tile from the parts of CTAs first .. last, in the
// order of the keys; a lane takes D / 32 columns, eight sources are read at a time.  CTA
// `first` wrote its part into its second buffer, the others into their first; each has two
// sources, from the two slots.  Bound: latency, one or two rounds of reads.
template <int DH>
__device__ __forceinline__ void join_row(const CacheDev& c, const AttendParams& p, const Seg& g, int first, int last,
                                         int r, int lane) {
    constexpr int V = DH / 32, B = 8;
    const int sources = (last - first + 1) * 2;
    float top = -INFINITY, l = 0.f, acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
#pragma unroll 1
    for (int s0 = 0; s0 < sources; s0 += B) {
        float2 ml[B];
        float o[B][V];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int s = min(s0 + i, sources - 1), k = s >> 1;
            const size_t row = (size_t)(k == 0 ? 2 * first + 1 : 2 * (first + k)) * 256 + (s & 1) * 128 + r;
            const float* src = c.part_o + row * DH + lane * V;
            ml[i] = __ldcg(c.part_ml + row);
#pragma unroll
            for (int j = 0; j < V; j += 2) {
                const float2 x = __ldcg(reinterpret_cast<const float2*>(src + j));
                o[i][j] = x.x;
                o[i][j + 1] = x.y;
            }
        }
#pragma unroll
        for (int i = 0; i < B; ++i) {
            float fa, fb;
            const bool there = join_source(ml[i], s0 + i < sources, top, l, fa, fb);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = there ? acc[j] * fa + o[i][j] * fb : acc[j];
        }
    }
    const int rep = c.rep;
    const float il = l == 0.f ? 0.f : 1.f / l;
    __nv_bfloat16* out = p.out + (size_t)(g.row + r / rep) * p.ld_out + (size_t)(g.head * rep + r % rep) * DH + lane * V;
#pragma unroll
    for (int j = 0; j < V; j += 2)
        *reinterpret_cast<uint32_t*>(out + j) = pack_bf16x2(acc[j] * il, acc[j + 1] * il);
}

// Joins 8 rows of a cut item, G times 16 columns of them, likewise; a lane has a row and 4
// columns of each 16, two sources are read at a time (each part is one: the slots have
// joined theirs, or have rows of their own).  Bound: L2.
template <int DH, int G>
__device__ __forceinline__ void join_rows(const CacheDev& c, const AttendParams& p, const CacheShare& sh, int rows,
                                          int r0, int k0, int lane) {
    constexpr int B = 2;
    const int sources = sh.last - sh.first + 1;
    const int r = r0 + (lane & 7), row = min(r, rows - 1), col = k0 + (lane >> 3) * 4;
    float top = -INFINITY, l = 0.f, acc[G][4];
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[g][j] = 0.f;
#pragma unroll 1
    for (int s0 = 0; s0 < sources; s0 += B) {
        float2 ml[B];
        float4 o[B][G];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int s = min(s0 + i, sources - 1);
            const size_t buf = s == 0 ? 2 * sh.first + 1 : 2 * (sh.first + s);
            ml[i] = __ldcg(c.part_ml + buf * 256 + row);
#pragma unroll
            for (int g = 0; g < G; ++g)
                o[i][g] = __ldcg(reinterpret_cast<const float4*>(c.part_o + part_at<DH>(buf, row, col + 16 * g)));
        }
#pragma unroll
        for (int i = 0; i < B; ++i) {
            float fa, fb;
            const bool there = join_source(ml[i], s0 + i < sources, top, l, fa, fb);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float x[4] = {o[i][g].x, o[i][g].y, o[i][g].z, o[i][g].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[g][j] = there ? acc[g][j] * fa + x[j] * fb : acc[g][j];
            }
        }
    }
    const int tile = r >> 7, in = r & 127;
    if (r >= rows || in >= c.tile_tokens * c.rep) return;
    const int token = sh.g.row + tile * c.tile_tokens + in / c.rep, h = sh.head * c.rep + in % c.rep;
    const float il = l == 0.f ? 0.f : 1.f / l;
    __nv_bfloat16* out = p.out + (size_t)token * p.ld_out + (size_t)h * DH + col;
#pragma unroll
    for (int g = 0; g < G; ++g)
        *reinterpret_cast<uint2*>(out + 16 * g) = make_uint2(pack_bf16x2(acc[g][0] * il, acc[g][1] * il),
                                                             pack_bf16x2(acc[g][2] * il, acc[g][3] * il));
}

template <int DH>
__global__ void __launch_bounds__(kThreads, 1)
cache_attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                       const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CacheDev c,
                       const __grid_constant__ AttendParams p) {
    using L = Layout<DH>;
    constexpr int ST = L::STAGES;
    extern __shared__ __align__(1024) uint8_t smem[];    // swizzled tiles start at multiples of 1024
    const uint32_t sb = smem_u32(smem);
    if (sb & 1023u) {
        if (threadIdx.x == 0) atomicCAS(c.err, 0, ERR_TIMEOUT_CACHE_ATTN);
        return;
    }
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
        mbar_init(smem_u32(&bars->q_empty), 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&bars->s_full[s]), 1);
            mbar_init(smem_u32(&bars->p_half[s]), 4);
            mbar_init(smem_u32(&bars->p_full[s]), 4);
            mbar_init(smem_u32(&bars->half_done[s]), 1);
            mbar_init(smem_u32(&bars->o_full[s]), 1);
        }
        for (int s = 0; s < 8; ++s) {
            mbar_init(smem_u32(&bars->x_full[s >> 2][s & 3]), 1);
            mbar_init(smem_u32(&bars->x_done[s >> 2][s & 3]), 1);
        }
        mbar_init(smem_u32(&bars->part_done), 8);
        mbar_init(smem_u32(&bars->join_go), 1);
        for (int s = 0; s < kSegSlots; ++s) {
            mbar_init(smem_u32(&bars->seg_full[s]), 1);
            mbar_init(smem_u32(&bars->seg_empty[s]), kSegReaders);
        }
        bars->abort_flag = bars->never = 0;
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
    pdl_wait();
    pdl_trigger();

    // (Addresses of single barriers are constants beside one base register.)
    const uint32_t bb = sb + L::BYTES;
    auto bar = [&](const uint64_t* b) {
        return bb + (uint32_t)(reinterpret_cast<const uint8_t*>(b) - reinterpret_cast<const uint8_t*>(bars));
    };
    const uint32_t abort_at = bb + (uint32_t)offsetof(Bars, abort_flag);
    auto wait = [&](const uint64_t* b, uint32_t parity) { return wait_probes(bar(b), parity & 1u, abort_at, c.err); };
    auto lost = [](uint32_t gave_up) { return __any_sync(0xffffffffu, gave_up) != 0; };
    // The it-th segment of this CTA (false: none left, or aborted).
    auto next_seg = [&](int it, Seg& g) {
        const int s = it % kSegSlots;
        if (lost(wait(&bars->seg_full[s], it / kSegSlots))) return false;
        g = bars->seg[s];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(&bars->seg_empty[s]));
        return __shfl_sync(0xffffffffu, g.valid, 0) != 0;
    };

    // Registers go from the first four warps to the softmax warps (104 x 128 + 200 x 256 of the
    // 168 x 384 at launch).  The two branches do not meet before the roles end: where
    // they met, the compiler would take the smaller number for all that follows.
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (warp == 0) {
            // ------------------------------------------------ segments and loads
            const int b = blockIdx.x;
            const CachePlan pl = *c.plan;
            const CacheShare sh = c.shares[b];      // (read with the plan, not after it)
            int it = 0, nseg = 0;
            uint32_t cnt = 0, masked = 0;           // ring entries issued, partly masked value tiles among them
            bool ok = true;
            auto give_seg = [&](const Seg& g) {
                const int s = it % kSegSlots;
                if (it >= kSegSlots && lost(wait(&bars->seg_empty[s], it / kSegSlots - 1))) return false;
                if (lane == 0) {
                    bars->seg[s] = g;
                    mbar_arrive(bar(&bars->seg_full[s]));
                }
                ++it;
                return true;
            };
            const int pages_per_tile = kCacheTile >> c.page_shift;
            const int my_page = lane / L::KB, my_kb = lane % L::KB;
            const bool my_box = lane < pages_per_tile * L::KB;
            // Whole items are drawn from a counter, longest first; else the CTA's share of the
            // line is walked item by item.
            const bool whole = pl.n_ctas == 0;
            const int items = whole ? pl.n_groups * c.Hkv : 0;
            int item = b, group = 0, head = 0;
            long long x = 0, x_end = 0, within = 0;
            CacheGroup g;
            bool any = pl.ok && (whole ? b < items : b < pl.n_ctas);
            if (any && !whole) {
                x = sh.begin;
                x_end = sh.end;
                within = sh.within;
                group = sh.group;
                head = sh.head;
                g = sh.g;
            }
            while (ok && any) {
                int drawn = 0;
                Seg sg;
                if (whole) {
                    if (lane == 0) drawn = atomicAdd(&c.plan->drawn, 1);
                    head = item % c.Hkv;
                    g = c.groups[item / c.Hkv];
                }
                const int two_tiles = cache_two_tiles(g.ntok, TT);
                sg.valid = 1;
                sg.seq = g.seq;
                sg.kv_len = g.kv_len;
                sg.row = g.row;
                sg.ntok = g.ntok;
                sg.first = g.first;
                sg.base = g.base;
                sg.head = head;
                if (whole) {
                    sg.t0 = 0;
                    sg.t1 = cache_item_tiles(g.cost, two_tiles);
                    sg.part = -1;
                } else {
                    const long long x1 = min((long long)g.cost, within + (x_end - x));
                    sg.t0 = cache_tiles_before(within, g.cost, two_tiles);
                    sg.t1 = cache_tiles_before(x1, g.cost, two_tiles);
                    const bool all = sg.t0 == 0 && sg.t1 == cache_item_tiles(g.cost, two_tiles);
                    sg.part = all ? -1 : 2 * b + (sg.t0 == 0);
                    x += x1 - within;
                    within = 0;
                    any = x < x_end;
                    if (any && ++head == c.Hkv) {
                        head = 0;
                        g = c.groups[++group];
                    }
                }
                if (sg.t0 < sg.t1) {
                    if (!give_seg(sg)) break;
                    const SegInfo si = seg_info(sg, TT, tree);
                    // Page indices of the tiles ahead travel in registers.
                    const int n_pages = (si.kmax + c.page - 1) >> c.page_shift;
                    const int* row = c.table + (size_t)sg.seq * c.max_pages;
                    auto page_of = [&](int t) {
                        const int j = t * pages_per_tile + my_page;
                        return (my_box && t < sg.t1 && j < n_pages) ? row[j] : -1;
                    };
                    auto load = [&](const CUtensorMap* tm, int t, int id) {
                        const int s = (int)(cnt % ST);
                        if (cnt >= (uint32_t)ST && lost(wait(&bars->kv_empty[s], cnt / ST - 1))) return false;
                        const int have = max(0, min(pages_per_tile, n_pages - t * pages_per_tile));
                        const uint32_t fb = bar(&bars->kv_full[s]);
                        if (lane == 0) mbar_arrive_expect_tx(fb, (uint32_t)have * c.page * 128 * L::KB);
                        __syncwarp();
                        if (my_box && my_page < have)
                            tma_load_2d(sb + L::RING + s * L::TILE + my_kb * kBox + my_page * c.page * 128, tm,
                                        my_kb * 64, (id * c.Hkv + sg.head) << c.page_shift, fb);
                        __syncwarp();
                        ++cnt;
                        return true;
                    };
                    int id0 = page_of(sg.t0), id1 = page_of(sg.t0 + 1), id2 = page_of(sg.t0 + 2);
                    const int lead = si.dual ? 1 : 2;
                    // K of the first `lead` tiles, the queries (once the previous segment's products
                    // have read theirs), then V of tile t and K of tile t + lead in turn.
#pragma unroll 1
                    for (int t = sg.t0 - lead; ok && t < sg.t1; ++t) {
                        const int tk = t + lead;
                        if (t >= sg.t0) {
                            ok = load(&tm_v, t, id0);
                            if ((t + 1) * kCacheTile > si.kall) {
                                if (lane == 0) mbar_arrive(bar(&bars->go[masked % ST]));
                                ++masked;
                            }
                        }
                        if (ok && tk < sg.t1) ok = load(&tm_k, tk, t < sg.t0 ? (tk == sg.t0 ? id0 : id1) : (lead == 1 ? id1 : id2));
                        if (ok && t == sg.t0 - 1) {
                            ok = nseg == 0 || !lost(wait(&bars->q_empty, nseg - 1));
                            if (ok && lane == 0) {
                                const uint32_t qb = bar(&bars->q_full);
                                const uint32_t bytes = (uint32_t)L::KB * TT * rep * 128;
                                mbar_arrive_expect_tx(qb, si.dual ? 2 * bytes : bytes);
                                for (int s = 0; s < (si.dual ? 2 : 1); ++s)
                                    for (int kb = 0; kb < L::KB; ++kb)
                                        tma_load_3d(sb + L::Q + s * L::TILE + kb * kBox, &tm_q, kb * 64, sg.head * rep,
                                                    sg.row + s * TT, qb);
                            }
                            __syncwarp();
                            nseg += ok;
                        }
                        if (t >= sg.t0) {
                            id0 = id1;
                            id1 = id2;
                            id2 = page_of(t + 3);
                        }
                    }
                }
                if (whole) {
                    item = (int)gridDim.x + __shfl_sync(0xffffffffu, drawn, 0);
                    any = item < items;
                }
            }
            if (lane == 0 && pl.ok && whole) {
                // The last CTA to finish drawing leaves the counter at zero for the next call.
                __threadfence();
                if (atomicAdd(&c.plan->done, 1) == (int)gridDim.x - 1) {
                    c.plan->drawn = 0;
                    c.plan->done = 0;
                }
            }
            if (ok) {
                Seg end = {};
                give_seg(end);
            }
            // The last copies have landed, and been read unless the CTA gave up, before
            // it ends.
            const uint32_t tail = min(cnt, (uint32_t)ST);
            const uint32_t never = bb + (uint32_t)offsetof(Bars, never);
            for (uint32_t k = cnt - tail; k < cnt; ++k) wait_probes(bar(&bars->kv_full[k % ST]), (k / ST) & 1, never, c.err);
            if (nseg > 0) wait_probes(bar(&bars->q_full), (nseg - 1) & 1, never, c.err);
            for (uint32_t k = cnt - tail; k < cnt; ++k) wait(&bars->kv_empty[k % ST], k / ST);
        } else if (warp == 1) {
            // -------------------------------------------------------------- MMAs
            // The ring's entries come in the order in which they are used: K of the first
            // `lead` tiles, then V of tile i and K of tile i + lead in turn.
            constexpr uint32_t idS = idesc_bf16_f32(128, 128);
            constexpr uint32_t idO = idesc_bf16_f32(128, DH) | kIdescBMn;
            const uint32_t tm = __shfl_sync(0xffffffffu, tbase, 0);
            const uint32_t d_q = (uint32_t)smem_desc_sw128(sb + L::Q), d_k = (uint32_t)smem_desc_sw128(sb + L::RING);
            const uint32_t d_v = (uint32_t)smem_desc_sw128_mn(sb + L::RING, kBox);
            constexpr uint32_t kTile16 = L::TILE >> 4;       // a tile in a descriptor's units
            uint32_t stage = 0, phase = 0, masked = 0, p_phase = 0, gave_up = 0;   // p_phase: one bit per slot
            auto entry = [&]() {                             // next ring entry, once it has landed
                const uint32_t e = stage;
                gave_up |= wait(&bars->kv_full[e], phase);
                if (++stage == (uint32_t)ST) {
                    stage = 0;
                    phase ^= 1u;
                }
                return e;
            };
            Seg g;
            for (int it = 0; !lost(gave_up) && next_seg(it, g); ++it) {
                const SegInfo si = seg_info(g, TT, tree);
                auto uniform = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
                const int dual = uniform(si.dual), lead = dual ? 1 : 2, nt = uniform(g.t1 - g.t0);
                const int n0 = uniform(si.n0 - g.t0), n1 = uniform(si.n1 - g.t0);   // the slots' tiles, from the segment's first
                const int first_masked = uniform(si.kall / kCacheTile - g.t0);
                gave_up |= wait(&bars->q_full, it);
                // Step i: O += P V of tile i, S = Q K^T of tile i + lead, slot by slot, so that
                // a slot's products run under the other slot's softmax.  (Given up: the waits
                // return at once, the products' results are not used.)
                uint32_t ev = 0, ek = 0;
                auto pv = [&](int s, int half, bool began) {             // keys 64 half .. 64 half + 63
                    const uint32_t va = d_v + ev * kTile16 + half * 4 * (2048 >> 4);
                    const uint32_t to = tm + 256 + s * DH, tp = tm + s * 128 + half * 32;
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            mma_ts(to, tp + kk * 8, va + kk * (2048 >> 4), idO, kk ? 1u : (uint32_t)began);
                        if (half == 0) tc_commit(bar(&bars->half_done[s]));
                    }
                };
                auto qk = [&](int s, bool last) {            // last: of the slots that read this key tile
                    const uint32_t qa = d_q + (dual ? s * kTile16 : 0u), ka = d_k + ek * kTile16;
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < DH / 16; ++kk) {
                            const uint32_t off = (kk >> 2) * (kBox >> 4) + (kk & 3) * (32 >> 4);
                            mma_ss(tm + s * 128, qa + off, ka + off, idS, kk ? 1u : 0u);
                        }
                        tc_commit(bar(&bars->s_full[s]));
                        if (last) tc_commit(bar(&bars->kv_empty[ek]));
                    }
                };
                // Steps below `plain` of a two-tile segment need none of the cases.
                const int plain = dual ? min(min(n0, n1) - 1, first_masked) : 0;
                bool have_v = false;                         // V of step i has been waited for
#pragma unroll 1
                for (int i = -lead; i < nt; ++i) {
                    if (i >= 0 && i < plain) {
                        if (!have_v) ev = entry();
                        gave_up |= wait(&bars->p_half[0], p_phase);
                        tc_fence_after();
                        pv(0, 0, i > 0);
                        gave_up |= wait(&bars->p_full[0], p_phase);
                        tc_fence_after();
                        pv(0, 1, true);
                        ek = entry();
                        tc_fence_after();
                        qk(0, false);
                        gave_up |= wait(&bars->p_half[1], p_phase >> 1);
                        tc_fence_after();
                        pv(1, 0, i > 0);
                        gave_up |= wait(&bars->p_full[1], p_phase >> 1);
                        p_phase ^= 3u;
                        tc_fence_after();
                        pv(1, 1, true);
                        if (elect_one()) tc_commit(bar(&bars->kv_empty[ev]));
                        ev = entry();                        // (step i + 1 exists) under the products queued
                        have_v = true;
                        qk(1, true);
                        continue;
                    }
                    const int next = i + lead;
                    const bool more = next < nt;
                    if (next == nt && elect_one()) tc_commit(bar(&bars->q_empty));    // no product reads the queries any more
                    int bad = 0;
                    if (i >= 0) {
                        if (!have_v) ev = entry();
                        have_v = false;
                        if (i >= first_masked) {
                            const uint32_t gs = masked % ST, gp = masked / ST;
                            ++masked;
                            gave_up |= wait(&bars->guard[gs], gp);
                            bad = uniform(bars->bad[gs][0] | bars->bad[gs][1]);
                        }
                    }
                    const int s0 = dual ? 0 : (next & 1), s1 = dual ? 1 : s0;
#pragma unroll 1
                    for (int s = s0; s <= s1; ++s) {
                        const int ns = s ? n1 : n0;
                        const bool here = i >= 0 && i < ns;
                        if (here) {
                            gave_up |= wait(&bars->p_half[s], p_phase >> s);
                            tc_fence_after();
                            if (!bad) pv(s, 0, dual ? i > 0 : i > 1);    // else the softmax warps do it
                            else if (elect_one()) tc_commit(bar(&bars->half_done[s]));
                            gave_up |= wait(&bars->p_full[s], p_phase >> s);
                            p_phase ^= 1u << s;
                            tc_fence_after();
                            if (!bad) pv(s, 1, true);
                        }
                        if (i >= 0 && s == s1 && elect_one()) tc_commit(bar(&bars->kv_empty[ev]));
                        if (more && s == s0) {
                            ek = entry();
                            tc_fence_after();
                        }
                        if (more && next < ns) {
                            qk(s, s == s1);
                        } else {
                            if (here && elect_one()) tc_commit(bar(&bars->o_full[s]));
                            if (more && s == s1 && elect_one()) tc_commit(bar(&bars->kv_empty[ek]));
                        }
                    }
                }
                __syncwarp();
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
                    // A parity names a phase only to who knows that the one before has passed: the
                    // load warp says when the entry's own phase has begun.
                    ok = !lost(wait(&bars->go[masked % ST], masked / ST) | wait(&bars->kv_full[e % ST], e / ST));
                    if (!ok) break;
                    uint8_t* v = smem + L::RING + (e % ST) * L::TILE;
                    const int lo = max(0, si.kall - t * kCacheTile), hi = max(0, min(kCacheTile, si.kmax - t * kCacheTile));
                    for (int x = hi * 8 + me; x < kCacheTile * 8; x += 64)
#pragma unroll
                        for (int kb = 0; kb < L::KB; ++kb)
                            *reinterpret_cast<uint4*>(v + kb * kBox + x * 16) = make_uint4(0, 0, 0, 0);
                    // x * 0 is NaN for an infinity or a NaN, and the sum keeps it.
                    __nv_bfloat162 sum = __floats2bfloat162_rn(0.f, 0.f);
                    const __nv_bfloat162 zero = sum;
#pragma unroll 4
                    for (int x = lo * 8 + me; x < hi * 8; x += 64)
#pragma unroll
                        for (int kb = 0; kb < L::KB; ++kb) {
                            const uint4 u = *reinterpret_cast<const uint4*>(v + kb * kBox + x * 16);
                            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                sum = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w[k]), zero, sum);
                        }
                    bool found = __hisnan(__low2bfloat16(sum)) || __hisnan(__high2bfloat16(sum));
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    found = __any_sync(0xffffffffu, found);
                    if (lane == 0) {
                        bars->bad[masked % ST][warp - 2] = found;
                        mbar_arrive(bar(&bars->guard[masked % ST]));
                    }
                    ++masked;
                }
                cnt += 2 * nt;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        // -------------------------------------------------- softmax and output
        // Little is kept in registers from tile to tile (the scores need them): the segment
        // is read in shared memory where it is needed, and of the barriers' phases there
        // is one bit each.
        constexpr uint32_t kPhS = 1, kPhO = 2, kPhX = 4, kPhJ = 8;
        const int slot = (warp - 4) >> 2;
        const int qw = warp & 3;                           // TMEM lane quarter
        const int r = qw * 32 + lane;
        const uint32_t tS = tbase + ((uint32_t)(qw * 32) << 16) + slot * 128;
        const uint32_t tO = tS - slot * 128 + 256 + slot * DH;
        const int tok_in_tile = r / rep;
        const float sl2 = p.scale_log2;
        uint32_t ph = 0, masked = 0, cnt = 0;
        bool ok = true, reads_mine = false;
        for (int it = 0; ok; ++it) {
            if (lost(wait(&bars->seg_full[it % kSegSlots], it / kSegSlots))) break;
            const Seg& g = bars->seg[it % kSegSlots];
            if (!g.valid) break;
            const bool dual = g.ntok > TT;
            const int tok0 = dual ? slot * TT : 0;
            const int ntok = min(TT, g.ntok - tok0);       // tokens of this slot's tile
            const bool live = (qw * 32) / rep < ntok;      // some row of the warp has one
            const int step = dual ? 1 : 2, begin = g.t0 + (dual ? 0 : slot);
            int lim, first_part, mask0;                    // tiles, first partly masked one, index of a tile among those
            {
                const SegInfo si = seg_info(g, TT, tree);
                lim = slot ? si.n1 : si.n0;
                first_part = si.kall / kCacheTile;
                const int m0 = max(g.t0, first_part);
                mask0 = (int)masked - m0;
                masked += max(0, g.t1 - m0);
            }
            const bool work = begin < lim;
            float m = 0.f, l = 0.f;                        // (no key seen yet: m is arbitrary)
#pragma unroll 1
            for (int t = begin; t < lim; t += step) {
                ok = !lost(wait(&bars->s_full[slot], ph));
                if (!ok) break;
                ph ^= kPhS;
                tc_fence_after();
                const bool part = t >= first_part;
                uint32_t see[4] = {~0u, ~0u, ~0u, ~0u};
                bool bad = false;
                if (part) {
                    const uint32_t mi = (uint32_t)(mask0 + t);
                    ok = !lost(wait(&bars->guard[mi % ST], mi / ST));
                    if (!ok) break;
                    bad = bars->bad[mi % ST][0] | bars->bad[mi % ST][1];
                    // Keys of the tile that this row sees, one bit each.
                    const int tok = tok0 + min(tok_in_tile, ntok - 1);
                    const int all = tree ? g.base : g.first + tok + 1;         // keys before this one are seen
                    const uint64_t word = tree ? __ldg(p.tree + g.row + tok) : 0;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int k0 = t * kCacheTile + q * 32, n = all - k0;
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
                    }
                }
                // One pass over the scores in TMEM, a quarter (32 columns) at a time with the next
                // load in flight, and P handed over in two halves, so that the first half's
                // product runs under the second half's exponentials.  These start from the
                // reference m at hand, beside the search for the half's maximum (other units);
                // when that is more than 2^8 above m, or far below the row's first one, m
                // moves there, O and l are scaled, and they are repeated.
                uint32_t u[3][32];
                float2 ls[2];
                auto hide = [&](int q) {                 // masked scores of quarter q
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (!(see[q] >> j & 1u)) u[q % 3][j] = 0xff800000u;        // -inf
                };
                auto maximum = [&](int q) {              // of quarter q, in the exponent's unit
                    const uint32_t(&x)[32] = u[q % 3];
                    float a[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) a[k] = fmaxf(__uint_as_float(x[8 * k]), __uint_as_float(x[8 * k + 1]));
#pragma unroll
                    for (int j = 2; j < 8; j += 2)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            a[k] = max3(a[k], __uint_as_float(x[8 * k + j]), __uint_as_float(x[8 * k + j + 1]));
                    return fmaxf(max3(a[0], a[1], a[2]), a[3]) * sl2;
                };
                auto exponentials = [&](int q) {
                    const uint32_t(&x)[32] = u[q % 3];
                    const float ms = -m;
                    uint32_t w[16];
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        float2 e = fma2(make_float2(__uint_as_float(x[j]), __uint_as_float(x[j + 1])),
                                        make_float2(sl2, sl2), make_float2(ms, ms));
                        e.x = ex2(e.x);
                        e.y = ex2(e.y);
                        ls[(j >> 1) & 1] = add2(ls[(j >> 1) & 1], e);
                        w[j >> 1] = pack_bf16x2(e.x, e.y);
                    }
                    tmem_st_32x16(tS + q * 16, w);
                };
                auto half_tile = [&](int half) {
                    ls[0] = ls[1] = make_float2(0.f, 0.f);
                    const float mx = fmaxf(maximum(2 * half), maximum(2 * half + 1));
                    exponentials(2 * half);
                    exponentials(2 * half + 1);
                    const bool move = mx - m > 8.f || (l == 0.f && mx - m < -8.f && mx != -INFINITY);
                    if (__builtin_expect(__any_sync(0xffffffffu, move), 0)) {
                        const float up = mx, f = move && l != 0.f ? ex2(m - up) : 1.f;   // l = 0: so is O
                        if (move) m = up;
                        l *= f;
                        if (half || t != begin) {
                            if (half && !bad) {
                                ok = !lost(wait(&bars->half_done[slot], ph ^ kPhS));
                                tc_fence_after();
                            }
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
                        ls[0] = ls[1] = make_float2(0.f, 0.f);
                        exponentials(2 * half);
                        exponentials(2 * half + 1);
                    }
                    l += (ls[0].x + ls[0].y) + (ls[1].x + ls[1].y);
                    tmem_st_wait();
                };
                auto by_hand = [&](int half) {
                    const int i = t - g.t0, nt = g.t1 - g.t0;
                    const uint32_t e = cnt + i + min(nt, i + (dual ? 1 : 2));
                    ok = !lost(wait(&bars->kv_full[e % ST], e / ST));
                    const int kmax = tree ? g.kv_len : g.first + g.ntok;
                    pv_by_hand<DH>(tS, tO, smem + L::RING + (e % ST) * L::TILE, 64 * half,
                                   min(64 * half + 64, kmax - t * kCacheTile), half ? see[2] : see[0],
                                   half ? see[3] : see[1], t == begin && !half);
                };
                auto hand_over = [&](uint64_t* b) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(b));
                };
                // The other slot reads this one's last O: until it has, nothing is stored there, by a
                // product or by hand (an item's first half scales nothing).
                auto other_has_read = [&] {
                    if (reads_mine) ok = !lost(wait(&bars->x_done[slot ^ 1][qw], (ph / kPhX) ^ 1u));
                    reads_mine = false;
                };
                if (live) {
                    tmem_ld_32x32(tS, u[0]);
                    tmem_ld_32x32(tS + 32, u[1]);
                    landed(u[0]);
                    landed(u[1]);
                    tmem_ld_32x32(tS + 64, u[2]);
                    if (part && !__all_sync(0xffffffffu, (see[0] & see[1]) == ~0u)) {
                        hide(0);
                        hide(1);
                    }
                    if (t == begin) {                    // a reference that the next tiles seldom leave
                        const float mx = fmaxf(maximum(0), maximum(1));
                        m = mx == -INFINITY ? 0.f : mx;
                    }
                    half_tile(0);
                    if (bad) {
                        other_has_read();
                        if (!ok) break;
                        by_hand(0);
                    }
                    tmem_ld_32x32(tS + 96, u[0]);
                }
                other_has_read();
                if (!ok) break;
                hand_over(&bars->p_half[slot]);
                if (live) {
                    landed(u[0]);
                    landed(u[2]);
                    if (part && !__any_sync(0xffffffffu, (see[2] | see[3]) != 0u)) {
                        uint32_t w[16];
#pragma unroll
                        for (int j = 0; j < 16; ++j) w[j] = 0u;
                        tmem_st_32x16(tS + 32, w);
                        tmem_st_32x16(tS + 48, w);
                        tmem_st_wait();
                    } else {
                        if (part) {
                            hide(2);
                            hide(3);
                        }
                        half_tile(1);
                    }
                    if (bad) by_hand(1);
                }
                if (!ok) break;
                hand_over(&bars->p_full[slot]);
            }
            if (!ok) break;
            cnt += 2 * (g.t1 - g.t0);
            // ---- the segment's result
            if (work) {
                ok = !lost(wait(&bars->o_full[slot], ph / kPhO));
                if (!ok) break;
                ph ^= kPhO;
                tc_fence_after();
            }
            const bool mine = tok_in_tile < ntok;          // (rows past tile_tokens * rep have no token)
            const int token = g.row + tok0 + min(tok_in_tile, ntok - 1);
            // In a one-tile item both slots hold parts of the same rows: they tell each other the
            // maxima and sums, and each puts out half of the columns, reading both O's.
            // (Apart: parts of a cut item that are joined right after go out as they are.)
            const bool apart = g.part >= 0 && p.join_here;
            const bool joins = !dual && !apart && g.t0 + 1 < lim;   // (without two tiles lim is the same for both)
            if (l == 0.f) m = -INFINITY;                   // no key seen
            float fo = 1.f, fx = 0.f;
            if (joins) {
                bars->xml[slot][r] = make_float2(m, l);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&bars->x_full[slot][qw]));
                ok = !lost(wait(&bars->x_full[slot ^ 1][qw], ph / kPhX));
                if (!ok) break;
                ph ^= kPhX;
                tc_fence_after();
                const float2 x = bars->xml[slot ^ 1][r];
                const float top = fmaxf(m, x.x), ms = top == -INFINITY ? 0.f : top;
                fo = ex2(m - ms);
                fx = ex2(x.x - ms);
                l = l * fo + x.y * fx;
                m = top;
            }
            if (live && (dual || slot == 0 || joins || apart)) {
                float* po = nullptr;
                int po_step = 0;                           // from column to column of a multiple of 4
                __nv_bfloat16* out = nullptr;
                if (g.part >= 0) {
                    const int row = (dual || apart ? slot * 128 : 0) + r;
                    po = c.part_o + (apart ? ((size_t)g.part * 256 + row) * DH : part_at<DH>(g.part, row, 0));
                    po_step = apart ? 1 : 32;
                    if (mine && !(joins && slot)) c.part_ml[(size_t)g.part * 256 + row] = make_float2(work ? m : -INFINITY, l);
                } else {
                    out = p.out + (size_t)token * p.ld_out + (size_t)(g.head * rep + r - tok_in_tile * rep) * DH;
                    const float il = l == 0.f ? 0.f : 1.f / l;
                    fo *= il;
                    fx *= il;
                }
                const uint32_t tX = slot ? tO - DH : tO + DH;
                const int k_end = joins && !slot ? DH / 2 : DH;
#pragma unroll 1
                for (int k = joins && slot ? DH / 2 : 0; k < k_end; k += 16) {
                    uint32_t o[16], y[16];
                    if (work) tmem_ld_32x16(tO + k, o);
                    if (joins) tmem_ld_32x16(tX + k, y);
                    tmem_ld_wait();
                    float f[16];
                    // A factor or sum of 0 says that nothing was summed (O may hold anything then).
#pragma unroll
                    for (int j = 0; j < 16; ++j) f[j] = work && l != 0.f && fo != 0.f ? __uint_as_float(o[j]) * fo : 0.f;
                    if (joins)
#pragma unroll
                        for (int j = 0; j < 16; ++j) f[j] = fx != 0.f ? fmaf(__uint_as_float(y[j]), fx, f[j]) : f[j];
                    if (mine) {
                        if (po) {
#pragma unroll
                            for (int j = 0; j < 16; j += 4)
                                *reinterpret_cast<float4*>(po + (k + j) * po_step) = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; j += 8)
                                *reinterpret_cast<uint4*>(out + k + j) =
                                    make_uint4(pack_bf16x2(f[j], f[j + 1]), pack_bf16x2(f[j + 2], f[j + 3]),
                                               pack_bf16x2(f[j + 4], f[j + 5]), pack_bf16x2(f[j + 6], f[j + 7]));
                        }
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            if (joins) {
                // The other slot's O may be overwritten: it waits for this before its next one.
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&bars->x_done[slot][qw]));
                reads_mine = true;
            }
            if (apart) {
                // Whoever writes an item's last missing part joins them all.  (The barrier
                // orders the CTA's writes before the one fence and count.)
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&bars->part_done));
                const CacheShare& sh = c.shares[g.t0 > 0 ? blockIdx.x : blockIdx.x + 1];   // a share that begins in the item
                const int first = sh.first, last = sh.last;
                ok = !lost(wait(&bars->part_done, ph / kPhJ));
                if (!ok) break;
                if (warp == 4 && lane == 0) {
                    __threadfence();
                    const bool mine_last = atomicAdd(&c.arrived[first], 1) == last - first;
                    if (mine_last) c.arrived[first] = 0;
                    __threadfence();
                    bars->last_part = mine_last;
                    mbar_arrive(bar(&bars->join_go));
                }
                ok = !lost(wait(&bars->join_go, ph / kPhJ));
                if (!ok) break;
                ph ^= kPhJ;
                if (bars->last_part)
                    for (int r0 = warp - 4; r0 < g.ntok * rep; r0 += 8) join_row<DH>(c, p, g, first, last, r0, lane);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(&bars->seg_empty[it % kSegSlots]));
        }
    }
    __syncthreads();
    if (warp == 0) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tbase, kTmemCols);
    }
}

// Joins the parts of cut items.  Block (b, y) takes rows [32 y, 32 y + 32) of the
// item that CTA b of the attention began and did not finish, a warp half of the columns
// of eight of them.
template <int DH>
__global__ void __launch_bounds__(256) cache_join_kernel(const __grid_constant__ CacheDev c,
                                                         const __grid_constant__ AttendParams p) {
    pdl_wait();
    pdl_trigger();
    const int n_ctas = c.plan->n_ctas, b = blockIdx.x;
    if (!c.plan->ok || b + 1 >= n_ctas) return;
    const CacheShare next = c.shares[b + 1];
    if (next.within == 0 || next.first != b || next.last == b) return;
    const int two = cache_two_tiles(next.g.ntok, c.tile_tokens);
    const int rows = two ? 128 + (next.g.ntok - c.tile_tokens) * c.rep : next.g.ntok * c.rep;
    const int warp = threadIdx.x >> 5, r0 = blockIdx.y * 32 + (warp >> 1) * 8;
    if (r0 < rows)
        join_rows<DH, DH / 32>(c, p, next, rows, r0, (warp & 1) * (DH / 2), threadIdx.x & 31);
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
    // What the warpgroups ask for has to be within what the block is launched with, or
    // they would wait for it.
    static PerDevice regs;
    const int nreg = regs.get([] {
        cudaFuncAttributes fa = {};
        return cudaFuncGetAttributes(&fa, cache_attention_kernel<DH>) == cudaSuccess ? fa.numRegs : 0;
    });
    if (nreg * kThreads < 104 * 128 + 200 * 256) return cudaErrorInvalidConfiguration;
    e = launch_pdl(cache_attention_kernel<DH>, dim3(c.num_sms), dim3(kThreads), smem_bytes<DH>(), st, tm_q, tm_k, tm_v,
                   c, p);
    if (e != cudaSuccess || p.join_here) return e;
    return launch_pdl(cache_join_kernel<DH>, dim3(c.num_sms, (max_rows + 31) / 32), dim3(256), 0, st, c, p);
}

}  // namespace

cudaError_t launch_cache_attend(const CacheDev& c, const CUtensorMap& tm_q, const CUtensorMap& tm_k,
                                const CUtensorMap& tm_v, const AttendParams& p, int max_rows, cudaStream_t st) {
    return c.dh == 64 ? attend<64>(c, tm_q, tm_k, tm_v, p, max_rows, st)
                      : attend<128>(c, tm_q, tm_k, tm_v, p, max_rows, st);
}

}  // namespace tmoe
