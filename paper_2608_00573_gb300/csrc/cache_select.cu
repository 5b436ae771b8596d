// Choice of the pages that a query reads: bounds of the keys of whole pages ("blocks"), and
// for each token and key/value head the blocks whose bounds promise the largest scores.
//
//   lo_d = min_i k_id, hi_d = max_i k_id over a page's keys, held as floor(lo / u) and
//   ceil(hi / u) in 8 bits; u = 2^e, e the least one with max(|lo|, |hi|) <= 127 u
//   score = u max_h u_h sum_d max(c_hd lo_d, c_hd hi_d),  c_h = rint(q_h / u_h)
//
// With q+ = max(c, 0) and q- = min(c, 0) the sum is q- . lo + q+ . hi, a product of 8-bit numbers
// with 2 D terms.  It is at most 128 * 127 * 127 < 2^24, so that every score is exact in fp32 (but where
// its products with the units leave the normal range) and the order of the blocks (ties: the lower one) does not
// depend on how the sum is computed.
#include <algorithm>
#include <type_traits>

#include "cache.cuh"

namespace tmoe {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// Exponent of the unit of 8-bit values up to amax: the least e >= -126 with amax <= 127 2^e.
// amax = 2^(x+1) m with m in [1/2, 1): x - 6 if m <= 127/128, else x - 5.
__device__ __forceinline__ int unit_exponent(float amax) {
    const uint32_t b = __float_as_uint(amax);
    return max(-126, (int)(b >> 23) - 133 + ((b & 0x7fffffu) > 0x7e0000u));
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Bounds of one page and head by a warp: DH / 8 lanes to a row, 8 columns each.
template <int DH>
__device__ __forceinline__ void page_bounds(const CacheDev& c, int layer, int id, int h, int lane) {
    constexpr int LANES = DH / 8, U = DH / 16;        // lanes of a row, loads in flight (a page has a multiple of them)
    const size_t unit = ((size_t)layer * c.n_pages + id) * c.Hkv + h;
    const uint4* src = reinterpret_cast<const uint4*>(c.k + unit * c.page * DH) + lane;
    const uint32_t inf2 = 0x7f807f80u;
    uint32_t lo[4] = {inf2, inf2, inf2, inf2}, hi[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) hi[j] = inf2 | 0x80008000u;
    auto b2 = [](uint32_t& x) -> __nv_bfloat162& { return reinterpret_cast<__nv_bfloat162&>(x); };
    const int loads = c.page * LANES / 32;
    for (int i = 0; i < loads; i += U) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = src[(i + u) * 32];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {             // (a NaN stays)
                b2(lo[j]) = __hmin2_nan(b2(lo[j]), b2(w[j]));
                b2(hi[j]) = __hmax2_nan(b2(hi[j]), b2(w[j]));
            }
        }
    }
#pragma unroll
    for (int o = 16; o >= LANES; o >>= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t y = __shfl_xor_sync(0xffffffffu, lo[j], o), z = __shfl_xor_sync(0xffffffffu, hi[j], o);
            b2(lo[j]) = __hmin2_nan(b2(lo[j]), b2(y));
            b2(hi[j]) = __hmax2_nan(b2(hi[j]), b2(z));
        }
    // Magnitudes as bit patterns: an infinity or a NaN is larger than all others.
    uint32_t amax = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t a = lo[j] & 0x7fff7fffu, b = hi[j] & 0x7fff7fffu;
        amax = max(amax, max(max(a << 16, a & 0xffff0000u), max(b << 16, b & 0xffff0000u)));
    }
    amax = __reduce_max_sync(0xffffffffu, amax);
    const bool finite = amax < 0x7f800000u;
    const int e = unit_exponent(__uint_as_float(amax));
    const float inv = finite ? two_to(-e) : 0.f;
    uint32_t cl[2] = {0, 0}, ch[2] = {0, 0};
    if (finite) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = j & 1 ? bf16_hi(lo[j >> 1]) : bf16_lo(lo[j >> 1]);
            const float b = j & 1 ? bf16_hi(hi[j >> 1]) : bf16_lo(hi[j >> 1]);
            // (Outwards also where the product is too small for a float.)
            const int l = a < 0.f ? min(__float2int_rd(a * inv), -1) : __float2int_rd(a * inv);
            const int u = b > 0.f ? max(__float2int_ru(b * inv), 1) : __float2int_ru(b * inv);
            cl[j >> 2] |= ((uint32_t)l & 0xffu) << (8 * (j & 3));
            ch[j >> 2] |= ((uint32_t)u & 0xffu) << (8 * (j & 3));
        }
    }
    uint2* to = reinterpret_cast<uint2*>(c.codes + unit * 2 * DH);
    if (lane < LANES) {
        to[lane] = make_uint2(cl[0], cl[1]);
        to[LANES + lane] = make_uint2(ch[0], ch[1]);
    }
    if (lane == 0) c.scales[unit] = finite ? two_to(e) : INFINITY;
}

// Pages [from, to) of a sequence: a warp takes one page and head at a time.
template <int DH>
__device__ __forceinline__ void sequence_bounds(const CacheDev& c, int layer, int seq, int from, int to) {
    const int lane = threadIdx.x & 31;
    const int* row = c.table + (size_t)seq * c.max_pages;
    for (long long u = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); u < (long long)(to - from) * c.Hkv;
         u += (long long)gridDim.x * kWarps) {
        const int id = row[from + (int)(u / c.Hkv)];
        if (id < 0 || id >= c.n_pages) {
            if (lane == 0) atomicCAS(c.err, 0, ERR_CACHE_STATE);
            continue;
        }
        page_bounds<DH>(c, layer, id, (int)(u % c.Hkv), lane);
    }
}

// Bound: HBM, each filled page's keys once: 9 prompts, 16384 tokens, 32 MB, 6.1 us in a row of
// launches (5.2 TB/s, part of it out of L2); a decode step fills few pages, 2.7 us, latency.  A warp to a page
// and head needs no sums across warps; rows of 8 columns a lane are whole lines.
template <int DH>
__global__ void __launch_bounds__(kThreads) cache_bounds_kernel(const __grid_constant__ CacheDev c, int layer, int whole) {
    pdl_wait();
    pdl_trigger();
    if (!c.plan->ok) return;
    const CacheSeq s = c.seqs[blockIdx.y];
    sequence_bounds<DH>(c, layer, s.seq, whole ? 0 : (s.kv_len - s.q_len) >> c.page_shift, s.kv_len >> c.page_shift);
}

// The pages that accepted drafts came to lie in, all layers.
template <int DH, int N>
__global__ void __launch_bounds__(kThreads) cache_bounds_accepted_kernel(const __grid_constant__ CacheDev c,
                                                                         const __grid_constant__ CacheList<N> l,
                                                                         const int* n_acc, const int* accepted) {
    pdl_wait();
    pdl_trigger();
    const int len = accepted[blockIdx.y];
    if (len < 0) return;                              // the sequence was left as it is
    const int from = (len - n_acc[blockIdx.y]) >> c.page_shift;
    for (int layer = blockIdx.z; layer < c.layers; layer += gridDim.z)
        sequence_bounds<DH>(c, layer, l.a[blockIdx.y], from, len >> c.page_shift);
}

// Scores as whole numbers in the same order.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// ------------------------------------------------------------------ queries and scores

// Query heads as columns of a matrix of 8-bit codes, 2 D rows: the negative ones first, then the
// positive ones, so that a block's score for a head is the product of its bounds, lo first, with
// that column.  A token has M columns (1, 2, 4), or with M = 8 a multiple of 8; those past its
// query heads repeat the last one.  Eight columns are a group; columns past the tokens are zero.
__host__ __device__ constexpr int columns_of(int rep) { return rep > 4 ? (rep + 7) & ~7 : rep == 3 ? 4 : rep; }
__host__ __device__ inline int coded_columns(int rep, int tokens) { return (tokens * columns_of(rep) + 7) & ~7; }
__host__ __device__ inline size_t coded_bytes(int rep, int dh, int tokens) { return (size_t)coded_columns(rep, tokens) * (2 * dh + 4); }

template <int DH>
struct Coded {
    int8_t* code;                      // [columns][2 DH]
    float* unit;                       // [columns]
    __device__ Coded(void* at, int columns) {
        code = static_cast<int8_t*>(at);
        unit = reinterpret_cast<float*>(code + (size_t)columns * 2 * DH);
    }
};

// Columns `from`, `from` + step and so on by this warp; `tokens` of the tokens exist.
template <int DH>
__device__ __forceinline__ void code_queries(const CacheDev& c, const SelectParams& p, const Coded<DH>& out, int columns, int h,
                                             int first_token, int tokens, int from, int step) {
    constexpr int K = DH / 64, SIDE = 4;              // (columns whose loads are in flight together)
    const int lane = threadIdx.x & 31, per = columns_of(c.rep);
    for (int u0 = from; u0 < columns; u0 += SIDE * step) {
        uint32_t w[SIDE][K];
        bool real[SIDE];
#pragma unroll
        for (int i = 0; i < SIDE; ++i) {
            const int u = min(u0 + i * step, columns - 1), k = u / per, r = min(u - k * per, c.rep - 1);
            real[i] = k < tokens;
            const __nv_bfloat16* q = p.q + (size_t)(first_token + (real[i] ? k : 0)) * p.ld_q + (size_t)(h * c.rep + r) * DH + lane * 2 * K;
#pragma unroll
            for (int j = 0; j < K; ++j) w[i][j] = reinterpret_cast<const uint32_t*>(q)[j];
        }
#pragma unroll
        for (int i = 0; i < SIDE; ++i) {
            const int u = u0 + i * step;
            if (u >= columns) break;
            uint32_t amax = 0;
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const uint32_t a = w[i][j] & 0x7fff7fffu;
                amax = max(amax, max(a << 16, a & 0xffff0000u));
            }
            amax = __reduce_max_sync(0xffffffffu, amax);
            const bool finite = real[i] && amax < 0x7f800000u;
            const int e = unit_exponent(__uint_as_float(amax));
            const float inv = finite ? two_to(-e) : 0.f;
            uint16_t* neg = reinterpret_cast<uint16_t*>(out.code + (size_t)u * 2 * DH) + lane * K;
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const int a = finite ? __float2int_rn(bf16_lo(w[i][j]) * inv) : 0, b = finite ? __float2int_rn(bf16_hi(w[i][j]) * inv) : 0;
                neg[j] = (uint16_t)((min(a, 0) & 0xff) | (min(b, 0) & 0xff) << 8);
                neg[DH / 2 + j] = (uint16_t)(max(a, 0) | max(b, 0) << 8);
            }
            if (lane == 0) out.unit[u] = finite ? two_to(e) : 0.f;
        }
    }
}

__device__ __forceinline__ void mma_s8(int (&c)[4], int a0, int a1, int a2, int a3, int b0, int b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Scores of one sequence's blocks for tokens [a, end) of the coded ones: put(token, block, key).
// A warp takes 16 blocks from 16 `from` on, then those `stride` times as many on, below F: the 16 rows
// of a product with 8 columns and 2 D terms in whole numbers.  The terms' order is free, so a
// lane takes 16 bytes of a row at a time, as they lie.  (Integer products are no faster here than four-number
// dot products, 151 and 149 T operations a second measured, but need no sums across lanes: 800 tokens' chunks 124 us
// with those, 28 with these and the choice by one histogram.)
// ONE: all columns are one group, which stays in registers.
template <int DH, int M, bool ONE, class Put>
__device__ __forceinline__ void score_blocks(const CacheDev& c, int layer_at, const Coded<DH>& q, int h, int seq, int F, int a, int end,
                                             int from, int stride, Put put) {
    constexpr int P = DH / 32;                        // 16-byte pieces of a lane and row
    const int lane = threadIdx.x & 31, r = lane >> 2, part = lane & 3;
    const int* row = c.table + (size_t)seq * c.max_pages;
    const size_t layer = (size_t)layer_at * c.n_pages;
    const int per = columns_of(c.rep);                // (M, or a multiple of 8)
    const int g0 = a * per / 8, g1 = (end * per + 7) / 8;
    int4 col[P];
    auto columns = [&](int g) {
#pragma unroll
        for (int k = 0; k < P; ++k) col[k] = reinterpret_cast<const int4*>(q.code + (size_t)(g * 8 + r) * 2 * DH)[4 * k + part];
    };
    if (ONE) columns(g0);
    int next[2];
    auto look_up = [&](int b0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) next[i] = b0 + r + 8 * i < F ? row[b0 + r + 8 * i] : 0;
    };
    look_up(from * 16);
    for (int b0 = from * 16; b0 < F; b0 += stride * 16) {
        int4 x[2][P];
        float scale[2];
        bool there[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            there[i] = next[i] >= 0 && next[i] < c.n_pages;
            const size_t unit = (layer + (there[i] ? next[i] : 0)) * c.Hkv + h;
            const int4* src = reinterpret_cast<const int4*>(c.codes + unit * 2 * DH) + part;
#pragma unroll
            for (int k = 0; k < P; ++k) x[i][k] = __ldg(src + 4 * k);
            scale[i] = __ldg(c.scales + unit);
        }
        look_up(b0 + stride * 16);
        // (A page without an index scores nothing; + 0 turns -0 into 0.)
        auto give = [&](int i, int t, float best) {
            const int b = b0 + r + 8 * i;
            if (b >= F || t < a || t >= end) return;
            const float s = scale[i] == INFINITY ? INFINITY : best * scale[i] + 0.f;
            put(t, b, there[i] ? ordered(s) : 0u);
            if (!there[i]) atomicCAS(c.err, 0, ERR_CACHE_STATE);
        };
        float best[2] = {-INFINITY, -INFINITY};
        for (int g = g0; g < g1; ++g) {
            if (!ONE) columns(g);
            int sum[4] = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < P; ++k) {
                mma_s8(sum, x[0][k].x, x[1][k].x, x[0][k].y, x[1][k].y, col[k].x, col[k].y);
                mma_s8(sum, x[0][k].z, x[1][k].z, x[0][k].w, x[1][k].w, col[k].z, col[k].w);
            }
            const float2 unit = *reinterpret_cast<const float2*>(q.unit + g * 8 + part * 2);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float s0 = (float)sum[2 * i] * unit.x, s1 = (float)sum[2 * i + 1] * unit.y;
                if (M == 1) {
                    give(i, g * 8 + part * 2, s0);
                    give(i, g * 8 + part * 2 + 1, s1);
                } else {
                    float s = fmaxf(s0, s1);
                    if (M == 2) give(i, g * 4 + part, s);
                    if (M >= 4) s = fmaxf(s, __shfl_xor_sync(0xffffffffu, s, 1));
                    if (M == 4 && !(part & 1)) give(i, g * 2 + (part >> 1), s);
                    if (M == 8) {
                        best[i] = fmaxf(best[i], fmaxf(s, __shfl_xor_sync(0xffffffffu, s, 2)));
                        if ((g * 8 + 8) % per == 0) {
                            if (part == 0) give(i, g * 8 / per, best[i]);
                            best[i] = -INFINITY;
                        }
                    }
                }
            }
        }
    }
}

// ------------------------------------------------------------------------------- choice

// Scratch of a choice in shared memory.
constexpr int kCandidates = 64;
struct Choice {
    uint32_t hist[288];                // counts of digits, see hist_at
    uint32_t key[kCandidates];
    int col[kCandidates];
    int count;                         // candidates
    uint32_t both[kWarps], any[kWarps];
    int digit, left, last;             // of the digit that holds the n-th key; column of the last key taken
    uint32_t bound;                    // that key
};

// Keys above `bound` are taken, and those equal to it up to column `last`.
struct Cut {
    uint32_t bound;
    int last;
    __device__ bool takes(uint32_t key, int col) const { return key > bound || (key == bound && col <= last); }
};

// Where a digit's count lies (a lane reads eight digits in a row: no two lanes the same bank).
__device__ __forceinline__ int hist_at(uint32_t digit) { return (int)(digit + (digit >> 3)); }

// The cut that takes the n largest of keys [lo, hi) (n < hi - lo; equal ones: lower columns first).
// WARPS warps take part, `me` their thread; sync is their barrier.  One pass counts the keys by
// the 8 bits below those that all agree on, one collects the keys of the digit that the n-th has,
// which are ranked one by one; when they are many (keys in few clusters), bits are
// decided one at a time instead.
template <int WARPS, class Key, class Sync>
__device__ __forceinline__ Cut cut_of(Key key, int lo, int hi, int n, int me, Choice& s, Sync sync) {
    constexpr int THREADS = WARPS * 32;
    const int warp = me >> 5, lane = me & 31;
    uint32_t both = 0xffffffffu, any = 0;
    for (int i = lo + me; i < hi; i += THREADS) {
        const uint32_t k = key(i);
        both &= k;
        any |= k;
    }
    for (int i = me; i < 288; i += THREADS) s.hist[i] = 0;
    if (me == 0) s.count = 0;
    both = __reduce_and_sync(0xffffffffu, both);
    any = __reduce_or_sync(0xffffffffu, any);
    if (WARPS > 1) {
        if (lane == 0) {
            s.both[warp] = both;
            s.any[warp] = any;
        }
    }
    sync();
    if (WARPS > 1) {
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            both &= s.both[w];
            any |= s.any[w];
        }
    }
    const int shift = max(0, 24 - __clz(both ^ any | 1u));      // the digit is the key's bits shift .. shift + 7
    const uint32_t high = shift > 23 ? 0u : both >> (shift + 8) << (shift + 8);   // common bits above it
    for (int i = lo + me; i < hi; i += THREADS) atomicAdd(&s.hist[hist_at(key(i) >> shift & 255u)], 1u);
    sync();
    if (warp == 0) {
        int mine[8], sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += mine[j] = s.hist[hist_at(255 - lane * 8 - j)];
        int upto = sum;                               // keys of this lane's digits and larger ones
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
        }
        int before = upto - sum;
        if (before < n && upto >= n) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (before < n && before + mine[j] >= n) {
                    s.digit = 255 - lane * 8 - j;
                    s.left = n - before;
                }
                before += mine[j];
            }
        }
    }
    sync();
    const uint32_t low = high | (uint32_t)s.digit << shift;     // least key with the digit
    const int left = s.left, count = (int)s.hist[hist_at(s.digit)];
    if (left == count) return low ? Cut{low - 1, -1} : Cut{0, 0x7fffffff};     // all of the digit
    const uint32_t mask = shift ? ~((1u << shift) - 1u) : ~0u;
    if (count <= kCandidates) {
        for (int i = lo + me; i < hi; i += THREADS) {
            const uint32_t k = key(i);
            if ((k & mask) == low) {
                const int at = atomicAdd(&s.count, 1);
                s.key[at] = k;
                s.col[at] = i;
            }
        }
        sync();
        if (warp == 0) {
#pragma unroll
            for (int x = lane; x < kCandidates; x += 32)
                if (x < count) {
                    int rank = 0;
                    for (int y = 0; y < count; ++y)
                        rank += s.key[y] > s.key[x] || (s.key[y] == s.key[x] && s.col[y] < s.col[x]);
                    if (rank == left - 1) {
                        s.bound = s.key[x];
                        s.last = s.col[x];
                    }
                }
        }
        sync();
        return Cut{s.bound, s.last};
    }
    // The largest key with at least `left` of the candidates at or above it, bit by bit.
    auto total = [&](int v) {
        v = __reduce_add_sync(0xffffffffu, v);
        if (WARPS == 1) return v;
        sync();
        if (lane == 0) s.hist[warp] = v;
        sync();
        int all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) all += s.hist[w];
        return all;
    };
    uint32_t bound = low;
    int above = 0;                                    // candidates above all that begin with bound's decided bits
    for (int bit = shift - 1; bit >= 0; --bit) {
        const uint32_t t = bound | 1u << bit;
        int at_least = 0;
        for (int i = lo + me; i < hi; i += THREADS) {
            const uint32_t k = key(i);
            at_least += (k & mask) == low && k >= t;
        }
        at_least = total(at_least);
        if (at_least >= left) bound = t;
        else above = at_least;
    }
    // Of the keys equal to it the first left - above: the column of the last of them.
    int tie = left - above, last = 0x7fffffff;
    for (int i0 = lo; i0 < hi && tie > 0; i0 += THREADS) {
        const int i = i0 + me;
        const bool same = i < hi && key(i) == bound;
        const uint32_t m = __ballot_sync(0xffffffffu, same);
        int before = 0;
        if (WARPS > 1) {
            sync();
            if (lane == 0) s.hist[warp] = __popc(m);
            sync();
            for (int w = 0; w < warp; ++w) before += s.hist[w];
        }
        if (same && before + __popc(m & ((1u << lane) - 1u)) == tie - 1) s.last = i;
        tie -= total(same);
    }
    sync();
    last = s.last;
    return Cut{bound, last};
}

// A sequence's list when all of its F blocks fit, or its forced columns: [0, first) and [F - last, F).
__device__ __forceinline__ void list_ends(int* out, int n, int F, int first, int last, int me, int threads) {
    if (F <= n) {
        for (int i = me; i < n; i += threads) out[i] = i < F ? i : -1;
    } else {
        for (int i = me; i < first; i += threads) out[i] = i;
        for (int i = me; i < last; i += threads) out[n - last + i] = F - last + i;
    }
}

// ------------------------------------------------------------------------------ kernels

// TILE tokens (eight, or one) and a key/value head: scores in shared memory, from bounds that are read once
// for the tokens of a sequence, then a warp chooses for each token, or all for the one.
//
// Bound: the chain of a list, which one warp makes (passes over its scores with atomics and barriers between, some 300
// instructions); issue slots are 50 % busy, integer products, 2 D per block of keys and query head, 20 %.  Measured: 800
// tokens' chunks behind 6000 to 15000 positions, 12 heads of 64 columns, pages of 32, 27.8 us; one token over 312 blocks,
// 32 heads on 8, 8.2 us, latency.
constexpr int kTile = 8, kTileBytes = 110 * 1024;
template <int TILE>
struct TileChoice {
    Choice of[TILE > 1 ? kWarps : 1];
    int taken[kWarps];
};
__host__ __device__ inline size_t score_row(const CacheDev& c) { return ((size_t)c.max_pages + 3) & ~size_t(3); }
template <int TILE>
__host__ __device__ inline size_t tile_bytes(const CacheDev& c) {
    return TILE * score_row(c) * 4 + coded_bytes(c.rep, c.dh, TILE) + sizeof(TileChoice<TILE>);
}

template <int DH, int M, int TILE>
__global__ void __launch_bounds__(kThreads, 3) cache_select_tile_kernel(const __grid_constant__ CacheDev c,
                                                                     const __grid_constant__ SelectParams p) {
    extern __shared__ __align__(16) uint32_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = p.n, columns = coded_columns(c.rep, TILE);
    const size_t row_len = score_row(c);
    const Coded<DH> q(smem + TILE * row_len, columns);
    TileChoice<TILE>& choice =
        *reinterpret_cast<TileChoice<TILE>*>(reinterpret_cast<uint8_t*>(smem + TILE * row_len) + coded_bytes(c.rep, DH, TILE));
    const int h = blockIdx.x % c.Hkv, first_token = blockIdx.x / c.Hkv * TILE, tokens = min(TILE, p.T - first_token);
    pdl_wait();
    pdl_trigger();
    if (!c.plan->ok) return;
    code_queries<DH>(c, p, q, columns, h, first_token, tokens, warp, kWarps);
    __syncthreads();
    // Runs of tokens of one sequence (one run for most blocks of threads).
    for (int a = 0; a < tokens;) {
        const CacheToken tok = c.tokens[first_token + a];
        const int end = min(tokens, a + tok.kv_len - tok.pos), F = tok.base >> c.page_shift;
        if (F > n) {
            score_blocks<DH, M, TILE == 1 ? M < 8 : M == 1>(c, p.layer, q, h, tok.seq, F, a, end, warp, kWarps, [&](int t, int b, uint32_t key) { smem[t * row_len + b] = key; });
            __syncthreads();
        }
        if (TILE == 1) {
            int* out = p.blocks + ((size_t)first_token * c.Hkv + h) * n;
            list_ends(out, n, F, p.first, p.last, threadIdx.x, kThreads);
            const int lo = p.first, hi = F - p.last, want = n - p.first - p.last;
            if (F <= n || want == 0) return;
            const Cut cut = cut_of<kWarps>([&](int i) { return smem[i]; }, lo, hi, want, threadIdx.x, choice.of[0], [] { __syncthreads(); });
            // A warp takes a range of columns: how many, then which.
            const int per = (hi - lo + kThreads - 1) / kThreads * 32, i0 = lo + warp * per, i1 = min(hi, i0 + per);
            int taken = 0;
            for (int i = i0 + lane; i - lane < i1; i += 32)
                taken += __popc(__ballot_sync(0xffffffffu, i < i1 && cut.takes(smem[i], i)));
            if (lane == 0) choice.taken[warp] = taken;
            __syncthreads();
            int at = p.first;
            for (int w = 0; w < warp; ++w) at += choice.taken[w];
            for (int i = i0 + lane; i - lane < i1; i += 32) {
                const bool take = i < i1 && cut.takes(smem[i], i);
                const uint32_t m = __ballot_sync(0xffffffffu, take);
                if (take) out[at + __popc(m & ((1u << lane) - 1u))] = i;
                at += __popc(m);
            }
            return;
        }
        for (int t = a + warp; t < end; t += kWarps) {
            int* out = p.blocks + ((size_t)(first_token + t) * c.Hkv + h) * n;
            list_ends(out, n, F, p.first, p.last, lane, 32);
            const int lo = p.first, hi = F - p.last, want = n - p.first - p.last;
            if (F <= n || want == 0) continue;
            const uint32_t* key = smem + t * row_len;
            const Cut cut = cut_of<1>([&](int i) { return key[i]; }, lo, hi, want, lane, choice.of[warp], [] { __syncwarp(); });
            int at = p.first;
            for (int i0 = lo; i0 < hi; i0 += 32) {
                const int i = i0 + lane;
                const bool take = i < hi && cut.takes(key[i], i);
                const uint32_t m = __ballot_sync(0xffffffffu, take);
                if (take) out[at + __popc(m & ((1u << lane) - 1u))] = i;
                at += __popc(m);
            }
            __syncwarp();
        }
        a = end;
        if (a < tokens) __syncthreads();              // the next run writes scores
    }
}

// Single tokens: the scores, to a buffer; then a block of threads per token and key/value head chooses.
// All sixteens of blocks of all tokens and heads lie on a line, token by token, and every warp takes
// the same number of them in a row: a warp meets few tokens, whose queries it codes for
// itself, and long sequences cost no one more than short ones.  (A block of threads for each
// token and head, or several for long ones: 48 contexts of 4000 to 40000 took 25.2 us with the choice, this way
// 23.0.)
//
// Bound: HBM, 2 D + 4 bytes per block of keys and head; 69 MB of bounds and the choice of 384 lists 23.0 us, 0.44
// of the copy rate: the integer pipe is 40 % busy, and the choice behind it takes a third.
constexpr int kSlice = 1024;                          // tokens at a time
__host__ __device__ inline int score_warps(const CacheDev& c) {
    const int fit = (int)(80 * 1024 / coded_bytes(c.rep, c.dh, 1));
    return fit < kWarps ? fit : kWarps;
}

template <int DH, int M>
__global__ void __launch_bounds__(kThreads, 3) cache_score_kernel(const __grid_constant__ CacheDev c,
                                                               const __grid_constant__ SelectParams p, int first_token, int tokens) {
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ int s_pre[kSlice + 1];                 // sixteens of one head before each token
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int columns = columns_of(c.rep);
    const Coded<DH> q(reinterpret_cast<uint8_t*>(smem) + warp * coded_bytes(c.rep, DH, 1), coded_columns(c.rep, 1));
    pdl_wait();
    pdl_trigger();
    const int ok = c.plan->ok;
    for (int t = threadIdx.x; t < tokens; t += blockDim.x) {
        const int F = c.tokens[first_token + t].base >> c.page_shift;
        s_pre[t] = F > p.n ? (F + 15) >> 4 : 0;
    }
    if (!ok) return;
    __syncthreads();
    if (warp == 0) {
        int sum = 0;
        for (int t0 = 0; t0 < tokens; t0 += 32) {
            const int t = t0 + lane, mine = t < tokens ? s_pre[t] : 0;
            int x = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            if (t < tokens) s_pre[t] = sum + x - mine;
            sum += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) s_pre[tokens] = sum;
    }
    __syncthreads();
    const long long all = (long long)s_pre[tokens] * c.Hkv, n_warps = (long long)gridDim.x * warps;
    const long long w = (long long)blockIdx.x * warps + warp;
    long long u = all * w / n_warps;
    const long long u1 = all * (w + 1) / n_warps;
    while (u < u1) {
        // The last token whose sixteens begin at or before u (tokens without any share their begin with the next).
        const int at = (int)(u / c.Hkv);
        int lo = 0, hi = tokens;
        while (hi - lo > 1) {
            const int m = (lo + hi) >> 1;
            if (s_pre[m] <= at) lo = m;
            else hi = m;
        }
        const int turns = s_pre[lo + 1] - s_pre[lo], in = (int)(u - (long long)s_pre[lo] * c.Hkv);
        const int h = in / turns, from = in - h * turns, to = (int)min((long long)turns, from + (u1 - u));
        const CacheToken tok = c.tokens[first_token + lo];
        code_queries<DH>(c, p, q, columns, h, first_token + lo, 1, 0, 1);
        __syncwarp();
        uint32_t* out = c.scores + (size_t)(lo * c.Hkv + h) * score_row(c);
        score_blocks<DH, M, M < 8>(c, p.layer, q, h, tok.seq, min(tok.base >> c.page_shift, to * 16), 0, 1, from, 1,
                                   [&](int, int b, uint32_t key) { out[b] = key; });
        __syncwarp();
        u += to - from;
    }
}

__global__ void __launch_bounds__(kThreads) cache_choose_kernel(const __grid_constant__ CacheDev c,
                                                                const __grid_constant__ SelectParams p, int first_token) {
    constexpr int kHeld = 8;                          // keys of a thread that stay in registers
    __shared__ Choice choice;
    __shared__ int s_taken[kHeld][kWarps];
    const int item = blockIdx.x, k = item / c.Hkv, h = item - k * c.Hkv, n = p.n;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    pdl_trigger();
    const int ok = c.plan->ok, F = c.tokens[first_token + k].base >> c.page_shift;
    if (!ok) return;
    int* out = p.blocks + ((size_t)(first_token + k) * c.Hkv + h) * n;
    const int lo = p.first, hi = F - p.last, want = n - p.first - p.last;
    const uint32_t* keys = c.scores + (size_t)item * score_row(c);
    // Turn j of the threads holds the columns lo + j kThreads ..: the first kHeld turns in registers.
    uint32_t held[kHeld];
    if (F > n) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            const int i = lo + j * kThreads + threadIdx.x;
            held[j] = i < hi ? __ldcg(keys + i) : 0u;
        }
    }
    list_ends(out, n, F, p.first, p.last, threadIdx.x, kThreads);
    if (F <= n || want == 0) return;
    auto sync = [] { __syncthreads(); };
    const bool few = hi - lo <= kHeld * kThreads;
    auto key = [&](int i) {
        uint32_t v = held[0];
#pragma unroll
        for (int j = 1; j < kHeld; ++j) v = i - lo >= j * kThreads ? held[j] : v;
        return v;
    };
    const Cut cut = few ? cut_of<kWarps>(key, lo, hi, want, threadIdx.x, choice, sync)
                        : cut_of<kWarps>([&](int i) { return __ldcg(keys + i); }, lo, hi, want, threadIdx.x, choice, sync);
    const uint32_t below = (1u << lane) - 1u;
    int at = p.first;
    for (int j0 = 0; lo + j0 * kThreads < hi; j0 += kHeld) {
        uint32_t takes[kHeld];
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            const int i = lo + (j0 + j) * kThreads + threadIdx.x;
            const uint32_t v = j0 == 0 ? held[j] : i < hi ? __ldcg(keys + i) : 0u;
            takes[j] = __ballot_sync(0xffffffffu, i < hi && cut.takes(v, i));
            if (lane == 0) s_taken[j][warp] = __popc(takes[j]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
            int mine = at;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const int v = s_taken[j][w];
                mine += w < warp ? v : 0;
                at += v;
            }
            if (takes[j] >> lane & 1u) out[mine + __popc(takes[j] & below)] = lo + (j0 + j) * kThreads + threadIdx.x;
        }
        __syncthreads();
    }
}

template <int DH, int M, int TILE>
cudaError_t tile_launch(const CacheDev& c, const SelectParams& p, cudaStream_t st, int& launches) {
    static PerDevice attr;
    const cudaError_t e = (cudaError_t)attr.get([] {
        return (int)cudaFuncSetAttribute(cache_select_tile_kernel<DH, M, TILE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTileBytes);
    }, true);
    if (e != cudaSuccess) return e;
    launches = 1;
    return launch_pdl(cache_select_tile_kernel<DH, M, TILE>, dim3((unsigned)((p.T + TILE - 1) / TILE * c.Hkv)), dim3(kThreads),
                      tile_bytes<TILE>(c), st, c, p);
}

template <int DH, int M>
cudaError_t select_launch(const CacheDev& c, const SelectParams& p, cudaStream_t st, int& launches) {
    // Eight tokens to a block of threads when sequences have as many and their scores fit beside those of another
    // block; one to a block for few tokens of short sequences (one launch less: one token over 312 blocks
    // 8.3 us instead of 8.6, and 3 us less on the host).  Both hold scores for all columns of the table, whose width decides,
    // because the host does not know the lengths: 800 tokens' chunks behind 6000 to 15000 positions, 12 heads of 64 columns, pages of
    // 32, take 33 us with 480 columns, 34 with 1480, 43 with 2480 and 2980 (two blocks to an SM instead of three), and token by token
    // 175 with 3980, 222 with 8670, 504 with 30480 (slices of fewer tokens); 32 heads on 8, pages of 64, 33, 33, 37, 37,
    // 103, 143, 292.  48 single tokens 23.0 with 1240 to 9430 columns, 34.5 with 31240.
    if (p.max_q >= kTile && tile_bytes<kTile>(c) <= kTileBytes) return tile_launch<DH, M, kTile>(c, p, st, launches);
    if ((long long)p.T * c.Hkv <= 64 && c.max_pages <= 1024 && tile_bytes<1>(c) <= kTileBytes) return tile_launch<DH, M, 1>(c, p, st, launches);
    // As many tokens at a time as the buffer has room for.
    const int most = (int)std::min<size_t>(std::min(p.T, kSlice), cache_score_keys(c) / (score_row(c) * c.Hkv));
    const int warps = score_warps(c);
    const size_t smem = coded_bytes(c.rep, c.dh, 1) * warps;
    static PerDevice attr;
    cudaError_t e = (cudaError_t)attr.get([] {
        return (int)cudaFuncSetAttribute(cache_score_kernel<DH, M>, cudaFuncAttributeMaxDynamicSharedMemorySize, 80 * 1024);
    }, true);
    for (int t = 0; t < p.T && e == cudaSuccess; t += most) {
        const int tokens = std::min(most, p.T - t);
        // As many warps as are resident, with a sixteen of blocks each at least.
        const long long turns = (long long)tokens * c.Hkv * ((c.max_pages + 15) / 16);
        const unsigned blocks = (unsigned)std::min<long long>(3LL * c.num_sms, (turns + warps - 1) / warps);
        e = launch_pdl(cache_score_kernel<DH, M>, dim3(blocks), dim3(warps * 32), smem, st, c, p, t, tokens);
        if (e == cudaSuccess) e = launch_pdl(cache_choose_kernel, dim3((unsigned)(tokens * c.Hkv)), dim3(kThreads), 0, st, c, p, t);
        launches += 2;
    }
    return e;
}

template <int N>
cudaError_t accepted_launch(const CacheDev& c, int n, const int* seq, const int* n_acc, const int* accepted, cudaStream_t st) {
    CacheList<N> l;
    l.n = n;
    std::copy(seq, seq + n, l.a);
    // At most 64 tokens: 64 / page + 1 pages fill.
    const unsigned x = (unsigned)(((kTreeMax / c.page + 1) * c.Hkv + kWarps - 1) / kWarps);
    const dim3 grid(x, (unsigned)n, (unsigned)std::min(c.layers, 65535));
    return c.dh == 64 ? launch_pdl(cache_bounds_accepted_kernel<64, N>, grid, dim3(kThreads), 0, st, c, l, n_acc, accepted)
                      : launch_pdl(cache_bounds_accepted_kernel<128, N>, grid, dim3(kThreads), 0, st, c, l, n_acc, accepted);
}

}  // namespace

cudaError_t launch_cache_bounds(const CacheDev& c, int layer, int n, int max_q, int whole, cudaStream_t st) {
    const long long pages = whole ? c.max_pages : std::min(max_q / c.page + 1, c.max_pages);
    const unsigned x = (unsigned)std::min<long long>((pages * c.Hkv + kWarps - 1) / kWarps, std::max(1, 8 * c.num_sms / n));
    const dim3 grid(x, (unsigned)n);
    return c.dh == 64 ? launch_pdl(cache_bounds_kernel<64>, grid, dim3(kThreads), 0, st, c, layer, whole)
                      : launch_pdl(cache_bounds_kernel<128>, grid, dim3(kThreads), 0, st, c, layer, whole);
}

cudaError_t launch_cache_bounds_accepted(const CacheDev& c, int n, const int* seq, const int* n_acc, const int* accepted,
                                         cudaStream_t st) {
    return n <= 64 ? accepted_launch<64>(c, n, seq, n_acc, accepted, st)
                   : accepted_launch<kCacheMaxSeqs>(c, n, seq, n_acc, accepted, st);
}

cudaError_t launch_cache_select(const CacheDev& c, const SelectParams& p, cudaStream_t st, int& launches) {
    launches = 0;
    auto heads = [&](auto dh) {
        constexpr int DH = decltype(dh)::value;
        switch (columns_of(c.rep)) {
            case 1: return select_launch<DH, 1>(c, p, st, launches);
            case 2: return select_launch<DH, 2>(c, p, st, launches);
            case 4: return select_launch<DH, 4>(c, p, st, launches);
            default: return select_launch<DH, 8>(c, p, st, launches);
        }
    };
    return c.dh == 64 ? heads(std::integral_constant<int, 64>{}) : heads(std::integral_constant<int, 128>{});
}

}  // namespace tmoe
