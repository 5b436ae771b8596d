// Choice of the pages that a query reads: bounds of the keys of whole pages ("blocks"), and
// for each token and key/value head the blocks whose bounds promise the largest scores.
//
//   lo_d = min_i k_id, hi_d = max_i k_id over a page's keys, held as floor(lo / u) and
//   ceil(hi / u) in 8 bits; u = 2^e, e the least one with max(|lo|, |hi|) <= 127 u
//   score = u max_h u_h sum_d max(c_hd lo_d, c_hd hi_d),  c_h = rint(q_h / u_h)
//
// With q+ = max(c, 0) and q- = min(c, 0) the sum is q+ . hi + q- . lo, two dot products of
// 8-bit numbers.  It is at most 128 * 127 * 127 < 2^24, so that every score is exact in fp32
// and the order of the blocks (ties: the lower one) does not depend on how it is computed.
#include <algorithm>

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

// Bound: HBM, each filled page's keys once (9 prompts, 16384 tokens, 32 MB); a decode step
// fills few pages and is bound by latency.
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

__host__ __device__ inline size_t select_smem(const CacheDev& c) {
    return (((size_t)c.max_pages * 4 + 15) & ~size_t(15)) + (size_t)c.rep * c.dh * 2;
}

// A block takes one token and key/value head: its query heads as 8-bit codes in shared
// memory, the blocks' scores (four lanes to a block), the n-th largest of them by four
// counting passes over its digits, and the columns at or above it in order.
template <int DH>
__global__ void __launch_bounds__(kThreads) cache_select_kernel(const __grid_constant__ CacheDev c,
                                                                const __grid_constant__ SelectParams p) {
    constexpr int K = DH / 64, G = 2;                 // 16-byte pieces of a lane, blocks in flight of a lane
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ float s_unit[128];
    __shared__ int s_hist[256], s_digit, s_left, s_all, s_gt[kWarps], s_eq[kWarps];
    uint32_t* key = smem;
    int8_t* s_pos = reinterpret_cast<int8_t*>(smem) + (((size_t)c.max_pages * 4 + 15) & ~size_t(15));
    int8_t* s_neg = s_pos + c.rep * DH;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t = blockIdx.x / c.Hkv, h = blockIdx.x - t * c.Hkv, n = p.n;
    pdl_wait();
    pdl_trigger();
    if (!c.plan->ok) return;
    const CacheSeq s = c.seqs[c.owner[t]];
    const int F = (s.kv_len - s.q_len) >> c.page_shift;
    int* out = p.blocks + ((size_t)t * c.Hkv + h) * n;
    if (F <= n) {
        for (int i = threadIdx.x; i < n; i += kThreads) out[i] = i < F ? i : -1;
        return;
    }
    for (int r = warp; r < c.rep; r += kWarps) {
        const __nv_bfloat16* q = p.q + (size_t)t * p.ld_q + (size_t)(h * c.rep + r) * DH + lane * 2 * K;
        uint32_t w[K], amax = 0;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            w[j] = reinterpret_cast<const uint32_t*>(q)[j];
            const uint32_t a = w[j] & 0x7fff7fffu;
            amax = max(amax, max(a << 16, a & 0xffff0000u));
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
        const bool finite = amax < 0x7f800000u;
        const int e = unit_exponent(__uint_as_float(amax));
        const float inv = finite ? two_to(-e) : 0.f;
        uint16_t* pos = reinterpret_cast<uint16_t*>(s_pos + r * DH) + lane * K;
        uint16_t* neg = reinterpret_cast<uint16_t*>(s_neg + r * DH) + lane * K;
#pragma unroll
        for (int j = 0; j < K; ++j) {
            const int a = finite ? __float2int_rn(bf16_lo(w[j]) * inv) : 0, b = finite ? __float2int_rn(bf16_hi(w[j]) * inv) : 0;
            pos[j] = (uint16_t)(max(a, 0) | max(b, 0) << 8);
            neg[j] = (uint16_t)((min(a, 0) & 0xff) | (min(b, 0) & 0xff) << 8);
        }
        if (lane == 0) s_unit[r] = finite ? two_to(e) : 0.f;
    }
    __syncthreads();
    // Lane 4 b + i holds bytes 16 i .. 16 i + 15 (and 64 more) of block b's lo and hi.
    const int part = lane & 3;
    const int* row = c.table + (size_t)s.seq * c.max_pages;
    const size_t layer = (size_t)p.layer * c.n_pages;
    for (int b0 = warp * 8 * G; b0 < F; b0 += kWarps * 8 * G) {
        int4 lo[G][K], hi[G][K];
        float scale[G], best[G];
        bool there[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int b = b0 + g * 8 + (lane >> 2), id = row[min(b, F - 1)];
            there[g] = id >= 0 && id < c.n_pages;
            const size_t unit = (layer + (there[g] ? id : 0)) * c.Hkv + h;
            const int4* src = reinterpret_cast<const int4*>(c.codes + unit * 2 * DH) + part;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                lo[g][k] = __ldg(src + 4 * k);
                hi[g][k] = __ldg(src + DH / 16 + 4 * k);
            }
            scale[g] = __ldg(c.scales + unit);
            best[g] = -INFINITY;
        }
        for (int r = 0; r < c.rep; ++r) {
            const float u = s_unit[r];
            int4 qp[K], qn[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                qp[k] = reinterpret_cast<const int4*>(s_pos + r * DH)[4 * k + part];
                qn[k] = reinterpret_cast<const int4*>(s_neg + r * DH)[4 * k + part];
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                int sum = 0;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    sum = __dp4a(qp[k].x, hi[g][k].x, sum);
                    sum = __dp4a(qn[k].x, lo[g][k].x, sum);
                    sum = __dp4a(qp[k].y, hi[g][k].y, sum);
                    sum = __dp4a(qn[k].y, lo[g][k].y, sum);
                    sum = __dp4a(qp[k].z, hi[g][k].z, sum);
                    sum = __dp4a(qn[k].z, lo[g][k].z, sum);
                    sum = __dp4a(qp[k].w, hi[g][k].w, sum);
                    sum = __dp4a(qn[k].w, lo[g][k].w, sum);
                }
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                best[g] = fmaxf(best[g], (float)sum * u);
            }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int b = b0 + g * 8 + (lane >> 2);
            if (part == 0 && b < F) {
                // (A page without an index scores nothing; + 0 turns -0 into 0.)
                const float x = scale[g] == INFINITY ? INFINITY : best[g] * scale[g] + 0.f;
                key[b] = b < p.first || b >= F - p.last ? 0xffffffffu : there[g] ? ordered(x) : 0u;
                if (!there[g]) atomicCAS(c.err, 0, ERR_CACHE_STATE);
            }
        }
    }
    // The n-th largest key: digit by digit from the top, `left` of the keys that agree so far
    // are still wanted.
    uint32_t prefix = 0, mask = 0;
    int left = n;
    bool all = false;                                 // all that agree with the digits so far are wanted
    for (int shift = 24; shift >= 0 && !all; shift -= 8) {
        s_hist[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < F; i += kThreads)
            if ((key[i] & mask) == prefix) atomicAdd(&s_hist[key[i] >> shift & 255u], 1);
        __syncthreads();
        if (warp == 0) {
            int mine[8], sum = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += mine[j] = s_hist[255 - lane * 8 - j];
            int below = sum;                          // of this lane's digits and all larger ones
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, below, o);
                if (lane >= o) below += y;
            }
            int before = below - sum;
            if (before < left && below >= left) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (before < left && before + mine[j] >= left) {
                        s_digit = 255 - lane * 8 - j;
                        s_left = left - before;
                        s_all = mine[j] == left - before;
                    }
                    before += mine[j];
                }
            }
        }
        __syncthreads();
        prefix |= (uint32_t)s_digit << shift;
        mask |= 255u << shift;
        left = s_left;
        all = s_all;
        __syncthreads();
    }
    // Keys above the prefix are taken, of those that agree with it the first `left`.
    const int per = ((F + kThreads - 1) / kThreads) * 32, i0 = warp * per, i1 = min(F, i0 + per);
    int gt = 0, eq = 0;
    for (int i = i0 + lane; i - lane < i1; i += 32) {
        const uint32_t k = i < i1 ? key[i] & mask : 0u;
        gt += __popc(__ballot_sync(0xffffffffu, i < i1 && k > prefix));
        eq += __popc(__ballot_sync(0xffffffffu, i < i1 && k == prefix));
    }
    if (lane == 0) {
        s_gt[warp] = gt;
        s_eq[warp] = eq;
    }
    __syncthreads();
    gt = eq = 0;
    for (int w = 0; w < warp; ++w) {
        gt += s_gt[w];
        eq += s_eq[w];
    }
    const uint32_t below = (1u << lane) - 1u;
    for (int i = i0 + lane; i - lane < i1; i += 32) {
        const uint32_t k = i < i1 ? key[i] & mask : 0u;
        const bool more = i < i1 && k > prefix, same = i < i1 && k == prefix;
        const uint32_t mg = __ballot_sync(0xffffffffu, more), me = __ballot_sync(0xffffffffu, same);
        const int g = gt + __popc(mg & below), e = eq + __popc(me & below);
        if (more || (same && e < left)) out[g + min(e, left)] = i;
        gt += __popc(mg);
        eq += __popc(me);
    }
}

template <int DH>
cudaError_t select_launch(const CacheDev& c, const SelectParams& p, cudaStream_t st) {
    static PerDevice attr;
    const cudaError_t e = (cudaError_t)attr.get([] {
        return (int)cudaFuncSetAttribute(cache_select_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
    }, true);
    if (e != cudaSuccess) return e;
    return launch_pdl(cache_select_kernel<DH>, dim3((unsigned)(p.T * c.Hkv)), dim3(kThreads), select_smem(c), st, c, p);
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

cudaError_t launch_cache_select(const CacheDev& c, const SelectParams& p, cudaStream_t st) {
    return c.dh == 64 ? select_launch<64>(c, p, st) : select_launch<128>(c, p, st);
}

}  // namespace tmoe
