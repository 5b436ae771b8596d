// A step's queries, keys and values of one layer: RMSNorm of each query and key
// head, rotation, and the keys and values into their pages, in one pass.
//
//   y = x * (1 / sqrt(mean(x^2) + eps)) * gamma                (when gamma is given)
//   (y_i, y_{i + D/2}) -> (y_i cos a - y_{i+D/2} sin a, y_{i+D/2} cos a + y_i sin a),
//   a = pos * theta^(-2i/D),   one rounding to bf16;   v is copied.
//
// A head is held by D / 8 lanes, each with 4 elements of the lower half and the 4 that
// they rotate with, so that only the sum of squares crosses lanes.  A warp takes one
// token and one or more batches of heads (4 per lane group, all queries, all keys or
// all values); gamma and the rotation are multiplied once per token and kind of head,
// after which an element costs three operations.  The phase pos * (theta^(-2i/D) / 2 pi)
// is formed modulo one turn in 64-bit fixed point, from the turns per position in double:
// off by at most 2^-32 + pos 2^-55 turns for a position >= 0 (2^-25 at 2^30), so no table
// is read and long positions lose nothing that bf16 shows; sine and cosine of
// the remainder are the hardware's (off by at most 2^-20 of the pair, bf16 rounds at 2^-8).
//
// Bound: HBM, (Hq + 2 Hkv) D 2 bytes read and written per token; a small step is bound
// by latency, and its tokens' batches go to different warps.  Measured (32 query heads on 8,
// D = 128, pages of 64): 16384 tokens 61.6 us, 6.2 TB/s, 0.92 of the copy rate; 113 tokens
// 2.8 us on the GPU.
#include <algorithm>

#include "cache.cuh"

namespace tmoe {

namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendBlocks = 4;       // blocks per SM
constexpr int kHeadsInFlight = 4;      // heads that a lane loads at a time

template <int DH>
__global__ void __launch_bounds__(kAppendThreads, kAppendBlocks)
cache_append_kernel(const __grid_constant__ CacheDev c, const __grid_constant__ AppendParams p) {
    constexpr int LANES = DH / 8;                    // lanes of a head
    constexpr int SIDE = 32 / LANES;                 // heads side by side in a warp
    constexpr int BATCH = SIDE * kHeadsInFlight;
    __shared__ uint64_t turn[DH / 2];
    for (int i = threadIdx.x; i < DH / 2; i += kAppendThreads) turn[i] = p.turn[i];
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = lane % LANES, side = lane / LANES;
    const int e0 = sub * 4;                          // this lane's first pair: elements e0 + j and DH / 2 + e0 + j
    const int nq = (c.Hq + BATCH - 1) / BATCH, nk = (c.Hkv + BATCH - 1) / BATCH;
    pdl_wait();
    pdl_trigger();
    const long long units = (long long)p.T * p.split;
    for (long long u = blockIdx.x * (kAppendThreads / 32) + warp; u < units;
         u += (long long)gridDim.x * (kAppendThreads / 32)) {
        const int t = (int)(u / p.split), part = (int)(u - (long long)t * p.split);
        const int slot = c.slot[t];
        if (slot < 0) continue;                      // the step was refused
        const int pos = p.pos ? p.pos[t] : c.pos[t];
        const __nv_bfloat16* src = p.qkv + (size_t)t * p.ld_qkv;
        const size_t page = (size_t)(slot >> c.page_shift) * c.Hkv, place = slot & (c.page - 1);
        float ac[4], bs[4], bc[4], as[4];            // gamma times cosine and sine, lower (a) and upper (b) half
        int kind_at = -1;
        for (int b = part; b < nq + 2 * nk; b += p.split) {
            const int kind = b < nq ? 0 : b < nq + nk ? 1 : 2;             // queries, keys, values
            const int H = kind == 0 ? c.Hq : c.Hkv, h0 = (b - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk)) * BATCH + side;
            const __nv_bfloat16* from = src + (size_t)(kind == 0 ? 0 : kind == 1 ? c.Hq : c.Hq + c.Hkv) * DH + e0;
            uint2 lo[kHeadsInFlight], hi[kHeadsInFlight];
#pragma unroll
            for (int w = 0; w < kHeadsInFlight; ++w) {
                const int h = min(h0 + w * SIDE, H - 1);
                lo[w] = *reinterpret_cast<const uint2*>(from + (size_t)h * DH);
                hi[w] = *reinterpret_cast<const uint2*>(from + (size_t)h * DH + DH / 2);
            }
            __nv_bfloat16* to = kind == 0 ? p.q_out + (size_t)t * p.ld_q + e0
                                          : (kind == 1 ? c.k : c.v) + p.layer_off + (page * c.page + place) * DH + e0;
            const size_t step = kind == 0 ? DH : (size_t)c.page * DH;      // from head to head
            if (kind < 2 && kind != kind_at) {
                kind_at = kind;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float sn = 0.f, cs = 1.f;
                    if (p.rope) {
                        // Signed fraction of a turn in [-1/2, 1/2), as an angle.
                        const int phase = (int)(uint32_t)(((uint64_t)(uint32_t)pos * turn[e0 + j]) >> 32);
                        __sincosf((float)phase * 1.4629180792671596e-9f, &sn, &cs);   // 2 pi / 2^32
                    }
                    ac[j] = bc[j] = cs;
                    as[j] = bs[j] = sn;
                }
                if (p.norm) {
                    const __nv_bfloat16* g = kind == 0 ? p.gamma_q : p.gamma_k;
                    const uint2 ga = __ldg(reinterpret_cast<const uint2*>(g + e0));
                    const uint2 gb = __ldg(reinterpret_cast<const uint2*>(g + e0 + DH / 2));
                    const float fa[4] = {bf16_lo(ga.x), bf16_hi(ga.x), bf16_lo(ga.y), bf16_hi(ga.y)};
                    const float fb[4] = {bf16_lo(gb.x), bf16_hi(gb.x), bf16_lo(gb.y), bf16_hi(gb.y)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        ac[j] *= fa[j];
                        as[j] *= fa[j];
                        bc[j] *= fb[j];
                        bs[j] *= fb[j];
                    }
                }
            }
#pragma unroll
            for (int w = 0; w < kHeadsInFlight; ++w) {
                const int h = h0 + w * SIDE;
                if (kind < 2) {
                    float x[4] = {bf16_lo(lo[w].x), bf16_hi(lo[w].x), bf16_lo(lo[w].y), bf16_hi(lo[w].y)};
                    float y[4] = {bf16_lo(hi[w].x), bf16_hi(hi[w].x), bf16_lo(hi[w].y), bf16_hi(hi[w].y)};
                    if (p.norm) {
                        float ss = 0.f;
#pragma unroll
                        for (int j = 0; j < 4; ++j) ss = fmaf(x[j], x[j], fmaf(y[j], y[j], ss));
#pragma unroll
                        for (int m = LANES / 2; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
                        const float rn = rsqrtf(ss * (1.f / DH) + p.eps);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            x[j] *= rn;
                            y[j] *= rn;
                        }
                    }
                    float a[4], d[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // (without rotation a factor 0 would still make NaN of an infinity)
                        a[j] = p.rope ? fmaf(x[j], ac[j], -y[j] * bs[j]) : x[j] * ac[j];
                        d[j] = p.rope ? fmaf(y[j], bc[j], x[j] * as[j]) : y[j] * bc[j];
                    }
                    lo[w] = make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]));
                    hi[w] = make_uint2(pack_bf16x2(d[0], d[1]), pack_bf16x2(d[2], d[3]));
                }
                if (h < H) {
                    *reinterpret_cast<uint2*>(to + h * step) = lo[w];
                    *reinterpret_cast<uint2*>(to + h * step + DH / 2) = hi[w];
                }
            }
        }
    }
}

}  // namespace

cudaError_t launch_cache_append(const CacheDev& c, const AppendParams& p0, cudaStream_t st) {
    AppendParams p = p0;
    const int warps = kAppendThreads / 32, batch = kHeadsInFlight * (256 / c.dh);
    // Warps per token: eight units of work for every resident warp, so that the last ones
    // end together, at most one warp per batch of heads.
    const int most = (c.Hq + batch - 1) / batch + 2 * ((c.Hkv + batch - 1) / batch);
    const long long resident = (long long)c.num_sms * kAppendBlocks * warps;
    p.split = (int)std::max<long long>(1, std::min<long long>(most, (8 * resident + p.T - 1) / p.T));
    const long long units = (long long)p.T * p.split;
    const dim3 grid((unsigned)std::min<long long>((units + warps - 1) / warps, c.num_sms * kAppendBlocks));
    return c.dh == 64 ? launch_pdl(cache_append_kernel<64>, grid, dim3(kAppendThreads), 0, st, c, p)
                      : launch_pdl(cache_append_kernel<128>, grid, dim3(kAppendThreads), 0, st, c, p);
}

}  // namespace tmoe
