// A step's queries, keys and values of one layer: RMSNorm of each query and key
// head, rotation, and the keys and values into their pages, in one pass.
//
//   y = x * (1 / sqrt(mean(x^2) + eps)) * gamma                (when gamma is given)
//   (y_i, y_{i + D/2}) -> (y_i cos a - y_{i+D/2} sin a, y_{i+D/2} cos a + y_i sin a),
//   a = pos * theta^(-2i/D),   one rounding to bf16;   v is copied.
//
// A head is held by D / 8 lanes, 8 elements (16 bytes) each; the lane half a head
// away has the rotation partners, which one shuffle of the packed input brings
// (the norm's factor is the head's own, so the partner's value needs no second
// exchange).  A warp takes one token, 4 heads at a time per lane group, and
// computes the token's angles once: the phase pos * (theta^(-2i/D) / 2 pi) is
// formed modulo one turn in 64-bit fixed point, exact to 2^-33 turns for any int32
// position, so no table is read and long positions lose nothing.
//
// Bound: HBM, (Hq + 2 Hkv) D 2 bytes read and written per token.  Small steps are
// latency: then a token's heads are spread over several warps (split).
#include <algorithm>

#include "cache.cuh"

namespace tmoe {

namespace {

constexpr int kAppendThreads = 256;
constexpr int kHeadsInFlight = 4;      // 16-byte loads in flight per lane

__device__ __forceinline__ void unpack(const uint4 v, float (&f)[8]) {
    f[0] = bf16_lo(v.x); f[1] = bf16_hi(v.x); f[2] = bf16_lo(v.y); f[3] = bf16_hi(v.y);
    f[4] = bf16_lo(v.z); f[5] = bf16_hi(v.z); f[6] = bf16_lo(v.w); f[7] = bf16_hi(v.w);
}

template <int DH>
__global__ void __launch_bounds__(kAppendThreads) cache_append_kernel(const __grid_constant__ CacheDev c,
                                                                      const __grid_constant__ AppendParams p) {
    constexpr int LANES = DH / 8;                    // lanes of a head
    constexpr int SIDE = 32 / LANES;                 // heads side by side in a warp
    __shared__ uint64_t turn[DH / 2];
    for (int i = threadIdx.x; i < DH / 2; i += kAppendThreads) turn[i] = p.turn[i];
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = lane % LANES, side = lane / LANES;
    const bool upper = sub >= LANES / 2;
    const int pair0 = (sub % (LANES / 2)) * 8;       // first of this lane's 8 rotation pairs
    const int mine = sub * 8, other = (sub ^ (LANES / 2)) * 8;
    const int H = c.Hq + 2 * c.Hkv;
    pdl_wait();
    pdl_trigger();
    const long long units = (long long)p.T * p.split;
    for (long long u = blockIdx.x * (kAppendThreads / 32) + warp; u < units;
         u += (long long)gridDim.x * (kAppendThreads / 32)) {
        const int t = (int)(u / p.split), part = (int)(u - (long long)t * p.split);
        const int slot = c.slot[t];
        if (slot < 0) continue;                      // the step was refused
        const int pos = p.pos ? p.pos[t] : c.pos[t];
        float cs[8], sn[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cs[j] = 1.f;
            sn[j] = 0.f;
        }
        if (p.rope) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // Signed fraction of a turn in [-1/2, 1/2), rounded to fp32.
                const int phase = (int)(uint32_t)(((uint64_t)(uint32_t)pos * turn[pair0 + j]) >> 32);
                sincospif((float)phase * 4.656612873077393e-10f, &sn[j], &cs[j]);   // 2^-31: half turns
                if (!upper) sn[j] = -sn[j];
            }
        }
        const __nv_bfloat16* src = p.qkv + (size_t)t * p.ld_qkv;
        const size_t page = (size_t)(slot >> c.page_shift) * c.Hkv, place = slot & (c.page - 1);
        for (int h0 = part * SIDE * kHeadsInFlight; h0 < H; h0 += p.split * SIDE * kHeadsInFlight) {
            uint4 in[kHeadsInFlight];
#pragma unroll
            for (int w = 0; w < kHeadsInFlight; ++w) {
                const int h = h0 + w * SIDE + side;
                in[w] = h < H ? *reinterpret_cast<const uint4*>(src + (size_t)h * DH + mine) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int w = 0; w < kHeadsInFlight; ++w) {
                const int hw = h0 + w * SIDE, h = hw + side;
                if (hw >= H) break;
                uint4 o = in[w];
                // The lanes of a warp may hold query, key and value heads together: the
                // shuffles run for all of them.
                if (hw < c.Hq + c.Hkv) {
                    uint4 y;
                    y.x = __shfl_xor_sync(0xffffffffu, o.x, LANES / 2);
                    y.y = __shfl_xor_sync(0xffffffffu, o.y, LANES / 2);
                    y.z = __shfl_xor_sync(0xffffffffu, o.z, LANES / 2);
                    y.w = __shfl_xor_sync(0xffffffffu, o.w, LANES / 2);
                    float a[8], b[8];
                    unpack(o, a);
                    unpack(y, b);
                    if (p.norm) {
                        float ss = 0.f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) ss = fmaf(a[j], a[j], ss);
#pragma unroll
                        for (int m = LANES / 2; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
                        const float rn = rsqrtf(ss * (1.f / DH) + p.eps);
                        const __nv_bfloat16* g = h < c.Hq ? p.gamma_q : p.gamma_k;
                        float ga[8], gb[8];
                        unpack(__ldg(reinterpret_cast<const uint4*>(g + mine)), ga);
                        unpack(__ldg(reinterpret_cast<const uint4*>(g + other)), gb);
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            a[j] = a[j] * rn * ga[j];
                            b[j] = b[j] * rn * gb[j];
                        }
                    }
                    if (h < c.Hq + c.Hkv) {
                        float r[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) r[j] = fmaf(a[j], cs[j], b[j] * sn[j]);
                        o = make_uint4(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]),
                                       pack_bf16x2(r[6], r[7]));
                    }
                }
                if (h >= H) continue;
                __nv_bfloat16* dst;
                if (h < c.Hq) {
                    dst = p.q_out + (size_t)t * p.ld_q + (size_t)h * DH;
                } else {
                    const int g = h - c.Hq < c.Hkv ? h - c.Hq : h - c.Hq - c.Hkv;
                    dst = (h < c.Hq + c.Hkv ? c.k : c.v) + p.layer_off + ((page + g) * c.page + place) * DH;
                }
                *reinterpret_cast<uint4*>(dst + mine) = o;
            }
        }
    }
}

}  // namespace

cudaError_t launch_cache_append(const CacheDev& c, const AppendParams& p0, cudaStream_t st) {
    AppendParams p = p0;
    const int H = c.Hq + 2 * c.Hkv, warps = kAppendThreads / 32, per = kHeadsInFlight * (256 / c.dh);
    // Warps per token: enough to fill the GPU once (about 32 warps per SM), at most
    // one per load batch of heads.
    const int most = (H + per - 1) / per;
    p.split = (int)std::max<long long>(1, std::min<long long>(most, (c.num_sms * 32LL + p.T - 1) / p.T));
    const long long units = (long long)p.T * p.split;
    const dim3 grid((unsigned)std::min<long long>((units + warps - 1) / warps, c.num_sms * 8LL));
    return c.dh == 64 ? launch_pdl(cache_append_kernel<64>, grid, dim3(kAppendThreads), 0, st, c, p)
                      : launch_pdl(cache_append_kernel<128>, grid, dim3(kAppendThreads), 0, st, c, p);
}

}  // namespace tmoe
