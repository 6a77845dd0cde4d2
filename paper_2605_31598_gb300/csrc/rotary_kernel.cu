// Rotary positions with several axes on q and k, and the transposed rotation
// (the gradient).
//
// Pair p of a head turns by theta = pos[axis[p]] * freq[p].  The angle enters
// as a fraction of a full turn in 64-bit fixed point: step[p] =
// round(freq[p] / 2 pi * 2^64), and pos * step mod 2^64 is the angle modulo one
// turn, exactly, for every int32 position (one 64-bit integer product; fp64
// runs at 1/60 of the fp32 rate here).  Its upper 32 bits, a signed multiple of
// 2^-31 half turns, go through sincospif, so no large argument is ever reduced
// in fp32.
//
// A CTA takes a token and forms its (cos, sin) pairs once, in shared memory.  A
// thread stays at one place of the head rows, eight pairs (two 16-byte loads), with
// their (cos, sin) in registers, and walks the heads; small CTAs, many to an SM, hide
// one another's steps.  12,544 tokens of 72 heads of 128: 70.8 us, 6.53 TB/s (86 us
// reading the pairs from shared memory for every head, 78 with 256 threads, 95 and
// more with several tokens to a CTA, whose registers leave too few CTAs).  Bound by
// HBM for long inputs and by the launch for short ones (8 tokens: 2.2 us).
#include "sm103_ptx.cuh"
#include "statekv_kernels.cuh"

namespace statekv {
namespace {


__device__ __forceinline__ float2 unit(const MropeParams& p, int token, int pair)
{
    const long long pos = p.positions[p.axis[pair] * p.position_stride + token];
    const unsigned long long turn = static_cast<unsigned long long>(pos) * p.step[pair];
    float sn, cs;
    sincospif(static_cast<float>(static_cast<int>(turn >> 32)) * 0x1p-31f, &sn, &cs);
    return make_float2(cs * p.scale, (p.transpose ? -sn : sn) * p.scale);
}

__device__ __forceinline__ float2 bf2(uint32_t w)
{
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w));
}

// Grid (tokens, slices of the heads).  An item is one place of a head row: VEC: eight
// pairs (adjacent: four), or eight copied elements; otherwise one pair, or one copied
// element.  Thread (place, lane of heads).
template <bool VEC, bool ADJ>
__global__ void __launch_bounds__(VEC ? 128 : 256) mrope_kernel(const __grid_constant__ MropeParams p, int places, int lanes)
{
    constexpr int kPairs = VEC ? (ADJ ? 4 : 8) : 1;  // pairs of a rotated item
    __shared__ float2 table[kMropeMaxPairs];
    const long long token = blockIdx.x;
    const int P = p.pairs, d = p.d;
    const int place = threadIdx.x % places, lane = threadIdx.x / places;
    const int rot = P / kPairs;                      // rotated places, then copied ones
    const int heads = p.t[0].heads + p.t[1].heads, step = lanes * gridDim.y;
    const int h0 = blockIdx.y * lanes + lane;
    const bool mine = lane < lanes;

    // element offsets of an item in its head row
    const int a = place < rot ? place * kPairs * (ADJ ? 2 : 1) : 2 * P + (place - rot) * (VEC ? 8 : 1);
    const int b = ADJ ? a + 1 : a + P;               // !VEC, or the half layout: the pairs' other elements
    uint4 xa, xb;
    auto read = [&](int h) {
        const int w = h >= p.t[0].heads;
        const __nv_bfloat16* s = p.t[w].x + token * p.t[w].stride + static_cast<long long>(h - (w ? p.t[0].heads : 0)) * d;
        if constexpr (VEC) {
            xa = __ldcs(reinterpret_cast<const uint4*>(s + a));
            if (!ADJ && place < rot) xb = __ldcs(reinterpret_cast<const uint4*>(s + b));
        } else {
            xa.x = __bfloat16_as_ushort(s[a]);
            if (place < rot) xb.x = __bfloat16_as_ushort(s[b]);
        }
    };
    if (mine && h0 < heads) read(h0);  // on their way while the pairs are formed
    for (int i = threadIdx.x; i < P; i += blockDim.x) table[i] = unit(p, blockIdx.x, i);
    __syncthreads();
    if (!mine) return;
    float2 cs[kPairs];
    if (place < rot) {
#pragma unroll
        for (int j = 0; j < kPairs; ++j) cs[j] = table[place * kPairs + j];
    }
    for (int h = h0; h < heads; h += step) {
        if (h != h0) read(h);
        const int w = h >= p.t[0].heads;
        __nv_bfloat16* y = p.t[w].y + token * p.t[w].out_stride + static_cast<long long>(h - (w ? p.t[0].heads : 0)) * d;
        if (place >= rot) {
            if constexpr (VEC) __stcs(reinterpret_cast<uint4*>(y + a), xa);
            else y[a] = __ushort_as_bfloat16(static_cast<unsigned short>(xa.x));
        } else if constexpr (!VEC) {
            const float fa = __uint_as_float(xa.x << 16), fb = __uint_as_float(xb.x << 16);
            y[a] = __float2bfloat16(fa * cs[0].x - fb * cs[0].y);
            y[b] = __float2bfloat16(fb * cs[0].x + fa * cs[0].y);
        } else if constexpr (ADJ) {
            uint32_t r[4] = {xa.x, xa.y, xa.z, xa.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 f = bf2(r[j]);
                r[j] = ptx::pack_bf16x2(f.x * cs[j].x - f.y * cs[j].y, f.y * cs[j].x + f.x * cs[j].y);
            }
            __stcs(reinterpret_cast<uint4*>(y + a), make_uint4(r[0], r[1], r[2], r[3]));
        } else {
            uint32_t ra[4] = {xa.x, xa.y, xa.z, xa.w}, rb[4] = {xb.x, xb.y, xb.z, xb.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 fa = bf2(ra[j]), fb = bf2(rb[j]), c0 = cs[2 * j], c1 = cs[2 * j + 1];
                ra[j] = ptx::pack_bf16x2(fa.x * c0.x - fb.x * c0.y, fa.y * c1.x - fb.y * c1.y);
                rb[j] = ptx::pack_bf16x2(fb.x * c0.x + fa.x * c0.y, fb.y * c1.x + fa.y * c1.y);
            }
            __stcs(reinterpret_cast<uint4*>(y + a), make_uint4(ra[0], ra[1], ra[2], ra[3]));
            __stcs(reinterpret_cast<uint4*>(y + b), make_uint4(rb[0], rb[1], rb[2], rb[3]));
        }
    }
}

}  // namespace

cudaError_t launch_mrope(const MropeParams& p, cudaStream_t st)
{
    const int heads = p.t[0].heads + p.t[1].heads;
    if (p.tokens <= 0 || heads <= 0) return cudaSuccess;
    const bool vec = p.adjacent ? p.pairs % 4 == 0 : p.pairs % 8 == 0;
    const int places = vec ? (p.adjacent ? p.pairs / 4 : p.pairs / 8) + (p.d - 2 * p.pairs) / 8
                           : p.pairs + p.d - 2 * p.pairs;  // at most 256
    const int threads = vec ? 128 : 256, lanes = threads / places;
    // a CTA walks all of its token's heads once the tokens alone give every SM 16 CTAs; below
    // that the heads are cut into slices of one item per thread
    const bool walk = static_cast<long long>(p.tokens) >= 16ll * current_sm_count();
    const dim3 grid(p.tokens, walk ? 1 : (heads + lanes - 1) / lanes);
    if (vec && p.adjacent) mrope_kernel<true, true><<<grid, threads, 0, st>>>(p, places, lanes);
    else if (vec) mrope_kernel<true, false><<<grid, threads, 0, st>>>(p, places, lanes);
    else if (p.adjacent) mrope_kernel<false, true><<<grid, threads, 0, st>>>(p, places, lanes);
    else mrope_kernel<false, false><<<grid, threads, 0, st>>>(p, places, lanes);
    return cudaGetLastError();
}

}  // namespace statekv
