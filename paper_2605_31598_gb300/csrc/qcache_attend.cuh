// What the two attention kernels over the 8-bit cache share: the visible rows of
// a unit, the line of all tiles' steps that the persistent CTAs cut into equal
// shares, bounded waits and the stores of a finished row.
#pragma once

#include <cuda_fp16.h>

#include "sm103_ptx.cuh"
#include "statekv_kernels.cuh"

namespace statekv {
namespace qc {

using namespace ptx;

constexpr float kRefBias = 6.f;    // a weight at the reference is 2^6
constexpr float kRefSlack = 8.f;   // the reference may trail the maximum by 2^8

__device__ __forceinline__ unsigned long long now_ns()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Bounded wait for an mbarrier phase.
__device__ __forceinline__ bool wait_full(uint64_t* bar, uint32_t parity, unsigned long long limit_ns)
{
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = now_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        if (now_ns() - t0 > limit_ns) return false;
    }
}

// Debug builds can have a call's first CTA take one wait as run out, in the odd lanes of
// each warp that comes by `there` (QAttendParams::expire).
__device__ __forceinline__ bool expire_here(const QAttendParams& p, bool there)
{
#if STATEKV_DEBUG_CHECKS
    return p.expire && there && blockIdx.x == 0 && (threadIdx.x & 1);
#else
    return false;
#endif
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// four e4m3 codes -> four fp16
__device__ __forceinline__ void f16_of(uint32_t codes, uint32_t& lo, uint32_t& hi)
{
    asm("{\n\t.reg .b16 a, b;\n\t"
        "mov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(codes));
}

// two fp32 values -> two e4m3 codes, the first in the low byte (beyond 448: 448)
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ void tma_load_3d(void* dst, const void* tmap, uint64_t* bar, int c0, int c1, int c2)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_addr(dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(smem_addr(bar)), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}

// Byte offset of byte `byte` of key row `key` in a tile of swizzled rows of D
// bytes (D = 64: two keys to a 128-byte row).
template <int D>
__device__ __forceinline__ uint32_t at(int key, int byte)
{
    const uint32_t lin = key * D + byte;
    return lin ^ ((lin >> 3) & 0x70u);
}

// What the rows of a call see of a unit's cache.  Row positions are below 2^31.
struct Span {
    int first, start, stop;  // visible rows begin at first; rows before the call; rows held
};

__device__ __forceinline__ Span span_of(const QAttendParams& p, int ua)
{
    Span s;
    s.start = p.start[ua];
    s.first = p.first ? max(0, p.first[ua]) : 0;
    s.stop = s.start + p.n;
    if (s.start < 0 || s.start > p.c.cap - p.n) {
        if (s.start >= 0) *reinterpret_cast<volatile int32_t*>(p.c.status) = DEV_QCACHE_FULL;
        s.first = s.start = s.stop = 0;  // nothing is visible
    }
    return s;
}

// Steps of KEYS keys from the first visible key's to `end`.
template <int KEYS>
__device__ __forceinline__ int steps_to(const Span& s, int end)
{
    return end > s.first ? (end - 1) / KEYS - s.first / KEYS + 1 : 0;
}

// How the persistent CTAs divide the tiles (unit, KV head, row tile) and their steps.
//   Few tiles: each is cut into shares of `share` steps, a CTA each, so no CTA works
//     on two tiles.
//   Many: every tile takes `cost` places for its fixed work and one for each step on
//     a line, of which CTA c has the places from c share to (c + 1) share; units of
//     any lengths load every SM alike.
// A tile of a unit without visible keys belongs to the CTA with its first place.
// The host keeps the line below 2^31 places.
struct Line {
    const uint32_t* prefix;  // [U + 1] first place (few tiles: first CTA) of each unit, in shared memory
    const int4* units;       // [U] first, start, stop, steps
    uint32_t total, share;
    int U, cost;
    bool few;

    __device__ Span span(int u) const { return Span{units[u].x, units[u].y, units[u].z}; }
};

// A CTA's share of a tile: steps [sa, sb) of the unit's `steps`; the CTAs ca .. cb
// have some of it.
struct Segment {
    int u, tile, sa, sb, steps, ca, cb;
};

constexpr int line_bytes(int units) { return units * 16 + (units + 1) * 4; }

// Sums each unit's `weight(steps)` for each of its tiles into prefix[].  All THREADS
// threads; `scratch` holds a word for each warp.
template <int THREADS, typename F>
__device__ __forceinline__ uint32_t sum_units(int U, uint32_t tiles, const int4* units, uint32_t* prefix, uint32_t* scratch,
                                              F weight)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) prefix[0] = 0;
    uint32_t carry = 0;
    for (int u0 = 0; u0 < U; u0 += THREADS) {
        const int u = u0 + threadIdx.x;
        uint32_t w = u < U ? tiles * weight(units[u].w) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += x;
        }
        if (lane == 31) scratch[warp] = w;
        __syncthreads();
        uint32_t before = carry;
#pragma unroll
        for (int i = 0; i < THREADS / 32; ++i) {
            const uint32_t x = scratch[i];
            if (i < warp) before += x;
            carry += x;
        }
        if (u < U) prefix[u + 1] = before + w;
        __syncthreads();
    }
    return carry;
}

// `least`: steps of a share that are worth a CTA and the join.
template <int THREADS, int KEYS>
__device__ __forceinline__ Line make_line(const QAttendParams& p, uint8_t* smem, uint32_t* scratch, int cost, int least)
{
    int4* units = reinterpret_cast<int4*>(smem);
    uint32_t* prefix = reinterpret_cast<uint32_t*>(units + kQCacheUnits);
    const uint32_t tiles = static_cast<uint32_t>(p.c.Hkv * p.row_tiles), N = gridDim.x;
    for (int u = threadIdx.x; u < p.U; u += THREADS) {  // read back by the same thread
        const Span s = span_of(p, p.units.unit_abs(u));
        units[u] = make_int4(s.first, s.start, s.stop, steps_to<KEYS>(s, s.stop));
    }
    Line ln;
    ln.prefix = prefix;
    ln.units = units;
    ln.U = p.U;
    ln.cost = cost;
    ln.total = sum_units<THREADS>(p.U, tiles, units, prefix, scratch,
                                  [&](int steps) { return static_cast<uint32_t>(steps + cost); });
    ln.share = max(static_cast<uint32_t>(least + cost), (ln.total + N - 1) / N);
    // shares of whole tiles: ceil(steps / s) of each come to at most steps / s + tiles
    const unsigned long long T = static_cast<unsigned long long>(tiles) * p.U;
    ln.few = false;
    if (T < N) {
        const uint32_t steps = ln.total - static_cast<uint32_t>(T) * cost, room = N - static_cast<uint32_t>(T);
        const uint32_t s = max(static_cast<uint32_t>(least), (steps + room - 1) / room);
        // (a segment's end costs the narrow kernel about a tenth of a typical share)
        if (10 * s <= (KEYS == 32 ? 11 : 10) * ln.share) {
            ln.few = true;
            ln.share = s;
            ln.total = sum_units<THREADS>(p.U, tiles, units, prefix, scratch,
                                          [&](int n) { return max(1u, (static_cast<uint32_t>(n) + s - 1) / s); });
        }
    }
    return ln;
}

// The segments of one CTA's share, in order.
struct Walk {
    uint32_t place, stop_at;
    int u;

    __device__ Walk(const Line& ln, int cta)
    {
        // clipped to the line: a CTA beyond it has none
        const uint32_t each = ln.few ? 1 : ln.share;
        place = static_cast<uint32_t>(min(static_cast<unsigned long long>(cta) * each, static_cast<unsigned long long>(ln.total)));
        stop_at = ln.total - place < each ? ln.total : place + each;
        int lo = 0, hi = ln.U;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (ln.prefix[mid] <= place) lo = mid;
            else hi = mid;
        }
        u = lo;
    }

    __device__ bool next(const Line& ln, Segment& s)
    {
        while (place < stop_at) {
            while (place >= ln.prefix[u + 1]) ++u;
            const int steps = ln.units[u].w;
            const uint32_t from = ln.prefix[u];
            s.u = u;
            s.steps = steps;
            if (ln.few) {
                const uint32_t shares = max(1u, (static_cast<uint32_t>(steps) + ln.share - 1) / ln.share);
                const uint32_t tile = (place - from) / shares, i = place - from - tile * shares;
                s.tile = static_cast<int>(tile);
                s.sa = static_cast<int>(i * ln.share);
                s.sb = min(steps, static_cast<int>((i + 1) * ln.share));
                s.ca = static_cast<int>(place - i);
                s.cb = s.ca + static_cast<int>(shares) - 1;
                ++place;
                return true;
            }
            const uint32_t each = static_cast<uint32_t>(steps + ln.cost);
            const uint32_t tile = (place - from) / each;
            const uint32_t base = from + tile * each;
            const uint32_t zone = base + ln.cost;  // places of the steps
            s.tile = static_cast<int>(tile);
            s.sa = place > zone ? static_cast<int>(place - zone) : 0;
            s.sb = stop_at >= zone + steps ? steps : stop_at > zone ? static_cast<int>(stop_at - zone) : 0;
            const bool empty = steps == 0 && place == base;
            place = zone + steps;
            if (s.sa < s.sb || empty) {
                s.ca = steps ? static_cast<int>(zone / ln.share) : 0;
                s.cb = steps ? static_cast<int>((zone + steps - 1) / ln.share) : 0;
                return true;
            }
        }
        return false;
    }
};

// Where query row r of KV head hkv of the call's unit u lies in q and out, in rows.
__device__ __forceinline__ size_t row_of(const QAttendParams& p, int u, int hkv, int r)
{
    const int t = r / p.G, gg = r - t * p.G;
    return (static_cast<size_t>(u) * p.n + t) * p.Hq + hkv * p.G + gg;
}

__device__ __forceinline__ float lse_of(float ref, float sum)
{
    return sum == 0.f ? -INFINITY : 0.6931471805599453f * (ref - kRefBias + log2f(sum));
}

}  // namespace qc
}  // namespace statekv
