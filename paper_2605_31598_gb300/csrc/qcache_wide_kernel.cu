// Attention over the cache held in 8 bits for many query rows (prompts).
//
// The same sums as qcache_attend_kernel.cu, on tcgen05.  A tile is 256 of the
// n * G query rows of a KV head of a unit, as two halves of 128, against the keys
// that its rows see in steps of 128; persistent CTAs take equal shares of all
// tiles' steps.
//
// Per step the codes of 128 K rows and 128 V rows arrive by TMA (16 KB each, D =
// 128), and both halves use them.
//   S = Q K^T  D = 128: on the codes as they are (kind::f8f6f4).  A row of
//     queries is scaled by the power of two that brings its largest element into [2^7,
//     2^8).  A bf16 element is then the sum of an e4m3 number, its first four significant
//     bits, and an e5m2 number, the rest: at most eight units of its last place, which
//     three bits hold.  Exactly so down to 2^-13 of the row's largest, where the first
//     part gets coarse; below, the sum is within 2^-21 of the largest (2^-17 if the rest
//     were e4m3 too).  Two products at twice the fp16 rate.  D = 64 (two keys to a
//     128-byte row): K codes are turned into fp16 like V's.
//   O += P V  P over S in TMEM; V's codes are turned into fp16 tiles in shared
//     memory by four converter warps.
// Shared memory bounds the step: the products read 192 KB of operands for both
// halves, and what the converters would move for K is another 48 KB (with it a step
// took 4,150 cycles, now 3,620).
// Measured: 1,000 tokens of 28 query and 4 KV heads behind 31,360 keys, D = 128: 414
// us, 1.10 PFLOP/s, 58% of the bf16 rate, where one key in twenty is three times the
// others (rows set their references again); 374 us, 64%, on keys of one size.  D = 64:
// 366 and 353 us.
// TMEM: S0 | S1 | O0 | O1, 128 columns each.  Each half has an issuer that runs
// PV(j), QK(j + 1), and the halves take turns: while one half's softmax works, the
// tensor core has the other half's two products.  Q K^T into a half's scores
// follows the P V that read its weights there; one thread issues both, in order.  A
// wait costs the tensor core more than an MMA, so an issuer waits once per step: on
// a barrier that takes the weights, the step's V tile and the next step's K tile.
//
// 512 threads, four warpgroups:
//   WG0  warp 0 TMA producer, warps 1 and 3 MMA issuers of half 0 and 1 (warp 1
//        owns TMEM)
//   WG1  converters, a key row per thread
//   WG2, WG3  softmax of half 0 and 1, a query row per thread
// Softmax and precision: weights 2^(s - ref), fp32, rounded to fp16 for P V.  A
// row's reference is its maximum when it was last set, with weight 2^6, and is set
// again when a step's weights sum to more than 2^15, so the maximum of a step is
// only looked for then.  O is held in units of a V scale that follows the blocks';
// the converters multiply a V row by its scale's ratio to that unit, 2^-6 to 1
// (exact in fp16 for the power-of-two scales of an append).  Moving the reference
// or the unit rescales O in TMEM, after the step's Q K^T has completed (and with
// it the P V before it).
// A CTA's share of a tile that others share too goes to the workspace; a second
// kernel joins such tiles in the order of the keys, with a CTA for every 16 rows
// (one CTA reading 256 rows of ten shares alone took 50 us of 97).
// Every wait is bounded; on expiry all roles stop, copies in flight are waited
// for, and TMEM is freed.
#include "qcache_attend.cuh"

namespace statekv {
namespace {

using namespace qc;

constexpr int kBK = 128;           // keys of a step
constexpr int kHalf = 128;         // query rows of a half
constexpr int kTileRows = 2 * kHalf;
static_assert(kTileRows == kQCacheWideRows, "rows of a tile");
constexpr int kThreads = 512;
// Ring slots.  D = 128: K tiles of codes (used as they are), V tiles of codes, V
// tiles in fp16.  D = 64: K has fp16 tiles too, and its codes go through V's ring.
constexpr int kKTiles = 3, kVRaw = 2, kConvTiles = 2;
constexpr int kCost = 6;           // a CTA's fixed cost per tile, in steps (4: 418 us where this takes 413, 9: 415)
constexpr int kLeast = 4;          // steps worth a CTA
constexpr uint32_t kColO = 256;    // S0 at 0, S1 at 128, O0, O1

template <int D>
struct Layout {
    static constexpr bool kDirect = D == 128;                         // K's codes are the MMA's operand
    static constexpr int kRawBytes = kBK * D;
    static constexpr int kF16Bytes = kBK * D * 2;
    static constexpr int kQBytes = kHalf * D * 2;                     // a half's Q: two e4m3 parts, or fp16
    static constexpr int kOffQ = 0;
    static constexpr int kOffK = kOffQ + 2 * kQBytes;                 // K operand tiles
    static constexpr int kKBytes = kDirect ? kRawBytes : kF16Bytes;
    static constexpr int kOffV = kOffK + kKTiles * kKBytes;           // V operand tiles, fp16
    static constexpr int kOffRaw = kOffV + kConvTiles * kF16Bytes;    // codes to be turned into fp16
    static constexpr int kOffBar = kOffRaw + kVRaw * kRawBytes;
    // raw_full[2] raw_empty[2] k_full[3] k_empty[3] v_empty[2] s_full[2] go[2][2] first[2][4] o_full[2]
    // o_read[2] drain turn[2]
    static constexpr int kBars = 33;
    static constexpr int kOffScale = kOffBar + ((kBars * 8 + 15) / 16) * 16;  // float[4 steps][16]: K groups, beta, unit
    static constexpr int kOffMisc = kOffScale + 4 * 16 * 4;           // tmem, abort, -, -, poison[8]
    static constexpr int kOffUnits = kOffMisc + 48;
    static_assert(kOffUnits % 16 == 0, "align");
    static constexpr int kAlloc = kOffUnits + line_bytes(kQCacheUnits) + 1024;
    static_assert(kOffScale % 16 == 0 && kRawBytes % 1024 == 0, "align");
    static_assert(kAlloc <= 232448, "shared memory budget");
};

// 16 consecutive 32-bit TMEM columns of this thread's lane <- registers.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0],"
        " {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Instruction descriptor, fp32 D: kind::f16 with fp16 A/B, or kind::f8f6f4 with
// e4m3 A/B (both formats have code 0).
constexpr uint32_t idesc_of(int M, int N, bool b_mn_major)
{
    return (1u << 4) | (static_cast<uint32_t>(b_mn_major) << 16) | (static_cast<uint32_t>(N >> 3) << 17) |
           (static_cast<uint32_t>(M >> 4) << 24);
}
constexpr uint32_t kE5m2A = 1u << 7;  // kind::f8f6f4: A in e5m2

// Products of NK k steps, fp16 inputs, fp32 accumulator.  The descriptors come as
// their 32-bit words and a step's offset goes onto the low one: the issuing warp
// shares its scheduler with softmax and converter warps, so every instruction
// beside the MMAs holds the tensor core up.
// S = A[smem, K-major] * B[smem, K-major], 32 bytes of the k axis per step.  fp16: one
// pass.  8 bits: A's two parts (e4m3, e5m2) one after the other, 128 rows of 128 bytes each.
template <int D>
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t alo, uint32_t blo, uint32_t hi, uint32_t idesc0)
{
    constexpr bool kDirect = Layout<D>::kDirect;
    constexpr int NK = kDirect ? 2 * (D / 32) : D / 16;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
        const uint32_t idesc = kDirect && k >= 4 ? idesc0 | kE5m2A : idesc0;
        // 16 KB per 128 bytes of the k axis (an e4m3 part), 32 bytes per step inside
        const uint32_t a = alo + (((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4);
        const uint32_t b = kDirect ? blo + (((k & 3) * 32) >> 4) : blo + (((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4);
        if constexpr (kDirect) {
            if (k == 0)
                asm volatile(
                    "{\n\t.reg .b64 ad, bd;\n\t"
                    "mov.b64 ad, {%1, %3};\n\t"
                    "mov.b64 bd, {%2, %3};\n\t"
                    "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, 0;\n\t}" ::"r"(d),
                    "r"(a), "r"(b), "r"(hi), "r"(idesc)
                    : "memory");
            else
                asm volatile(
                    "{\n\t.reg .b64 ad, bd;\n\t"
                    "mov.b64 ad, {%1, %3};\n\t"
                    "mov.b64 bd, {%2, %3};\n\t"
                    "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], ad, bd, %4, 1;\n\t}" ::"r"(d),
                    "r"(a), "r"(b), "r"(hi), "r"(idesc)
                    : "memory");
        } else {
            if (k == 0)
                asm volatile(
                    "{\n\t.reg .b64 ad, bd;\n\t"
                    "mov.b64 ad, {%1, %3};\n\t"
                    "mov.b64 bd, {%2, %3};\n\t"
                    "tcgen05.mma.cta_group::1.kind::f16 [%0], ad, bd, %4, 0;\n\t}" ::"r"(d),
                    "r"(a), "r"(b), "r"(hi), "r"(idesc)
                    : "memory");
            else
                asm volatile(
                    "{\n\t.reg .b64 ad, bd;\n\t"
                    "mov.b64 ad, {%1, %3};\n\t"
                    "mov.b64 bd, {%2, %3};\n\t"
                    "tcgen05.mma.cta_group::1.kind::f16 [%0], ad, bd, %4, 1;\n\t}" ::"r"(d),
                    "r"(a), "r"(b), "r"(hi), "r"(idesc)
                    : "memory");
        }
    }
}

// O (+)= A[tmem] * B[smem, MN-major]
template <int NK>
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t blo, uint32_t hi, uint32_t idesc, bool accumulate)
{
#pragma unroll
    for (int k = 0; k < NK; ++k) {
        if (k == 0 && !accumulate)
            asm volatile(
                "{\n\t.reg .b64 bd;\n\t"
                "mov.b64 bd, {%2, %3};\n\t"
                "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], bd, %4, 0;\n\t}" ::"r"(d),
                "r"(a), "r"(blo), "r"(hi), "r"(idesc)
                : "memory");
        else
            asm volatile(
                "{\n\t.reg .b64 bd;\n\t"
                "mov.b64 bd, {%2, %3};\n\t"
                "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], bd, %4, 1;\n\t}" ::"r"(d),
                "r"(a + 8 * k), "r"(blo + ((k * 2048) >> 4)), "r"(hi), "r"(idesc)
                : "memory");
    }
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32"
        " {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}

// two fp32 values -> two e5m2 codes, the first in the low byte
__device__ __forceinline__ uint32_t e5m2x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// Packed pair of floats in one 64-bit register (f32x2 arithmetic).
struct f2 {
    uint64_t r;
};

__device__ __forceinline__ f2 pk(float lo, float hi)
{
    f2 o;
    asm("mov.b64 %0, {%1, %2};" : "=l"(o.r) : "f"(lo), "f"(hi));
    return o;
}

__device__ __forceinline__ void upk(f2 x, float& lo, float& hi)
{
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x.r));
}

__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.r) : "l"(a.r), "l"(b.r), "l"(c.r));
    return d;
}

__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.r) : "l"(a.r), "l"(b.r));
    return d;
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// A tile's rows and keys.
struct Tile {
    Span sp;
    int hkv, head, row0, begin, hi, s1, halves;
};

__device__ __forceinline__ Tile tile_of(const QAttendParams& p, const Line& line, const Segment& s)
{
    Tile t;
    t.hkv = s.tile / p.row_tiles;
    const int rt = s.tile - t.hkv * p.row_tiles, R = p.row_end;
    const int ua = p.units.unit_abs(s.u);
    t.head = ua * p.c.Hkv + t.hkv;
    t.sp = line.span(s.u);
    t.row0 = p.row_begin + rt * kTileRows;
    const int last = min(R, t.row0 + kTileRows) - 1;
    t.hi = t.sp.stop == 0 ? 0 : p.causal ? t.sp.start + last / p.G + 1 : t.sp.stop;
    t.begin = t.sp.first / kBK * kBK;
    t.s1 = min(s.sb, steps_to<kBK>(t.sp, t.hi));
    t.halves = R - t.row0 > kHalf ? 2 : 1;
    return t;
}

// Keys [first, lim) that query row r (clipped to the rows there are) sees.
__device__ __forceinline__ int lim_of(const QAttendParams& p, const Span& sp, int r)
{
    return sp.stop == 0 ? 0 : p.causal ? sp.start + min(r, p.row_end - 1) / p.G + 1 : sp.stop;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    qcache_attend_wide(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                       const __grid_constant__ QAttendParams p)
{
    using L = Layout<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
    uint8_t* sQ = sm + L::kOffQ;
    uint8_t* sK = sm + L::kOffK;
    uint8_t* sV = sm + L::kOffV;
    uint8_t* sRaw = sm + L::kOffRaw;
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + L::kOffBar);
    uint64_t* raw_full = bars;
    uint64_t* raw_empty = bars + 2;
    uint64_t* k_full = bars + 4;    // D = 128: K codes have landed
    uint64_t* k_empty = bars + 7;   // both halves' Q K^T have read the tile
    uint64_t* v_empty = bars + 10;  // both halves' P V have read the tile
    uint64_t* s_full = bars + 12;   // per half: Q K^T of the step is done (and every MMA before it)
    uint64_t* go = bars + 14;       // [half][2] a half's step: P, the V tile, the next K tile
    // [half][4] a half's tile: Q and the first K tile.  K tiles may arrive while the Q of three
    // tiles of a step each is still to come.
    uint64_t* first = bars + 18;
    uint64_t* o_full = bars + 26;   // per half and tile: every P V is done
    uint64_t* o_read = bars + 28;   // per half and tile: O has been read out
    uint64_t* drain = bars + 30;
    uint64_t* turn = bars + 31;     // [half] the other half's products are issued
    float* scales = reinterpret_cast<float*>(sm + L::kOffScale);
    uint32_t* misc = reinterpret_cast<uint32_t*>(sm + L::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 1);
    volatile int* poison = reinterpret_cast<volatile int*>(misc + 4);  // [8 tiles], a byte per converter warp
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = blockIdx.x;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kVRaw; ++i) {
            mbar_init(&raw_full[i], 1);
            mbar_init(&raw_empty[i], 4);
        }
        for (int i = 0; i < kKTiles; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], 2);
        }
        for (int i = 0; i < kConvTiles; ++i) mbar_init(&v_empty[i], 2);
        for (int i = 0; i < 4; ++i) mbar_init(&go[i], 3 * 4);
        for (int i = 0; i < 8; ++i) mbar_init(&first[i], 2 * 4);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&o_full[i], 1);
            mbar_init(&o_read[i], 4);
            mbar_init(&turn[i], 1);
        }
        mbar_init(drain, 2);
        *abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(misc, 512);
        tmem_relinquish();
    }
    // (also the barrier after the initialisation above)
    const Line line = make_line<kThreads, kBK>(p, sm + L::kOffUnits, reinterpret_cast<uint32_t*>(sm), kCost, kLeast);
    tc_fence_after();
    const uint32_t tbase = misc[0];
    Walk walk(line, cta);
    Segment seg;

    auto wait = [&](uint64_t* bar, uint32_t parity) { return wait_full(bar, parity, p.watchdog_ns); };
    // one arrival for the warp: 128 arrivals at one barrier take longer than a tile's conversion
    auto warp_arrive = [&](uint64_t* bar) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar);
    };
    auto fail = [&] {
        *abort_flag = 1;
        *reinterpret_cast<volatile int32_t*>(p.c.status) = DEV_TIMEOUT_DECODE;
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;" ::: "memory");
        if (warp == 0) {
            // ---------------------------------------------------------- producer
            if (lane == 0) {
                tma_prefetch_desc(&tm_k);
                tma_prefetch_desc(&tm_v);
                bool ok = true;
                int n = 0, nk = 0;  // tiles so far in the ring of codes, and K tiles used as they are
                auto load = [&](uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int row, int head) {
                    mbar_arrive_expect_tx(bar, L::kRawBytes);
#pragma unroll
                    for (int b = 0; b < kBK / kQCacheKeyBox; ++b)
                        tma_load_3d(dst + b * kQCacheKeyBox * D, map, bar, 0, row + b * (kQCacheKeyBox * D / 128), head);
                };
                while (ok && walk.next(line, seg)) {
                    const Tile t = tile_of(p, line, seg);
                    for (int j = seg.sa; ok && j < t.s1; ++j) {
                        // below 2^31: statekv_qcache_init bounds the rows of 128 bytes
                        const int row = static_cast<int>(static_cast<long long>(t.begin + j * kBK) * D / 128);
                        for (int v = 0; v < 2; ++v) {
                            const bool direct = L::kDirect && v == 0;
                            int& c = direct ? nk : n;
                            const int slots = direct ? kKTiles : kVRaw, slot = c % slots, use = c / slots;
                            if (*abort_flag || (use >= 1 && !wait(direct ? &k_empty[slot] : &raw_empty[slot], (use - 1) & 1))) {
                                ok = false;
                                break;
                            }
                            if (direct) load(sK + slot * L::kKBytes, &tm_k, &k_full[slot], row, t.head);
                            else load(sRaw + slot * L::kRawBytes, v ? &tm_v : &tm_k, &raw_full[slot], row, t.head);
                            ++c;
                        }
                    }
                }
                if (!ok) fail();
                // copies in flight land before the CTA's memory goes away
                for (int i = n > kVRaw ? n - kVRaw : 0; i < n; ++i) wait(&raw_full[i % kVRaw], (i / kVRaw) & 1);
                for (int i = nk > kKTiles ? nk - kKTiles : 0; i < nk; ++i) wait(&k_full[i % kKTiles], (i / kKTiles) & 1);
            }
            __syncwarp();
        } else if (warp == 1 || warp == 3) {
            // ---------------------------------------------------------- MMA issuers
            if (lane == 0) {
                constexpr uint32_t kIdQK = idesc_of(kHalf, kBK, false), kIdPV = idesc_of(kHalf, D, true);
                constexpr uint32_t kKStep = L::kKBytes >> 4, kVStep = L::kF16Bytes >> 4;
                const int h = warp >> 1;
                // K-major and MN-major descriptors differ in the low word only (the stride of
                // 64-wide blocks)
                const uint64_t dk64 = sdesc_sw128(smem_addr(sK), 16, 1024);
                const uint32_t dq = static_cast<uint32_t>(sdesc_sw128(smem_addr(sQ) + h * L::kQBytes, 16, 1024));
                const uint32_t dv = static_cast<uint32_t>(sdesc_sw128(smem_addr(sV), kBK * 128, 1024));
                const uint32_t dk = static_cast<uint32_t>(dk64), hi = static_cast<uint32_t>(dk64 >> 32);
                const uint32_t tS = tbase + h * 128, tO = tbase + kColO + h * 128;
                bool ok = true;
                int n = 0;                      // steps so far, of both halves: K and V tiles
                uint32_t steps = 0, tiles = 0;  // of this half
                // The halves take turns at the tensor core, a step's products at a time.  Free to
                // run, they fall into step: both share it and then both leave it idle, with the
                // softmax warps idle first and crowded then (4,850 cycles a step against 4,150 at the time).
                uint32_t turns = 0;
                auto my_turn = [&] {
                    const uint32_t k = turns++;
                    return h == 1 ? wait(&turn[1], k & 1) : k == 0 || wait(&turn[0], (k - 1) & 1);
                };
                auto pass_turn = [&] { mbar_arrive(&turn[1 - h]); };
                while (ok && walk.next(line, seg)) {
                    const Tile t = tile_of(p, line, seg);
                    const int nt = t.s1 - seg.sa;
                    if (nt <= 0) continue;  // nothing visible: no MMA, no barrier of this tile is used
                    if (h >= t.halves) {
                        n += nt;
                        continue;
                    }
                    // a slot is free when both halves have read it; alone, this one arrives twice
                    const bool alone = t.halves == 1;
                    auto release = [&](uint64_t* bar) {
                        umma_commit(bar);
                        if (alone) mbar_arrive(bar);
                    };
                    auto qk = [&](int i) {
                        mma_ss<D>(tS, dq, dk + (i % kKTiles) * kKStep, hi, kIdQK);
                        umma_commit(&s_full[h]);
                        release(&k_empty[i % kKTiles]);
                    };
                    ok = wait(&first[4 * h + (tiles & 3)], (tiles >> 2) & 1) && (alone || my_turn());
                    if (!ok) break;
                    tc_fence_after();
                    qk(n);
                    if (!alone) pass_turn();
                    // the first P V overwrites O
                    ok = tiles == 0 || wait(&o_read[h], (tiles - 1) & 1);
                    for (int j = 0; ok && j < nt; ++j, ++steps) {
                        const int i = n + j;
                        ok = wait(&go[2 * h + (steps & 1)], (steps >> 1) & 1) && (alone || my_turn());
                        if (!ok) break;
                        tc_fence_after();
                        mma_ts<kBK / 16>(tO, tS, dv + (i % kConvTiles) * kVStep, hi, kIdPV, j > 0);
                        if (j == nt - 1) umma_commit(&o_full[h]);
                        release(&v_empty[i % kConvTiles]);
                        if (j < nt - 1) qk(i + 1);
                        if (!alone) pass_turn();
                    }
                    n += nt;
                    ++tiles;
                }
                if (!ok) fail();
                // every MMA issued so far finishes before TMEM is released
                umma_commit(drain);
                wait(drain, 0);
            }
            __syncwarp();
        }
        tc_fence_before();
        __syncthreads();
        if (warp == 1) tmem_dealloc(tbase, 512);
        pdl_wait();  // launched beside the call's other kernel: not complete before that is
    } else if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;" ::: "memory");
        // -------------------------------------------------------------- converters
        const int key = threadIdx.x - 128;
        // the warp's byte of each tile's poison word: the warps may be a step apart, so none
        // clears what another has set
        volatile uint8_t* mark = reinterpret_cast<volatile uint8_t*>(misc + 4) + (warp - 4);
        bool ok = true;
        int n = 0, step = 0, tiles = 0;  // raw tiles, steps, tiles with steps so far
        uint32_t gsteps0 = 0, gsteps1 = 0, gtiles0 = 0, gtiles1 = 0;  // steps and tiles of each half so far
        while (ok && walk.next(line, seg)) {
            const Tile t = tile_of(p, line, seg);
            if (t.s1 <= seg.sa) continue;
            const int first_lim = lim_of(p, t.sp, t.row0);
            const float* scale0 = p.c.scale[0] + static_cast<size_t>(t.head) * static_cast<size_t>(p.c.cap >> p.c.block_log2);
            const float* scale1 = p.c.scale[1] + (scale0 - p.c.scale[0]);
            // Scales of the step's 16-key groups, lane % 8 each, read a step ahead; a group that
            // no row of the tile sees counts as its nearest that some row does.
            float vs, ks;
            auto read_scales = [&](int j) {
                const int at = min(max(t.begin + j * kBK + 16 * (lane & 7), t.sp.first), t.hi - 1) >> p.c.block_log2;
                vs = scale1[at];
                ks = scale0[at];
            };
            read_scales(seg.sa);
            float vref = 0.f, vinv = 0.f, vmax = 0.f;
            // the softmax warpgroups are fewer than eight tiles with steps behind
            if (lane == 0) mark[4 * (tiles & 7)] = 0;
            __syncwarp();
            for (int j = seg.sa; ok && j < t.s1; ++j, ++step) {
                const int base = t.begin + j * kBK;
                // the unit of O follows the step's V scale: up at once, down when the scale is
                // below 2^-6 of it, and never below 2^-64 of the largest seen
                float vtop = vs, beta = 1.f;
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) vtop = fmaxf(vtop, __shfl_xor_sync(0xffffffffu, vtop, o));
                const float mine = __shfl_sync(0xffffffffu, vs, key >> 4);
                if (vtop > vref || vtop < vref * 0x1p-6f) {
                    const float now = fmaxf(vtop, vmax * 0x1p-64f);
                    beta = vref / now;
                    vref = now;
                    vinv = 1.f / now;
                    vmax = fmaxf(vmax, vtop);
                }
                const __half2 ratio = __float2half2_rn(mine * vinv);
                float* ss = scales + (step & 3) * 16;
                if (key < 10) ss[key] = key < 8 ? ks : key == 8 ? beta : vref;
                if (j + 1 < t.s1) read_scales(j + 1);
                const bool whole = base >= t.sp.first && base + kBK <= first_lim;
                const bool keep = base + key >= t.sp.first && base + key < t.hi;
                for (int v = 0; v < 2; ++v) {
                    const bool direct = L::kDirect && v == 0;
                    const int raw = n % kVRaw;
                    // K's codes are used as they are: the warp only passes their arrival on
                    bool there = direct ? wait(&k_full[step % kKTiles], (step / kKTiles) & 1)
                                        : wait(&raw_full[raw], (n / kVRaw) & 1);
                    if (expire_here(p, step == 1)) there = false;
                    // one verdict for the warp: a lane that gave up alone would be missed at the next __syncwarp
                    ok = __all_sync(0xffffffffu, there);
                    if (!ok) break;
                    if (!direct) {
                    const uint8_t* src = sRaw + raw * L::kRawBytes;
                    uint4 x[D / 16];
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) x[c] = *reinterpret_cast<const uint4*>(src + at<D>(key, 16 * c));
                    if (v == 1 && !whole) {
                        // a V row that no query of the tile sees may hold anything: zero.  A NaN in
                        // one that only some see is taken out too and put back row by row at the end
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t* w = reinterpret_cast<uint32_t*>(&x[c]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t bad = __vcmpeq4(w[i] & 0x7f7f7f7fu, 0x7f7f7f7fu);
                                if (keep && bad) mark[4 * (tiles & 7)] = 1;
                                w[i] = keep ? w[i] & ~bad : 0u;
                            }
                        }
                    }
                    const int slots = v ? kConvTiles : kKTiles, slot = step % slots, use = step / slots;
                    ok = __all_sync(0xffffffffu, use == 0 || wait(v ? &v_empty[slot] : &k_empty[slot], (use - 1) & 1));
                    if (!ok) break;
                    uint8_t* dst = v ? sV + slot * L::kF16Bytes : sK + slot * L::kKBytes;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        const uint32_t w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
                        uint32_t f[8];
#pragma unroll
                        for (int i = 0; i < 4; ++i) f16_of(w[i], f[2 * i], f[2 * i + 1]);
                        if (v == 1) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&f[i]), ratio);
                                f[i] = *reinterpret_cast<const uint32_t*>(&y);
                            }
                        }
                        uint8_t* block = dst + (c >> 2) * (kBK * 128);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            *reinterpret_cast<uint4*>(block + sw128_offset(key, 2 * (c & 3) + i)) =
                                make_uint4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
                    }
                    fence_proxy_async_smem();
                    }
                    // who waits for the tile: K starts a half's tile or is part of its step before;
                    // V is part of its step, and stands for the next K where there is none
                    __syncwarp();
                    // lanes 0 and 1 tell the two halves, lane 2 the producer: only here, after the
                    // stores that need them, have the warp's reads of the raw tile surely returned
                    // (an arrival behind the bare loads let the next copy overtake them)
                    if (lane < (direct ? 2 : 3) && (lane != 1 || t.halves == 2)) {
                        const uint32_t gs = (lane == 1 ? gsteps1 : gsteps0) - (v == 0), gt = lane == 1 ? gtiles1 : gtiles0;
                        uint64_t* bar = lane == 2 ? &raw_empty[raw]
                                        : v == 0 && j == seg.sa ? &first[4 * lane + (gt & 3)] : &go[2 * lane + (gs & 1)];
                        mbar_arrive(bar);
                        if (lane < 2 && v == 1 && j == t.s1 - 1) mbar_arrive(bar);
                    }
                    n += !direct;
                    gsteps0 += v;
                    gsteps1 += v & (t.halves - 1);
                }
            }
            ++gtiles0;
            gtiles1 += t.halves - 1;
            ++tiles;
        }
        if (!ok) fail();
        __syncthreads();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 192;" ::: "memory");
        // -------------------------------------------------------------- softmax
        const int h = (warp >> 2) - 2;
        const int row = threadIdx.x & 127;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t tS = tbase + lanes + h * 128, tO = tbase + lanes + kColO + h * 128;
        const int R = p.row_end;
        bool ok = true;
        uint32_t steps = 0, used = 0;  // of this half
        int4 starts = make_int4(-1, 0, 0, 0);  // the shared tile that begins in this CTA's share
        int step = 0, tiles = 0;
        while (ok && walk.next(line, seg)) {
            const Tile t = tile_of(p, line, seg);
            const int nt = max(0, t.s1 - seg.sa);
            const int r = t.row0 + h * kHalf + row;   // query row of the KV head
            const bool active = h < t.halves;
            float ref = -INFINITY, l = 0.f, vref = 0.f;
            const int lim = lim_of(p, t.sp, r);
            if (active && nt > 0) {
                // Q row, scaled by a power of two: into [2^14, 2^15) as fp16, or [2^7, 2^8) as an
                // e4m3 and an e5m2 part; K-major swizzled
                float qscale;
                {
                    uint4 x[D / 8];
                    const uint4* q = reinterpret_cast<const uint4*>(p.q + row_of(p, seg.u, t.hkv, min(r, R - 1)) * D);
                    uint32_t top = 0;
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) {
                        x[c] = r < R ? q[c] : make_uint4(0u, 0u, 0u, 0u);
                        top = __vmaxu2(top, __vmaxu2(__vmaxu2(x[c].x & 0x7fff7fffu, x[c].y & 0x7fff7fffu),
                                                     __vmaxu2(x[c].z & 0x7fff7fffu, x[c].w & 0x7fff7fffu)));
                    }
                    constexpr int kTop = L::kDirect ? 7 : 14;
                    const int e = min(254, max(kTop + 1, static_cast<int>(max(top & 0xffffu, top >> 16) >> 7)));
                    const float up = __uint_as_float(static_cast<uint32_t>(min(254, 254 + kTop - e)) << 23);
                    qscale = __uint_as_float(static_cast<uint32_t>(e - kTop) << 23) * p.scale_log2;
                    uint8_t* sq = sQ + h * L::kQBytes;
                    // a non-finite element makes the row's scores NaN, as its softmax is
                    const bool bad = (top & 0xffffu) >= 0x7f80u || (top >> 16) >= 0x7f80u;
                    if constexpr (L::kDirect) {
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t hi4[4], lo4[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint4& y = x[2 * c + (i >> 1)];
                                const uint32_t w0 = i & 1 ? y.z : y.x, w1 = i & 1 ? y.w : y.y;
                                const float f[4] = {__uint_as_float(w0 << 16) * up, __uint_as_float(w0 & 0xffff0000u) * up,
                                                    __uint_as_float(w1 << 16) * up, __uint_as_float(w1 & 0xffff0000u) * up};
                                uint32_t part[2] = {0u, 0u};
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    uint32_t a, g, l0, l1;
                                    const uint32_t code = e4m3x2(f[2 * b], f[2 * b + 1]);
                                    f16_of(code, a, g);  // the codes' values
                                    const float2 v2 = __half22float2(*reinterpret_cast<const __half2*>(&a));
                                    l0 = e5m2x2(f[2 * b] - v2.x, f[2 * b + 1] - v2.y);
                                    l1 = bad ? 0x7f7fu : code;
                                    part[0] |= l1 << (16 * b);
                                    part[1] |= l0 << (16 * b);
                                }
                                hi4[i] = part[0];
                                lo4[i] = part[1];
                            }
                            *reinterpret_cast<uint4*>(sq + sw128_offset(row, c)) = make_uint4(hi4[0], hi4[1], hi4[2], hi4[3]);
                            *reinterpret_cast<uint4*>(sq + kHalf * 128 + sw128_offset(row, c)) =
                                make_uint4(lo4[0], lo4[1], lo4[2], lo4[3]);
                        }
                    } else {
                        auto cv = [&](uint32_t w) {
                            return bad ? 0x7fff7fffu : pack_f16(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xffff0000u) * up);
                        };
#pragma unroll
                        for (int c = 0; c < D / 8; ++c)
                            *reinterpret_cast<uint4*>(sq + (c >> 3) * (kHalf * 128) + sw128_offset(row, c & 7)) =
                                make_uint4(cv(x[c].x), cv(x[c].y), cv(x[c].z), cv(x[c].w));
                    }
                    fence_proxy_async_smem();
                    warp_arrive(&first[4 * h + (used & 3)]);
                }
                const int lim0 = lim_of(p, t.sp, t.row0 + h * kHalf);  // the half's first row sees the fewest
                for (int j = 0; j < nt; ++j, ++step) {
                    const int base = t.begin + (seg.sa + j) * kBK;
                    ok = __all_sync(0xffffffffu, wait(&s_full[h], steps & 1));
                    if (!ok) break;
                    ++steps;
                    tc_fence_after();
                    const float* ss = scales + (step & 3) * 16;
                    float v[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(tS + 32 * c, v[c]);
                    tmem_ld_wait();
                    if (base < t.sp.first || base + kBK > lim0) {  // some row misses some key
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                const int key = base + 32 * c + i;
                                if (key < t.sp.first || key >= lim) v[c][i] = -INFINITY;
                            }
                    }
                    float cs[8], sum;
#pragma unroll
                    for (int gr = 0; gr < 8; gr += 4) {
                        const float4 x = *reinterpret_cast<const float4*>(ss + gr);
                        // positive, also where a zero query meets a zero block: a masked score stays
                        // -inf under it (the addend rounds away beside a product from 2^-102 on, and
                        // scores of smaller ones are 0 beside any reference)
                        cs[gr] = fmaf(qscale, x.x, 0x1p-126f);
                        cs[gr + 1] = fmaf(qscale, x.y, 0x1p-126f);
                        cs[gr + 2] = fmaf(qscale, x.z, 0x1p-126f);
                        cs[gr + 3] = fmaf(qscale, x.w, 0x1p-126f);
                    }
                    const float2 bu = *reinterpret_cast<const float2*>(ss + 8);
                    float beta = bu.x;
                    vref = bu.y;
                    // a row that has seen no key yet sets its reference first
                    bool set = __any_sync(0xffffffffu, ref == -INFINITY) || beta != 1.f;
#pragma unroll 1
                    for (int pass = 0;; ++pass) {
                        if (set) {
                            // the largest score in log2 units: of each 16-key group, then times its scale
                            float high = -INFINITY;
#pragma unroll
                            for (int gr = 0; gr < 8; ++gr) {
                                const float* x = &v[gr >> 1][16 * (gr & 1)];
                                float m0 = fmaxf(x[0], x[1]), m1 = fmaxf(x[2], x[3]);
#pragma unroll
                                for (int i = 4; i < 16; i += 4) {
                                    m0 = max3(m0, x[i], x[i + 1]);
                                    m1 = max3(m1, x[i + 2], x[i + 3]);
                                }
                                high = fmaxf(high, fmaxf(m0, m1) * cs[gr]);
                            }
                            const float now = fmaxf(ref, high);
                            float alpha = now == ref ? 1.f : ex2(ref - now);
                            ref = now;
                            l *= alpha;
                            alpha *= beta;
                            beta = 1.f;
                            if (j > 0) {  // the P V before this step's Q K^T have completed
#pragma unroll 1
                                for (int c = 0; c < D / 16; ++c) {
                                    uint32_t w[16];
                                    tmem_ld16(tO + 16 * c, w);
                                    tmem_ld_wait();
#pragma unroll
                                    for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) * alpha);
                                    tmem_st16(tO + 16 * c, w);
                                }
                            }
                        }
                        const float sub = ref == -INFINITY ? 0.f : kRefBias - ref;
                        const f2 sub2 = pk(sub, sub);
                        f2 acc[2] = {pk(0.f, 0.f), pk(0.f, 0.f)};
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t w[16];
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                const float cg = cs[2 * c + (i >> 4)];
                                float a, b;
                                upk(fma2(pk(v[c][i], v[c][i + 1]), pk(cg, cg), sub2), a, b);
                                a = ex2(a);
                                b = ex2(b);
                                acc[(i >> 1) & 1] = add2(acc[(i >> 1) & 1], pk(a, b));
                                w[i >> 1] = pack_f16(a, b);
                            }
                            tmem_st16(tS + 16 * c, w);
                        }
                        float s0, s1;
                        upk(add2(acc[0], acc[1]), s0, s1);
                        sum = s0 + s1;
                        // weights that fp16 may not hold: set the reference and weigh again (the
                        // scores are in registers); a NaN stays one
                        if (pass == 1 || !__any_sync(0xffffffffu, !(sum <= 0x1p15f))) break;
                        set = true;
                    }
                    l += sum;
                    tmem_st_wait();
                    tc_fence_before();
                    warp_arrive(&go[2 * h + ((steps - 1) & 1)]);
                }
                if (!ok) break;
            } else {
                step += nt;  // the other half's steps
            }

            // O of the row: normalised to the output, or this CTA's share of it
            const bool split = seg.steps > 0 && seg.ca != seg.cb;
            const float scale = l == 0.f ? 0.f : vref / l;
            bool poisoned = false;
            if (active && nt > 0) {
                ok = __all_sync(0xffffffffu, wait(&o_full[h], used & 1));
                if (!ok) break;
                ++used;
                tc_fence_after();
                poisoned = poison[tiles & 7] != 0;
            }
            tiles += nt > 0;
            const size_t out_row = row_of(p, seg.u, t.hkv, min(r, R - 1));
            const size_t slot = 2 * static_cast<size_t>(cta) + (cta == seg.ca);
            float* part = p.part_o + slot * kTileRows * D + (h * kHalf + row) * 4;  // [D / 4][row][4]
            if (active) {
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    float o[32];
                    if (nt > 0) {
                        tmem_ld32(tO + 32 * c, o);
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = 0.f;
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = l == 0.f ? 0.f : o[i] * scale;
                    if (poisoned && r < R) {
                        // the NaN codes that the converters took out, for the keys this row sees
                        const uint8_t* codes = p.c.codes[1] + static_cast<size_t>(t.head) * p.c.cap * D + 32 * c;
                        const int lim_all = lim_of(p, t.sp, t.row0);
                        const int from = max(t.sp.first, t.begin + seg.sa * kBK), to = min(lim, t.begin + t.s1 * kBK);
                        for (int key = from; key < to; ++key) {
                            const int base = key / kBK * kBK;
                            if (base >= t.sp.first && base + kBK <= lim_all) continue;  // a whole step kept its NaN
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if ((codes[static_cast<size_t>(key) * D + i] & 0x7f) == 0x7f) o[i] = NAN;
                        }
                    }
                    if (r < R) {
                        if (split) {
#pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                *reinterpret_cast<float4*>(part + static_cast<size_t>(8 * c + i / 4) * kTileRows * 4) =
                                    make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; i += 8)
                                *reinterpret_cast<uint4*>(p.out + out_row * D + 32 * c + i) =
                                    make_uint4(pack_bf16x2(o[i], o[i + 1]), pack_bf16x2(o[i + 2], o[i + 3]),
                                               pack_bf16x2(o[i + 4], o[i + 5]), pack_bf16x2(o[i + 6], o[i + 7]));
                        }
                    }
                }
                if (nt > 0) {
                    tc_fence_before();
                    warp_arrive(&o_read[h]);
                }
                if (r < R) {
                    if (split) *reinterpret_cast<float2*>(p.part_ml + (slot * kTileRows + h * kHalf + row) * 2) = make_float2(ref, l);
                    else if (p.lse) p.lse[out_row] = lse_of(ref, l);
                }
            }
            if (split && seg.ca == cta) starts = make_int4(seg.u, t.hkv, t.row0, seg.cb);
        }
        if (warp == 8 && lane == 0) p.starts[cta] = ok ? starts : make_int4(-1, 0, 0, 0);
        if (!ok) fail();
        tc_fence_before();
        __syncthreads();
    }
}

// A record of the kernel before.  The join is launched while that kernel runs, so the
// words are not read-only for its whole life: a plain load, and it stays behind pdl_wait().
__device__ __forceinline__ int4 read_record(const int4* at)
{
    int4 x;
    asm volatile("ld.global.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(at) : "memory");
    return x;
}

// Joins the shared tile that began with CTA blockIdx.x (kFew: tile blockIdx.x, if it is
// shared), 16 rows of it: weights l_c 2^(ref_c - M) of the shares, in the order of the
// keys; one pass with kAhead shares under way.  kFew is for tiles of four shares and
// more: no CTAs without work (2,400 of them take longer to start than the others work)
// and one round trip (126 rows over 12.5k keys in 4 tiles: 31 -> 26 us for the call), where
// two or three shares want more CTAs on an SM.
template <int D, bool kFew>
__global__ void __launch_bounds__(16 * D / 4) qcache_join(const __grid_constant__ QAttendParams p)
{
    constexpr int kAhead = kFew ? 10 : 2;
    pdl_wait();
    // the tile's record: of the CTA it begins with
    __shared__ int found[2];
    int4 tile;
    int ca = blockIdx.x, cb;
    if constexpr (kFew) {
        const int tiles = p.c.Hkv * p.row_tiles, u = blockIdx.x / tiles, t = blockIdx.x - u * tiles;
        tile = make_int4(u, t / p.row_tiles, p.row_begin + t % p.row_tiles * kTileRows, -1);
        if (threadIdx.x == 0) found[1] = -1;
        __syncthreads();
        for (int c = threadIdx.x; c < p.ctas; c += blockDim.x) {
            const int4 x = read_record(p.starts + c);
            if (x.x == tile.x && x.y == tile.y && x.z == tile.z) {
                found[0] = c;
                found[1] = x.w;
            }
        }
        __syncthreads();
        ca = found[0];
        cb = found[1];
        if (cb < 0) return;
    } else {
        tile = read_record(p.starts + ca);
        cb = tile.w;
        if (tile.x < 0) return;
    }
    const int row = blockIdx.y * 16 + (threadIdx.x & 15), col = threadIdx.x >> 4, r = tile.z + row;
    if (r >= p.row_end) return;
    auto slot_of = [&](int c) { return (2 * static_cast<size_t>(c) + (c == ca)) * kTileRows; };
    const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + row;
    const float4* po = reinterpret_cast<const float4*>(p.part_o) + static_cast<size_t>(col) * kTileRows + row;
    float M = -INFINITY, total = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = ca; c0 <= cb; c0 += kAhead) {
        float2 x[kAhead];
        float4 o[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const size_t at = slot_of(min(c0 + k, cb));
            x[k] = ml[at];
            o[k] = po[at * (D / 4)];
            if (c0 + k > cb) x[k] = make_float2(-INFINITY, 0.f);
        }
        float now = M;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) now = fmaxf(now, x[k].x);
        const float old = M == -INFINITY ? 0.f : ex2(M - now);
        M = now;
        total *= old;
        a = make_float4(a.x * old, a.y * old, a.z * old, a.w * old);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const float f = x[k].y == 0.f ? 0.f : x[k].y * ex2(x[k].x - M);
            total += f;
            a.x += o[k].x * f;
            a.y += o[k].y * f;
            a.z += o[k].z * f;
            a.w += o[k].w * f;
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const size_t out_row = row_of(p, tile.x, tile.y, r);
    *reinterpret_cast<uint2*>(p.out + out_row * D + 4 * col) =
        make_uint2(pack_bf16x2(a.x * inv, a.y * inv), pack_bf16x2(a.z * inv, a.w * inv));
    if (col == 0 && p.lse) p.lse[out_row] = lse_of(M, total);
}

// The register split (WG0 48, WG1 80, the softmax warpgroups 192 per thread) must
// fit the registers the CTA is launched with, or setmaxnreg.inc would wait forever.
constexpr int kLaunchRegs = 128;
static_assert(128 * (48 + 80 + 192 + 192) <= kThreads * kLaunchRegs, "register split");

template <int D>
cudaError_t prepare()
{
    cudaFuncAttributes fa;
    const cudaError_t e = cudaFuncGetAttributes(&fa, qcache_attend_wide<D>);
    if (e != cudaSuccess) return e;
    if (fa.numRegs < kLaunchRegs) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(qcache_attend_wide<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<D>::kAlloc);
}

}  // namespace

cudaError_t qcache_wide_prepare()
{
    const cudaError_t e = prepare<64>();
    return e != cudaSuccess ? e : prepare<128>();
}

template <int D>
static cudaError_t launch(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const QAttendParams& p, bool overlap,
                          cudaStream_t st)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(p.ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Layout<D>::kAlloc;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = overlap ? 1 : 0;
    cudaError_t e = cudaLaunchKernelEx(&cfg, qcache_attend_wide<D>, tm_k, tm_v, p);
    if (e != cudaSuccess) return e;
    // programmatic launch: the join's CTAs are ready when the last CTA above ends
    const long long tiles = static_cast<long long>(p.U) * p.c.Hkv * p.row_tiles;
    const bool few = 4 * tiles <= p.ctas;
    const int rows = p.row_end - p.row_begin;
    cfg.gridDim = dim3(few ? static_cast<unsigned>(tiles) : p.ctas, ((rows < kTileRows ? rows : kTileRows) + 15) / 16);
    cfg.blockDim = dim3(16 * D / 4);
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, few ? qcache_join<D, true> : qcache_join<D, false>, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_qcache_wide(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const QAttendParams& p, bool overlap,
                               cudaStream_t st)
{
    return p.c.D == 64 ? launch<64>(tm_k, tm_v, p, overlap, st) : launch<128>(tm_k, tm_v, p, overlap, st);
}

}  // namespace statekv
