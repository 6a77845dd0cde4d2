// Attention over the cache held in 8 bits.
//
//   s_ij = (scale * ks_b) q_i . k_j,   o_i = sum_j softmax_j(s_i) vs_b v_j
// with e4m3 codes k_j, v_j and the scales of row j's block b: one pass over the
// keys with the running reference and sum of a softmax.
//
// Work.  A tile is 8 NT of the n * G query rows of a KV head of a unit (row r =
// token r / G, head r % G) against the keys that its rows see, in steps of 32
// keys.  One CTA per SM takes an equal share of all tiles' steps, laid end to
// end in the order (unit, KV head, row tile), so units of any lengths load every
// SM alike; a CTA's share of a tile is dealt to its warps step by step.  The
// lengths are read on the device: every CTA sums the units' steps itself.  A
// tile that several CTAs share is joined by the last of them to finish (a counter
// in the workspace), always in the order of the keys, so results do not depend on
// timing.
//
// Bound by HBM for a token of D = 128: 28 layers, 28 query and 4 KV heads, 50,194 keys:
// 212.6 us, 6.77 TB/s.  One layer alone: 19.7 us, of which the 51 MB are 7.6 and the
// start and the join the rest.  Two tiles of 16 rows read the codes twice, as
// they lie apart on the line: 28 rows of 28 layers over 12,548 keys 128 us, 106 for what
// they read.  With D = 64 the warps' chain from codes to products bounds a token (two
// warps to a scheduler, which issues in 40% of its cycles): 28 layers 149 us for 106.
//
// Inside a warp.  K and V codes of a step arrive as TMA copies (128-byte swizzle)
// in the warp's ring, each stage behind an mbarrier.  Codes become fp16 in
// registers (exact).  The products are transposed, S^T = K Q^T and O^T = V^T P^T,
// so that the m16n8k16 shape takes 16 keys (or head dims) by 8 query rows: the
// seven or eight query heads of a KV head fill it, and one conversion of a code
// serves all NT row groups.  The weights of S^T become the second product's B
// operand by an 8x8 transpose (movmatrix).
//
// Softmax.  Each row's weights are 2^(s - ref) with a reference that follows the
// maximum only when a score passes it by 2^8: scores, references, sums and O are
// fp32, a weight is at most 2^14 and is rounded to fp16 for its product with V
// (the sum takes it unrounded); weights stay normal in fp16 down to 2^-20 of the
// row's largest.  O is held in units of a V scale that follows the blocks' (a
// rescaling in fp32 loses nothing), and a block's scale enters P as its ratio to
// that unit, 2^-6 to 1.
//
// Fragments.  Any order of head dims and of keys inside a product's k axis, and
// any order of its m axis, gives the same sums, so the order is the one that makes
// shared-memory reads 16 bytes wide without bank conflicts (D = 128; 8-byte V
// reads, two-way, for D = 64).  Thread (g, tig) = (lane / 4, lane % 4):
//   K Q^T: reads bytes 16 tig ... of key rows key_of(g) and 8 + key_of(g); word i
//     is k step i: elements 4i, 4i+1 as the first pair, 4i+2, 4i+3 as the second.
//     D = 128 has bytes 64 + 16 tig ... as the steps 4..7.
//   V^T P^T: reads the V rows of its four keys of a k step at column group g; the
//     keys' bytes 2i and 2i + 1 are m tile i's rows g and g + 8.
#include <algorithm>

#include "qcache_attend.cuh"

namespace statekv {
namespace {

using namespace qc;

constexpr int kKeys = kQCacheKeyBox;
constexpr int kSegmentCost = 32;   // a CTA's fixed cost per tile, in steps
constexpr int kLeastSteps = 16;    // two rounds of the warps: less is not worth a CTA and the join
constexpr int kCounters = 256;     // arrival counters at the workspace's start, and the most CTAs
constexpr size_t kCounterBytes = 4096;

// Eight warps with three ring stages of 8 KB (D = 128) each: 12 x 2 took 225 us where
// this takes 214 on 28 layers of one token over 50,194 keys, and spilled with two row
// groups (92 us against 71 on 14 rows over 12,546 keys).
template <int D, int NT>
struct Layout {
    static constexpr int kWarps = 8;
    static constexpr int kStages = 3;
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kRows = 8 * NT;
    static constexpr int kMat = kKeys * D;
    static constexpr int kStage = 2 * kMat;
    static constexpr int kPitch = D + 4;                                  // floats of a joined row
    static constexpr int kMerge = kWarps * kRows * (kPitch + 3) * 4;      // O, reference, sum, V unit of each warp
    static constexpr int kRing = kWarps * kStages * kStage > kMerge ? kWarps * kStages * kStage : kMerge;
    static constexpr int kOffBar = (kRing + 1023) / 1024 * 1024;
    static constexpr int kOffUnits = (kOffBar + kWarps * kStages * 8 + 15) / 16 * 16;
    static constexpr int kAlloc = kOffUnits + line_bytes(kQCacheUnits) + 16 + 1024;
    static_assert(kMat % 1024 == 0, "swizzle atoms stay aligned");

    static_assert(kAlloc <= 232448, "shared memory budget");
};

// 8x8 transpose of 16-bit values across the warp (row lane / 4, columns 2 (lane % 4), + 1)
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// D (16x8, fp32) += A (16x16 fp16, row) * B (16x8 fp16, col)
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7},"
        " {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Key of an eight-key group that row m of a transposed score tile stands for.
template <int D>
__device__ __forceinline__ int key_of(int m)
{
    return D == 128 ? (m & 1) * 4 + (m >> 1) : m;
}

__device__ __forceinline__ void store_out(const QAttendParams& p, size_t row, int col, const float4& v)
{
    *reinterpret_cast<uint2*>(p.out + row * p.c.D + col) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

template <int D, int NT>
__global__ void __launch_bounds__(Layout<D, NT>::kThreads, 1)
    qcache_attend(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ QAttendParams p)
{
    using L = Layout<D, NT>;
    constexpr int kWarps = L::kWarps, kStages = L::kStages, kRows = L::kRows, kPitch = L::kPitch;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, tig = lane & 3;
    const int R = p.row_end;

    uint8_t* ring = sm + warp * (kStages * L::kStage);
    uint64_t* full = reinterpret_cast<uint64_t*>(sm + L::kOffBar) + warp * kStages;
    if (lane == 0) {
        for (int s = 0; s < kStages; ++s) mbar_init(&full[s], 1);
        fence_mbar_init();
        tma_prefetch_desc(&tm_k);
        tma_prefetch_desc(&tm_v);
    }

    const Line line = make_line<L::kThreads, kKeys>(p, sm + L::kOffUnits, reinterpret_cast<uint32_t*>(sm), kSegmentCost,
                                                    kLeastSteps);
    const int cta = blockIdx.x;
    if (p.row_begin > 0) pdl_launch_dependents();  // the wide kernel of the call comes next
    volatile int* flag = reinterpret_cast<volatile int*>(sm + L::kOffUnits + line_bytes(kQCacheUnits));

    int used = 0;  // this warp's ring steps so far (stage and phase)
    bool ok = true;
    Walk walk(line, cta);
    Segment seg;
    while (walk.next(line, seg)) {
        const int u = seg.u, tile = seg.tile, sa = seg.sa, ca = seg.ca, cb = seg.cb;
        const int hkv = tile / p.row_tiles, rt = tile - hkv * p.row_tiles;
        const int ua = p.units.unit_abs(u);
        const int head = ua * p.c.Hkv + hkv;
        const Span sp = line.span(u);
        const int row0 = p.row_begin + rt * kRows, last_row = min(R, row0 + kRows) - 1;
        // keys that some row (hi) and that every row (lo_end) of the tile sees; rows beyond
        // R have zero queries and no output, so it does not matter what they see
        const int hi = sp.stop == 0 ? 0 : p.causal ? sp.start + last_row / p.G + 1 : sp.stop;
        const int lo_end = sp.stop == 0 ? 0 : p.causal ? sp.start + row0 / p.G + 1 : sp.stop;
        const int begin = sp.first / kKeys * kKeys;
        const int s1 = min(seg.sb, steps_to<kKeys>(sp, hi));

        const int mine = sa + warp;
        const int count = mine < s1 ? (s1 - mine + kWarps - 1) / kWarps : 0;
        auto load = [&](int i) {
            if (lane == 0) {
                const int st = (used + i) % kStages;
                uint8_t* ks = ring + st * L::kStage;
                // below 2^31: statekv_qcache_init bounds the rows of 128 bytes
                const int row = static_cast<int>(static_cast<long long>(begin + (mine + i * kWarps) * kKeys) * D / 128);
                fence_proxy_async_smem();  // the warp's earlier reads of this stage come first
                mbar_arrive_expect_tx(&full[st], L::kStage);
                tma_load_3d(ks, &tm_k, &full[st], 0, row, head);
                tma_load_3d(ks + L::kMat, &tm_v, &full[st], 0, row, head);
            }
        };
        for (int i = 0; i < kStages - 1 && i < count; ++i) load(i);

        // Q fragments: row 8 t + g, scaled by a power of two into [2^14, 2^15); qscale is
        // that of the rows 8 t + 2 tig + e that this thread's scores belong to
        uint32_t qb[NT][D / 16][2];
        float qscale[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = row0 + 8 * t + g;
            uint4 raw[D / 32];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) raw[i] = make_uint4(0u, 0u, 0u, 0u);
            if (r < R) {
                const __nv_bfloat16* q = p.q + row_of(p, u, hkv, r) * D;
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
                    raw[i] = *reinterpret_cast<const uint4*>(q + (i >> 1) * 64 + 16 * tig + (i & 1) * 8);
            }
            const uint32_t* w = reinterpret_cast<const uint32_t*>(raw);
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
            top = max(top & 0xffffu, top >> 16);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = min(254, max(15, static_cast<int>(top >> 7)));
            const float up = __uint_as_float(static_cast<uint32_t>(268 - e) << 23);
            // a non-finite element makes the row's scores NaN, as its softmax is
            const float mys = top >= 0x7f80u ? NAN : __uint_as_float(static_cast<uint32_t>(e - 14) << 23) * p.scale_log2;
#pragma unroll
            for (int x = 0; x < 2; ++x) qscale[t][x] = __shfl_sync(0xffffffffu, mys, 4 * (2 * tig + x));
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t x = w[2 * s + b];
                    qb[t][s][b] = pack_f16(__uint_as_float(x << 16) * up, __uint_as_float(x & 0xffff0000u) * up);
                }
        }

        float ref[NT][2], l[NT][2];  // ref: the row's reference score, log2 units
        float o[NT][D / 16][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                ref[t][e] = -INFINITY;
                l[t][e] = 0.f;
            }
#pragma unroll
            for (int md = 0; md < D / 16; ++md)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][md][e] = 0.f;
        }
        float vref = 0.f, vinv = 0.f, vmax = 0.f;
        const size_t scale0 = static_cast<size_t>(head) * static_cast<size_t>(p.c.cap >> p.c.block_log2);
        const float* ksc = p.c.scale[0] + scale0;
        const float* vsc = p.c.scale[1] + scale0;

        // Scales of a step's two 16-key halves (K, K, V, V), read a step ahead; a half that
        // nothing sees counts as the other.
        float next[4] = {0.f, 0.f, 0.f, 0.f};
        auto read_scales = [&](int i) {
            const int base = begin + (mine + i * kWarps) * kKeys;
            const int b0 = base >> p.c.block_log2, b1 = (base + 16) >> p.c.block_log2;
            const int x = base + 16 > sp.first ? b0 : b1, y = base + 16 < hi ? b1 : b0;
            next[0] = ksc[x];
            next[1] = ksc[y];
            next[2] = vsc[x];
            next[3] = vsc[y];
        };
        if (count > 0) read_scales(0);
        int it = 0;
        for (; it < count; ++it) {
            const int base = begin + (mine + it * kWarps) * kKeys;
            const int st = (used + it) % kStages;
            // the stage that this load fills was read by step it - 1, which this warp has finished
            if (it + kStages - 1 < count) load(it + kStages - 1);
            const float ks2[2] = {next[0], next[1]}, vs2[2] = {next[2], next[3]};
            read_scales(min(it + 1, count - 1));
            ok = __all_sync(0xffffffffu, wait_full(&full[st], ((used + it) / kStages) & 1, p.watchdog_ns) &&
                                             !expire_here(p, warp == 0 && used + it == 1));
            if (!ok) break;
            const uint8_t* ks = ring + st * L::kStage;
            const uint8_t* vs = ks + L::kMat;
            const bool whole = base >= sp.first && base + kKeys <= lo_end;  // every row sees every key

            float sc[NT][2][4];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[t][mt][e] = 0.f;
                const int key = 16 * mt + key_of<D>(g);
#pragma unroll
                for (int hb = 0; hb < D / 64; ++hb) {
                    const uint4 x = *reinterpret_cast<const uint4*>(ks + at<D>(key, 64 * hb + 16 * tig));
                    const uint4 y = *reinterpret_cast<const uint4*>(ks + at<D>(key + 8, 64 * hb + 16 * tig));
                    const uint32_t xx[4] = {x.x, x.y, x.z, x.w}, yy[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t a[4];
                        f16_of(xx[i], a[0], a[2]);
                        f16_of(yy[i], a[1], a[3]);
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma(sc[t][mt], a, qb[t][4 * hb + i][0], qb[t][4 * hb + i][1]);
                    }
                }
            }
            // scores in log2 units, relative to the reference
            float high = -INFINITY;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int lim = whole ? 0 : p.causal ? sp.start + min(row0 + 8 * t + 2 * tig + e, last_row) / p.G + 1 : sp.stop;
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        const float c = qscale[t][e] * ks2[mt];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float& v = sc[t][mt][2 * h + e];
                            v *= c;
                            if (!whole) {
                                const int key = base + 16 * mt + 8 * h + key_of<D>(g);
                                if (key < sp.first || key >= lim) v = -INFINITY;
                            }
                            high = fmaxf(high, v - ref[t][e]);  // -inf - -inf: NaN, which fmaxf drops
                        }
                    }
                }
            // O is held in units of vref, which follows the step's V scale: up at once, down
            // when the scale is below 2^-6 of it, and never below 2^-64 of the largest seen
            const float vtop = fmaxf(vs2[0], vs2[1]);
            const bool unit = vtop > vref || vtop < vref * 0x1p-6f;
            if (__any_sync(0xffffffffu, high > kRefSlack) || unit) {
                float beta = 1.f;
                if (unit) {
                    const float now = fmaxf(vtop, vmax * 0x1p-64f);
                    beta = vref / now;
                    vref = now;
                    vinv = 1.f / now;
                    vmax = fmaxf(vmax, vtop);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float alpha[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(fmaxf(sc[t][0][e], sc[t][0][2 + e]), fmaxf(sc[t][1][e], sc[t][1][2 + e]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        const float now = fmaxf(ref[t][e], mx);
                        alpha[e] = now == ref[t][e] ? 1.f : ex2(ref[t][e] - now);
                        ref[t][e] = now;
                        l[t][e] *= alpha[e];
                        alpha[e] *= beta;
                    }
#pragma unroll
                    for (int md = 0; md < D / 16; ++md)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[t][md][e] *= alpha[e & 1];
                }
            }
            const float ratio[2] = {vs2[0] * vinv, vs2[1] * vinv};
            uint32_t pb[NT][2][2];  // P^T: row group, k step, half
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                // a row that has seen nothing has weights 2^-inf
                const float sub[2] = {ref[t][0] == -INFINITY ? 0.f : ref[t][0] - kRefBias,
                                      ref[t][1] == -INFINITY ? 0.f : ref[t][1] - kRefBias};
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float w0 = ex2(sc[t][mt][2 * h] - sub[0]), w1 = ex2(sc[t][mt][2 * h + 1] - sub[1]);
                        l[t][0] += w0;
                        l[t][1] += w1;
                        pb[t][mt][h] = transpose8(pack_f16(w0 * ratio[mt], w1 * ratio[mt]));
                    }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // this thread's four keys of the k step: (half, e) = (x >> 1, x & 1)
                uint32_t w[4][D / 32];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int key = 16 * j + 8 * (x >> 1) + key_of<D>(2 * tig + (x & 1));
                    const uint8_t* src = vs + at<D>(key, D == 128 ? 16 * key_of<D>(g) : 8 * g);
                    if constexpr (D == 128) {
                        const uint4 v = *reinterpret_cast<const uint4*>(src);
                        w[x][0] = v.x;
                        w[x][1] = v.y;
                        w[x][2] = v.z;
                        w[x][3] = v.w;
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2*>(src);
                        w[x][0] = v.x;
                        w[x][1] = v.y;
                    }
                }
                // A fragments of m tiles 2 i, 2 i + 1: bytes of a key pair, interleaved
                auto fragments = [&](int i, uint32_t (&a0)[4], uint32_t (&a1)[4]) {
                    const uint32_t lo0 = __byte_perm(w[0][i], w[1][i], 0x5140), lo1 = __byte_perm(w[2][i], w[3][i], 0x5140);
                    const uint32_t hi0 = __byte_perm(w[0][i], w[1][i], 0x7362), hi1 = __byte_perm(w[2][i], w[3][i], 0x7362);
                    f16_of(lo0, a0[0], a0[1]);
                    f16_of(lo1, a0[2], a0[3]);
                    f16_of(hi0, a1[0], a1[1]);
                    f16_of(hi1, a1[2], a1[3]);
                };
                bool nan = false;
                if (!whole) {
                    // rows that no query of the tile sees hold anything; a NaN in one that some
                    // queries see must not reach the others through 0 * NaN
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int key = base + 16 * j + 8 * (x >> 1) + key_of<D>(2 * tig + (x & 1));
                        const bool keep = key >= sp.first && key < hi;
#pragma unroll
                        for (int i = 0; i < D / 32; ++i) {
                            if (!keep) w[x][i] = 0;
                            nan = nan || __vcmpeq4(w[x][i] & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
                        }
                    }
                    nan = __any_sync(0xffffffffu, nan);
                }
                if (!nan) {
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        uint32_t a0[4], a1[4];
                        fragments(i, a0, a1);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            mma(o[t][2 * i], a0, pb[t][j][0], pb[t][j][1]);
                            mma(o[t][2 * i + 1], a1, pb[t][j][0], pb[t][j][1]);
                        }
                    }
                } else {
                    // key by key, each product added to the rows that see the key
#pragma unroll 1
                    for (int kk = 0; kk < 16; ++kk) {
                        uint32_t saved[4][D / 32];
#pragma unroll
                        for (int x = 0; x < 4; ++x)
#pragma unroll
                            for (int i = 0; i < D / 32; ++i) {
                                saved[x][i] = w[x][i];
                                if (kk != 8 * (x >> 1) + key_of<D>(2 * tig + (x & 1))) w[x][i] = 0;
                            }
                        const int key = base + 16 * j + kk;
#pragma unroll
                        for (int i = 0; i < D / 32; ++i) {
                            uint32_t a[2][4];
                            fragments(i, a[0], a[1]);
#pragma unroll
                            for (int t = 0; t < NT; ++t)
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    float one[4] = {0.f, 0.f, 0.f, 0.f};
                                    mma(one, a[b], pb[t][j][0], pb[t][j][1]);
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        const int r = min(row0 + 8 * t + 2 * tig + (e & 1), last_row);
                                        const int lim = p.causal ? sp.start + r / p.G + 1 : sp.stop;
                                        if (key >= sp.first && key < lim) o[t][2 * i + b][e] += one[e];
                                    }
                                }
                        }
#pragma unroll
                        for (int x = 0; x < 4; ++x)
#pragma unroll
                            for (int i = 0; i < D / 32; ++i) w[x][i] = saved[x][i];
                    }
                }
            }
            __syncwarp();  // the stage is refilled kStages - 1 steps later
        }
        if (!ok && lane == 0) {
            *reinterpret_cast<volatile int32_t*>(p.c.status) = DEV_TIMEOUT_DECODE;
            // let the copies already issued land before the shared memory is reused
            for (int s = it; s < min(count, it + kStages); ++s)
                wait_full(&full[(used + s) % kStages], ((used + s) / kStages) & 1, p.watchdog_ns);
        }
        used += count;
        // after an expired wait every warp still takes part in the join and the CTA then stops
        const bool abort = __syncthreads_or(!ok);

        // join the warps (in the ring's memory): row r's O = sum_w o_w vref_w 2^(ref_w - M) over
        // the same sum of l_w
        float* mo = reinterpret_cast<float*>(sm);            // [warp][row][kPitch]
        float* mm = mo + kWarps * kRows * kPitch;            // [warp][row]
        float* ml = mm + kWarps * kRows;
        float* mv = ml + kWarps * kRows;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float s = l[t][e];
                s += __shfl_xor_sync(0xffffffffu, s, 4);
                s += __shfl_xor_sync(0xffffffffu, s, 8);
                s += __shfl_xor_sync(0xffffffffu, s, 16);
                const int r = 8 * t + 2 * tig + e;
                if (g == 0) {
                    mm[warp * kRows + r] = ref[t][e];
                    ml[warp * kRows + r] = s;
                    mv[warp * kRows + r] = vref;
                }
                // m tile md, row g (h = 0) or g + 8 (h = 1): head dim (D / 8) key_of(g) + 2 md + h
                float* dst = mo + (warp * kRows + r) * kPitch + (D / 8) * key_of<D>(g);
#pragma unroll
                for (int md = 0; md < D / 16; md += 2)
                    *reinterpret_cast<float4*>(dst + 2 * md) = make_float4(o[t][md][e], o[t][md][2 + e], o[t][md + 1][e], o[t][md + 1][2 + e]);
            }
        __syncthreads();
        const int rows = last_row - row0 + 1;
        const size_t slot = 2 * static_cast<size_t>(cta) + (cta == ca);
        for (int i = threadIdx.x; i < rows * (D / 4); i += L::kThreads) {
            const int r = i / (D / 4), col = i % (D / 4) * 4;
            float M = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, mm[w * kRows + r]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float lw = ml[w * kRows + r];
                if (lw == 0.f) continue;  // this warp saw nothing of the row
                float f = ex2(mm[w * kRows + r] - M);
                sum += lw * f;
                f *= mv[w * kRows + r];
                const float4 x = *reinterpret_cast<const float4*>(mo + (w * kRows + r) * kPitch + col);
                acc.x += x.x * f;
                acc.y += x.y * f;
                acc.z += x.z * f;
                acc.w += x.w * f;
            }
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            acc = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
            if (ca == cb) {
                const size_t row = row_of(p, u, hkv, row0 + r);
                store_out(p, row, col, acc);
                if (col == 0 && p.lse) p.lse[row] = lse_of(M, sum);
            } else {
                *reinterpret_cast<float4*>(p.part_o + (slot * kRows + r) * D + col) = acc;
                if (col == 0) *reinterpret_cast<float2*>(p.part_ml + (slot * kRows + r) * 2) = make_float2(M, sum);
            }
        }
        if (ca != cb) {
            __syncthreads();
            if (threadIdx.x == 0) {
                // releases the CTA's share (the barrier above orders it before), acquires the others'
                int before;
                asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(p.counters + ca) : "memory");
                const bool last = before == cb - ca;
                if (last) p.counters[ca] = 0;  // as it was found
                *flag = last;
            }
            __syncthreads();
            if (*flag) {
                // one pass over the shares in the order of the keys, many loads ahead: running
                // reference, sum and row of the weights l_c 2^(M_c - M)
                for (int i = threadIdx.x; i < rows * (D / 4); i += L::kThreads) {
                    const int r = i / (D / 4), col = i % (D / 4) * 4;
                    const float2* ml2 = reinterpret_cast<const float2*>(p.part_ml) + r;
                    const float4* po = reinterpret_cast<const float4*>(p.part_o) + i;
                    auto slot_of = [&](int c) { return (2 * static_cast<size_t>(c) + (c == ca)) * kRows; };
                    float M = -INFINITY, sum = 0.f;
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    constexpr int kAhead = NT == 1 ? 20 : 12;
                    for (int c0 = ca; c0 <= cb; c0 += kAhead) {
                        float2 m2[kAhead];
                        float4 x[kAhead];
#pragma unroll
                        for (int k = 0; k < kAhead; ++k) {
                            const size_t at0 = slot_of(min(c0 + k, cb));
                            m2[k] = __ldcg(ml2 + at0);
                            x[k] = __ldcg(po + at0 * (D / 4));
                            if (c0 + k > cb) m2[k] = make_float2(-INFINITY, 0.f);
                        }
                        float now = M;
#pragma unroll
                        for (int k = 0; k < kAhead; ++k) now = fmaxf(now, m2[k].x);
                        const float old = M == -INFINITY ? 0.f : ex2(M - now);
                        M = now;
                        sum *= old;
                        acc = make_float4(acc.x * old, acc.y * old, acc.z * old, acc.w * old);
#pragma unroll
                        for (int k = 0; k < kAhead; ++k) {
                            const float f = m2[k].y == 0.f ? 0.f : m2[k].y * ex2(m2[k].x - M);
                            sum += f;
                            acc.x += x[k].x * f;
                            acc.y += x[k].y * f;
                            acc.z += x[k].z * f;
                            acc.w += x[k].w * f;
                        }
                    }
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    const size_t row = row_of(p, u, hkv, row0 + r);
                    store_out(p, row, col, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
                    if (col == 0 && p.lse) p.lse[row] = lse_of(M, sum);
                }
            }
        }
        if (abort) break;
        __syncthreads();  // the ring takes the next tile's copies
    }
}

template <int D, int NT>
cudaError_t prepare()
{
    return cudaFuncSetAttribute(qcache_attend<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Layout<D, NT>::kAlloc);
}

template <int D, int NT>
void launch(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const QAttendParams& p, cudaStream_t st)
{
    using L = Layout<D, NT>;
    qcache_attend<D, NT><<<p.ctas, L::kThreads, L::kAlloc, st>>>(tm_k, tm_v, p);
}

template <int D>
cudaError_t launch_nt(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const QAttendParams& p, cudaStream_t st)
{
    switch (p.tile_rows / 8) {
    case 1: launch<D, 1>(tm_k, tm_v, p, st); break;
    case 2: launch<D, 2>(tm_k, tm_v, p, st); break;
    default: launch<D, 3>(tm_k, tm_v, p, st); break;
    }
    static_assert(kQCacheNarrowRows == 24, "three row groups");
    return cudaGetLastError();
}

}  // namespace

QAttendPlan qcache_attend_plan(int U, int Hkv, int D, long long cap, int n, int G, int sms)
{
    QAttendPlan a{};
    a.rows = n * G;
    // Up to 32 rows are two tiles of 16 (28 rows over 8,000 keys, 28 layers of 4 KV heads: 91 us
    // here, 104 on tcgen05; 42 rows as two tiles of 24: 118 and 105).  More rows go in tiles of 24
    // while there are no more tiles than SMs and no more than 24 steps of 32 keys to an SM: the
    // tcgen05 kernel's start and join outlast such calls (56 rows over 1,000 keys, 4 KV heads: 17
    // us here, 20 there; 126 rows over 4,000: 19 and 22; over 8,000, 40 steps to an SM: 25 and
    // 24).  Keys are counted by the capacity, lengths are on the device.
    const long long small_tiles = static_cast<long long>(U) * Hkv * ((a.rows + kQCacheNarrowRows - 1) / kQCacheNarrowRows);
    if (a.rows > kQCacheFewRows && (small_tiles > sms || small_tiles * (cap / kKeys) > 24ll * sms)) {
        a.wide_rows = a.rows;
        // A few rows beyond whole tiles would cost the tcgen05 kernel most of a tile's time for
        // each step; where there are steps enough to fill the SMs, the other kernel reads the
        // cache once more for them instead.
        const int left = a.rows % kQCacheWideRows;
        if (a.rows > kQCacheWideRows && left <= kQCacheNarrowRows &&
            static_cast<long long>(U) * Hkv * (cap / 128) >= 8ll * sms)
            a.wide_rows -= left;
    }
    a.ctas = sms < kCounters ? sms : kCounters;
    const long long tiles = static_cast<long long>(Hkv) * ((a.rows + kQCacheWideRows - 1) / kQCacheWideRows);
    a.fits = tiles * (cap / (a.wide_rows > 0 ? 128 : kKeys) + 2 + kSegmentCost) <= 0x7fffffffll &&
             Hkv * (cap / kKeys + 2 + kSegmentCost) <= 0x7fffffffll;
    // one size for every call that the warp-level kernel takes alone, one for the others (in which
    // both kernels may be at work at once)
    const size_t row = 2 * static_cast<size_t>(a.ctas) * (static_cast<size_t>(D) * 4 + 8);
    a.part_o = kCounterBytes;
    a.part_wide = a.part_o + kQCacheNarrowRows * row;
    a.bytes = a.part_wide + (a.wide_rows > 0 ? kQCacheWideRows * row + static_cast<size_t>(a.ctas) * sizeof(int4) : 0);
    return a;
}

cudaError_t qcache_attend_prepare()
{
    cudaError_t e = qcache_wide_prepare();
    for (cudaError_t x : {prepare<64, 1>(), prepare<64, 2>(), prepare<64, 3>(), prepare<128, 1>(), prepare<128, 2>(),
                          prepare<128, 3>()})
        if (x != cudaSuccess) e = x;
    return e;
}

cudaError_t launch_qcache_attend(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const QAttendPlan& plan,
                                 const QAttendParams& p, uint8_t* workspace, cudaStream_t st)
{
    // Rows left over first: the wide kernel's CTAs come to the SMs as the other kernel's leave.
    for (int wide = 0; wide < 2; ++wide) {
        QAttendParams x = p;
        x.row_begin = wide ? 0 : plan.wide_rows;
        x.row_end = wide ? plan.wide_rows : plan.rows;
        if (x.row_begin >= x.row_end) continue;
        x.ctas = plan.ctas;
        const int count = x.row_end - x.row_begin, most_rows = wide ? kQCacheWideRows : kQCacheNarrowRows;
        x.row_tiles = (count + most_rows - 1) / most_rows;
        x.tile_rows = wide ? kQCacheWideRows : ((count + x.row_tiles - 1) / x.row_tiles + 7) / 8 * 8;
        x.counters = reinterpret_cast<int*>(workspace);
        x.part_o = reinterpret_cast<float*>(workspace + (wide ? plan.part_wide : plan.part_o));
        x.part_ml = x.part_o + 2 * static_cast<size_t>(x.ctas) * x.tile_rows * p.c.D;
        x.starts = reinterpret_cast<int4*>(x.part_ml + 4 * static_cast<size_t>(x.ctas) * x.tile_rows);
        // Units are stream-major: a launch takes whole streams, or some of one stream's layers,
        // as many as keep the line of places below 2^31.
        const long long places = static_cast<long long>(p.c.Hkv) * x.row_tiles * (p.c.cap / (wide ? 128 : kKeys) + 2 + kSegmentCost);
        const int most = static_cast<int>(std::min<long long>(kQCacheUnits, 0x7fffffffll / places));
        const int L = p.units.layer_count, S = p.U / L;
        const int ls = L < most ? L : most, ss = most / L > 0 ? most / L : 1;
        const size_t rows = static_cast<size_t>(p.n) * p.Hq;
        for (int s = 0; s < S; s += ss)
            for (int l = 0; l < L; l += ls) {
                QAttendParams y = x;
                y.units.stream_begin += s;
                y.units.layer_begin += l;
                y.units.layer_count = ls < L - l ? ls : L - l;
                y.U = (ss < S - s ? ss : S - s) * y.units.layer_count;
                const size_t u0 = static_cast<size_t>(s) * L + l;
                y.q += u0 * rows * p.c.D;
                y.out += u0 * rows * p.c.D;
                if (y.lse) y.lse += u0 * rows;
                cudaError_t e;
                if (wide) e = launch_qcache_wide(tm_k, tm_v, y, plan.wide_rows < plan.rows && s == 0 && l == 0, st);
                else if (p.c.D == 64) e = launch_nt<64>(tm_k, tm_v, y, st);
                else e = launch_nt<128>(tm_k, tm_v, y, st);
                if (e != cudaSuccess) return e;
            }
    }
    return cudaSuccess;
}

}  // namespace statekv
