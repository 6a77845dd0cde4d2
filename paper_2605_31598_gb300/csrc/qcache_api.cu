// Host side of the handle-free decoding operators in include/statekv.h: rotary
// positions with several axes, appending to the cache held in 8 bits, and
// attention over it.  Argument checks, TMA descriptors and launch parameters;
// no call here allocates or synchronises (statekv_qcache_sync does).
#include "../../include/statekv.h"
#include "statekv_kernels.cuh"

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdlib>
#include <cstring>

using namespace statekv;

namespace statekv {

int current_sm_count()
{
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices) return 1;
    if ((n = known[dev].load(std::memory_order_relaxed)) > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 1;
    known[dev].store(n, std::memory_order_relaxed);
    return n;
}

}  // namespace statekv

namespace {

constexpr unsigned long long kWaitNs = 2000000000ull;

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// What statekv_qcache_init leaves in a cache's opaque words: both descriptors
// (64-byte aligned copies are taken for a launch), a mark, and the fields that
// the descriptors stand for.
struct Prepared {
    CUtensorMap k, v;
    uint64_t mark, fields;
};
static_assert(sizeof(CUtensorMap) == 128, "size of a TMA descriptor");
static_assert(2 * 128 + 16 <= sizeof(statekv_qcache::opaque), "opaque words hold the descriptors");
constexpr uint64_t kMark = 0x716361636865'0001ull;

// Order-dependent mix of the fields that the descriptors and checks depend on.
uint64_t fields_of(const statekv_qcache& c)
{
    const uint64_t f[] = {static_cast<uint64_t>(c.num_streams), static_cast<uint64_t>(c.num_layers),
                          static_cast<uint64_t>(c.num_kv_heads), static_cast<uint64_t>(c.head_dim),
                          static_cast<uint64_t>(c.block_tokens), static_cast<uint64_t>(c.capacity),
                          reinterpret_cast<uint64_t>(c.k_codes), reinterpret_cast<uint64_t>(c.v_codes),
                          reinterpret_cast<uint64_t>(c.k_scale), reinterpret_cast<uint64_t>(c.v_scale),
                          reinterpret_cast<uint64_t>(c.k_tail), reinterpret_cast<uint64_t>(c.v_tail),
                          reinterpret_cast<uint64_t>(c.status)};
    uint64_t h = 1469598103934665603ull;
    for (uint64_t x : f) h = (h ^ x) * 1099511628211ull ^ (h >> 29);
    return h;
}

bool prepared(const statekv_qcache* c, Prepared* out)
{
    if (!c) return false;
    uint64_t tail[2];
    std::memcpy(tail, reinterpret_cast<const uint8_t*>(c->opaque) + 256, 16);
    if (tail[0] != kMark || tail[1] != fields_of(*c)) return false;
    if (out) {
        std::memcpy(&out->k, c->opaque, 128);
        std::memcpy(&out->v, reinterpret_cast<const uint8_t*>(c->opaque) + 128, 128);
    }
    return true;
}

QCacheView view_of(const statekv_qcache& c)
{
    QCacheView v{};
    v.codes[0] = static_cast<uint8_t*>(c.k_codes);
    v.codes[1] = static_cast<uint8_t*>(c.v_codes);
    v.scale[0] = c.k_scale;
    v.scale[1] = c.v_scale;
    v.tail[0] = static_cast<__nv_bfloat16*>(c.k_tail);
    v.tail[1] = static_cast<__nv_bfloat16*>(c.v_tail);
    v.status = c.status;
    v.Hkv = c.num_kv_heads;
    v.D = c.head_dim;
    v.block_log2 = c.block_tokens == 16 ? 4 : c.block_tokens == 32 ? 5 : c.block_tokens == 64 ? 6 : 7;
    v.cap = c.capacity;
    return v;
}

bool range_ok(const statekv_qcache& c, int sb, int sc, int lb, int lc)
{
    return sb >= 0 && sc >= 1 && sc <= c.num_streams && sb <= c.num_streams - sc && lb >= 0 && lc >= 1 &&
           lc <= c.num_layers && lb <= c.num_layers - lc;
}

}  // namespace

extern "C" {

statekv_status statekv_mrope(const statekv_mrope_args* a, statekv_stream stream)
{
    if (!a || a->num_tokens < 0 || a->num_q_heads < 0 || a->num_kv_heads < 0 || a->head_dim < 1 ||
        a->num_axes < 1 || a->num_axes > kMropeMaxAxes || a->num_pairs < 1 || 2 * a->num_pairs > a->head_dim ||
        (a->adjacent != 0 && a->adjacent != 1) || (a->transpose != 0 && a->transpose != 1) ||
        !std::isfinite(a->scale) || !a->freq || !a->axis)
        return STATEKV_ERR_INVALID_ARG;
    if (a->head_dim % 8 != 0 || a->head_dim > 2 * kMropeMaxPairs) return STATEKV_ERR_UNSUPPORTED;
    MropeParams p{};
    for (int i = 0; i < a->num_pairs; ++i) {
        if (a->axis[i] < 0 || a->axis[i] >= a->num_axes || !(std::fabs(a->freq[i]) < 3.141592653589793))
            return STATEKV_ERR_INVALID_ARG;
        // turns per position in 64-bit fixed point: |freq| / 2 pi < 1/2
        p.step[i] = static_cast<unsigned long long>(std::llrint(a->freq[i] / 6.283185307179586476925286766559 * 0x1p64));
        p.axis[i] = static_cast<uint8_t>(a->axis[i]);
    }
    if (a->num_tokens == 0) return STATEKV_OK;
    if (!a->positions || !aligned(a->positions, 4) || a->position_stride < 0 ||
        (a->position_stride > 0 && a->position_stride < a->num_tokens))
        return STATEKV_ERR_INVALID_ARG;
    const void* src[2] = {a->q, a->k};
    void* dst[2] = {a->q_out, a->k_out};
    const int64_t stride[2] = {a->q_stride, a->k_stride}, out_stride[2] = {a->q_out_stride, a->k_out_stride};
    const int heads[2] = {a->num_q_heads, a->num_kv_heads};
    for (int w = 0; w < 2; ++w) {
        if (!src[w]) continue;
        const int64_t row = static_cast<int64_t>(heads[w]) * a->head_dim;
        if (heads[w] < 1 || !dst[w] || !aligned(src[w], 16) || !aligned(dst[w], 16) || stride[w] < row ||
            out_stride[w] < row || stride[w] % 8 != 0 || out_stride[w] % 8 != 0 ||
            (src[w] == dst[w] && stride[w] != out_stride[w]))
            return STATEKV_ERR_INVALID_ARG;
        p.t[w].x = static_cast<const __nv_bfloat16*>(src[w]);
        p.t[w].y = static_cast<__nv_bfloat16*>(dst[w]);
        p.t[w].stride = stride[w];
        p.t[w].out_stride = out_stride[w];
        p.t[w].heads = heads[w];
    }
    if (p.t[0].heads + p.t[1].heads == 0) return STATEKV_ERR_INVALID_ARG;
    p.positions = a->positions;
    p.position_stride = a->position_stride;
    p.tokens = a->num_tokens;
    p.d = a->head_dim;
    p.pairs = a->num_pairs;
    p.adjacent = a->adjacent;
    p.transpose = a->transpose;
    p.scale = a->scale;
    return launch_mrope(p, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? STATEKV_OK : STATEKV_ERR_CUDA;
}

statekv_status statekv_qcache_init(statekv_qcache* c)
{
    if (!c || c->num_streams < 1 || c->num_layers < 1 || c->num_kv_heads < 1 || c->head_dim < 1 ||
        c->block_tokens < 1 || c->capacity < 1 || c->capacity % c->block_tokens != 0)
        return STATEKV_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return STATEKV_ERR_UNSUPPORTED;
    if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128)
        return STATEKV_ERR_UNSUPPORTED;
    const long long units = static_cast<long long>(c->num_streams) * c->num_layers;
    if (c->num_kv_heads > 32767 || units > 65535 || units * c->num_kv_heads > 0x7FFFFFFFll ||
        c->capacity > 0x7FFFFFFFll ||
        c->capacity * c->head_dim / 128 > (1ll << 31) / (units * c->num_kv_heads))
        return STATEKV_ERR_UNSUPPORTED;
    if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !c->status ||
        !aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scale, 4) ||
        !aligned(c->v_scale, 4) || !aligned(c->k_tail, 16) || !aligned(c->v_tail, 16) || !aligned(c->status, 4))
        return STATEKV_ERR_INVALID_ARG;
    Prepared d{};
    const int heads = static_cast<int>(units * c->num_kv_heads);
    if (qcache_attend_prepare() != cudaSuccess ||
        !encode_qcache(&d.k, c->k_codes, heads, c->capacity, c->head_dim) ||
        !encode_qcache(&d.v, c->v_codes, heads, c->capacity, c->head_dim))
        return STATEKV_ERR_CUDA;
    d.mark = kMark;
    d.fields = fields_of(*c);
    std::memcpy(c->opaque, &d.k, 128);
    std::memcpy(reinterpret_cast<uint8_t*>(c->opaque) + 128, &d.v, 128);
    std::memcpy(reinterpret_cast<uint8_t*>(c->opaque) + 256, &d.mark, 16);
    return STATEKV_OK;
}

statekv_status statekv_qcache_append(const statekv_qcache* c, const statekv_qcache_append_args* a,
                                     statekv_stream stream)
{
    if (!a || !prepared(c, nullptr) || !range_ok(*c, a->stream_begin, a->stream_count, a->layer_begin, a->layer_count) ||
        a->num_tokens < 0 || a->num_tokens > c->capacity)
        return STATEKV_ERR_INVALID_ARG;
    if (a->num_tokens == 0) return STATEKV_OK;
    if (!a->start || !aligned(a->start, 4)) return STATEKV_ERR_INVALID_ARG;
    QAppendParams p{};
    const void* src[2] = {a->k, a->v};
    const statekv_qcache_strides* strides[2] = {&a->k_strides, &a->v_strides};
    for (int w = 0; w < 2; ++w) {
        const statekv_qcache_strides& s = *strides[w];
        if (!src[w] || !aligned(src[w], 16) || s.unit < 0 || s.token < 0 || s.head < 0 || s.unit % 8 != 0 ||
            s.token % 8 != 0 || s.head % 8 != 0)
            return STATEKV_ERR_INVALID_ARG;
        p.src[w] = static_cast<const __nv_bfloat16*>(src[w]);
        p.unit_stride[w] = s.unit;
        p.token_stride[w] = s.token;
        p.head_stride[w] = s.head;
    }
    p.c = view_of(*c);
    p.units = UnitRange{a->stream_begin, a->layer_begin, a->layer_count, c->num_layers};
    p.U = a->stream_count * a->layer_count;
    p.n = a->num_tokens;
    p.start = a->start;
    return launch_qcache_append(p, reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? STATEKV_OK
                                                                                          : STATEKV_ERR_CUDA;
}

statekv_status statekv_qcache_workspace_bytes(const statekv_qcache* c, int32_t stream_count, int32_t layer_count,
                                              int32_t num_tokens, int32_t num_q_heads, size_t* bytes)
{
    if (!bytes || !prepared(c, nullptr) || !range_ok(*c, 0, stream_count, 0, layer_count) || num_tokens < 0 ||
        num_tokens > c->capacity || num_q_heads < 1 || num_q_heads % c->num_kv_heads != 0)
        return STATEKV_ERR_INVALID_ARG;
    const int G = num_q_heads / c->num_kv_heads;
    if (static_cast<long long>(num_tokens) * G > (1 << 24)) return STATEKV_ERR_UNSUPPORTED;
    const QAttendPlan plan = qcache_attend_plan(stream_count * layer_count, c->num_kv_heads, c->head_dim, c->capacity,
                                                num_tokens > 0 ? num_tokens : 1, G, current_sm_count());
    if (!plan.fits) return STATEKV_ERR_UNSUPPORTED;
    *bytes = plan.bytes;
    return STATEKV_OK;
}

statekv_status statekv_qcache_attend(const statekv_qcache* c, const statekv_qcache_attend_args* a,
                                     statekv_stream stream)
{
    Prepared d;
    if (!a || !prepared(c, &d) || !range_ok(*c, a->stream_begin, a->stream_count, a->layer_begin, a->layer_count) ||
        a->num_tokens < 0 || a->num_tokens > c->capacity || a->num_q_heads < 1 ||
        a->num_q_heads % c->num_kv_heads != 0 || (a->causal != 0 && a->causal != 1) || !(a->softmax_scale >= 0.f) ||
        !std::isfinite(a->softmax_scale))
        return STATEKV_ERR_INVALID_ARG;
    if (a->num_tokens == 0) return STATEKV_OK;
    if (!a->start || !aligned(a->start, 4) || !aligned(a->first, 4) || !a->q ||
        !a->out || !aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->lse, 4))
        return STATEKV_ERR_INVALID_ARG;
    const int G = a->num_q_heads / c->num_kv_heads;
    if (static_cast<long long>(a->num_tokens) * G > (1 << 24)) return STATEKV_ERR_UNSUPPORTED;
    const int U = a->stream_count * a->layer_count;
    const QAttendPlan plan = qcache_attend_plan(U, c->num_kv_heads, c->head_dim, c->capacity, a->num_tokens, G,
                                                current_sm_count());
    if (!plan.fits) return STATEKV_ERR_UNSUPPORTED;
    if (!a->workspace || !aligned(a->workspace, 256) || a->workspace_bytes < plan.bytes) return STATEKV_ERR_INVALID_ARG;
    QAttendParams p{};
    p.c = view_of(*c);
    p.units = UnitRange{a->stream_begin, a->layer_begin, a->layer_count, c->num_layers};
    p.U = U;
    p.n = a->num_tokens;
    p.Hq = a->num_q_heads;
    p.G = G;
    p.causal = a->causal;
    p.scale_log2 = (a->softmax_scale > 0.f ? a->softmax_scale : 1.0f / std::sqrt(static_cast<float>(c->head_dim))) *
                   1.4426950408889634f;
    p.start = a->start;
    p.first = a->first;
    p.q = static_cast<const __nv_bfloat16*>(a->q);
    p.out = static_cast<__nv_bfloat16*>(a->out);
    p.lse = a->lse;
    p.watchdog_ns = kWaitNs;
#if STATEKV_DEBUG_CHECKS
    // for the test of what follows an expired wait: one is taken as run out, the others' limit is this
    if (const char* ms = std::getenv("STATEKV_QCACHE_EXPIRE_MS")) {
        p.expire = 1;
        p.watchdog_ns = std::strtoull(ms, nullptr, 10) * 1000000ull;
    }
#endif
    return launch_qcache_attend(d.k, d.v, plan, p, static_cast<uint8_t*>(a->workspace),
                                reinterpret_cast<cudaStream_t>(stream)) == cudaSuccess ? STATEKV_OK : STATEKV_ERR_CUDA;
}

statekv_status statekv_qcache_sync(const statekv_qcache* c, statekv_stream stream)
{
    if (!prepared(c, nullptr)) return STATEKV_ERR_INVALID_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    int32_t word = 0;
    if (cudaMemcpyAsync(&word, c->status, 4, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess)
        return STATEKV_ERR_CUDA;
    if (word == 0) return STATEKV_OK;
    if (cudaMemsetAsync(c->status, 0, 4, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
        return STATEKV_ERR_CUDA;
    return (word & 0xFF) == DEV_QCACHE_FULL ? STATEKV_ERR_CACHE_FULL : STATEKV_ERR_DEVICE_TIMEOUT;
}

}  // extern "C"
