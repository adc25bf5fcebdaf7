// Attention over a paged key/value cache: dip_window_attention, dip_tree_attention.
//
// First form: one wavefront per (row, query head), one key at a time, the running maximum and sum
// of the softmax in fp32.

#include <cmath>

#include "dip_decode_internal.h"

namespace dip {
namespace {

constexpr int kThreads = 256;

struct AttnParams {
    KvView c;
    BatchView b;
    const int32_t* parents;   // null: window attention
    const char* q;
    char* out;
    int64_t q_stride;         // elements
    int64_t out_stride;
    int64_t layer_offset;     // 16-byte pieces
    int layer;
    int n_q_heads;
    int group;
    int head_dim;
    float scale;
    int window;
    int sinks;
    int max_len;
};

template <typename E>
__device__ __forceinline__ float widen(E x);
template <>
__device__ __forceinline__ float widen<float>(float x) { return x; }
template <>
__device__ __forceinline__ float widen<uint16_t>(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <typename E>
__device__ __forceinline__ E narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ uint16_t narrow<uint16_t>(float x) {
    const uint32_t u = __float_as_uint(x);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (uint16_t)((u >> 16) | 0x40);
    return (uint16_t)((u + 0x7fff + ((u >> 16) & 1)) >> 16);
}

template <typename E>
__global__ void __launch_bounds__(kThreads) attn_simple_kernel(const AttnParams p) {
    const int lane = threadIdx.x & 63;
    const int head = blockIdx.z * (kThreads / 64) + (threadIdx.x >> 6);
    const EntryRows er = entry_rows(p.b, blockIdx.x);
    const int t = blockIdx.y;
    if (head >= p.n_q_heads || t >= er.rows) return;
    const int row = er.first + t;
    const int seq = entry_seq(p.b, p.c, blockIdx.x);
    const int len = seq >= 0 ? min(entry_len(p.c, seq), p.max_len) : 0;
    uint64_t anc = 0;
    int depth = t;
    if (p.parents) {
        anc = 0;
        depth = -1;
        for (int a = t; a >= 0;) {
            anc |= 1ull << a;
            ++depth;
            const int up = p.parents[er.first + a];
            if (up < -1 || up >= a) { anc = 0; break; }
            a = up;
        }
    }
    const int pos = len + depth;
    const int lo = p.window ? max(0, pos - p.window + 1) : 0;
    const int total = seq < 0 || (p.parents && !anc) ? 0 : min(len + (p.parents ? er.rows : t + 1), p.max_len);
    constexpr int PER = 2;                            // dims of a lane: lane, lane + 64
    float qv[PER], acc[PER];
    const E* q = (const E*)p.q + row * p.q_stride + head * p.head_dim;
    for (int i = 0; i < PER; ++i) {
        const int d = lane + 64 * i;
        qv[i] = d < p.head_dim ? widen(q[d]) * p.scale : 0.f;
        acc[i] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    for (int j = 0; j < total; ++j) {
        const bool sees = j < len || !p.parents ? j >= lo || j < p.sinks : (anc >> (j - len)) & 1;
        if (!sees) continue;
        int page = p.c.table[(size_t)seq * p.c.max_pages + (j >> p.c.page_shift)];
        if ((unsigned)page >= (unsigned)p.c.n_pages) page = 0;
        const int64_t at = 16 / (int64_t)sizeof(E) * (p.layer * p.c.layer_stride + page * p.c.page_stride +
                           (head / p.group) * p.c.head_stride + (j & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride);
        const E* k = (const E*)p.c.k + at;
        const E* v = (const E*)p.c.v + at;
        float z = 0.f;
        for (int i = 0; i < PER; ++i)
            if (lane + 64 * i < p.head_dim) z = fmaf(qv[i], widen(k[lane + 64 * i]), z);
        for (int off = 32; off; off >>= 1) z += __shfl_xor(z, off);
        const float m2 = fmaxf(m, z), w = __expf(z - m2), old = __expf(m - m2);
        l = l * old + w;
        for (int i = 0; i < PER; ++i)
            if (lane + 64 * i < p.head_dim) acc[i] = acc[i] * old + w * widen(v[lane + 64 * i]);
        m = m2;
    }
    E* out = (E*)p.out + row * p.out_stride + head * p.head_dim;
    for (int i = 0; i < PER; ++i)
        if (lane + 64 * i < p.head_dim) out[lane + 64 * i] = narrow<E>(l > 0.f ? acc[i] / l : l == 0.f ? 0.f : l);
}

int32_t check_attention(const dip_kv_cache* c, const dip_batch* b, int32_t n_q_heads, int32_t window, int32_t sinks) {
    int32_t st = validate_kv(c);
    if (!st) st = validate_batch(b, true);
    if (st) return st;
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128)
        return fail(DIP_ERR_UNSUPPORTED, "attention: head_dim %d is none of 64, 96, 128", c->head_dim);
    if (n_q_heads < 1 || n_q_heads % c->n_kv_heads)
        return fail(DIP_ERR_INVALID_ARG, "attention: %d query heads are no multiple of %d", n_q_heads, c->n_kv_heads);
    if (n_q_heads > 65535) return fail(DIP_ERR_UNSUPPORTED, "attention: more than 65535 query heads");
    if (window < 0 || sinks < 0) return fail(DIP_ERR_INVALID_ARG, "attention: window and sinks must be >= 0");
    return DIP_OK;
}

int32_t attend(const dip_kv_cache* c, int32_t layer, const dip_batch* b, const int32_t* parents, const void* q, int64_t q_stride,
               int32_t n_q_heads, float scale, int32_t window, int32_t sinks, void* out, int64_t out_stride, void* ws, size_t ws_bytes,
               void* stream) {
    int32_t st = check_attention(c, b, n_q_heads, window, sinks);
    if (st) return st;
    if (layer < 0 || layer >= c->n_layers) return fail(DIP_ERR_INVALID_ARG, "attention: layer %d of %d", layer, c->n_layers);
    if (!q || !out) return fail(DIP_ERR_INVALID_ARG, "attention: null pointer");
    if (!std::isfinite(scale) || scale <= 0.f) return fail(DIP_ERR_INVALID_ARG, "attention: scale must be finite and > 0");
    const int es = elem_bytes(c->dtype);
    const int64_t width = (int64_t)n_q_heads * c->head_dim;
    if (q_stride < width || out_stride < width) return fail(DIP_ERR_INVALID_ARG, "attention: strides smaller than a row");
    if (q_stride * es % 16 || out_stride * es % 16 || !aligned16(q) || !aligned16(out))
        return fail(DIP_ERR_UNSUPPORTED, "attention: rows of q and out must start on 16-byte boundaries");
    st = validate_ws(ws, ws_bytes, dip_attention_workspace_bytes(c, b, n_q_heads, window, sinks));
    if (st) return st;
    AttnParams p;
    p.c = view_of(c);
    p.b = view_of(b);
    p.parents = parents;
    p.q = (const char*)q;
    p.out = (char*)out;
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.layer = layer;
    p.n_q_heads = n_q_heads;
    p.group = n_q_heads / c->n_kv_heads;
    p.head_dim = c->head_dim;
    p.scale = scale;
    p.window = window;
    p.sinks = sinks;
    const int fit = c->max_pages * c->page_size;
    p.max_len = b->max_len && b->max_len < fit ? b->max_len : fit;
    const dim3 grid(b->n_batch, p.b.max_rows, (n_q_heads + 3) / 4);
    if (c->dtype == DIP_F32)
        return check_hip(launch_timed(attn_simple_kernel<float>, grid, dim3(kThreads), (hipStream_t)stream, DIP_KERNEL_ATTENTION, p), "attention launch");
    return check_hip(launch_timed(attn_simple_kernel<uint16_t>, grid, dim3(kThreads), (hipStream_t)stream, DIP_KERNEL_ATTENTION, p), "attention launch");
}

}  // namespace
}  // namespace dip

using namespace dip;

extern "C" {

size_t dip_attention_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch, int32_t n_q_heads, int32_t window, int32_t sinks) {
    if (check_attention(cache, batch, n_q_heads, window, sinks)) return 0;
    return 256;
}

int32_t dip_window_attention(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const void* q, int64_t q_stride,
                             int32_t n_q_heads, float scale, int32_t window, int32_t sinks, void* out, int64_t out_stride, void* ws,
                             size_t ws_bytes, void* stream) {
    return attend(cache, layer, batch, nullptr, q, q_stride, n_q_heads, scale, window, sinks, out, out_stride, ws, ws_bytes, stream);
}

int32_t dip_tree_attention(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const int32_t* parents, const void* q,
                           int64_t q_stride, int32_t n_q_heads, float scale, int32_t window, int32_t sinks, void* out,
                           int64_t out_stride, void* ws, size_t ws_bytes, void* stream) {
    if (!parents) return fail(DIP_ERR_INVALID_ARG, "tree_attention: null parents");
    if (batch && batch->max_rows > DIP_MAX_TREE && batch->n_rows > DIP_MAX_TREE)
        return fail(DIP_ERR_UNSUPPORTED, "tree_attention: a tree has at most %d nodes", DIP_MAX_TREE);
    return attend(cache, layer, batch, parents, q, q_stride, n_q_heads, scale, window, sinks, out, out_stride, ws, ws_bytes, stream);
}

}  // extern "C"
