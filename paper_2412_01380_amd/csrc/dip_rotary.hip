// Rows turned to their positions (dip_rotate_rows), and on their way into the cache (dip_kv_append_rotary).
//
// A pair (a, b) of a head at position pos becomes s (a cos t - b sin t, a sin t + b cos t), t = pos * freq.  The angle
// is worked out in fp64, in turns, and reduced to the nearest half turn there: an fp32 product is off by 2^-24 of the
// angle, 0.06 at a million radians.  What is left fits fp32, and so do sine, cosine and the turned pair, which is
// rounded once.  Sines and cosines are worked out once for a row and pair, into LDS, whatever the number of heads.
//
// Bound by bytes, every element read and written once: 8192 rows of 40 heads of 128 dims, half of them turned, 168 MB in 39.9 us
// (34.7 at the rate of a large copy, 4.83 TB/s); 7095 rows of two prompts, 40 query heads and 10 for keys and values, 218 MB in 50.7
// us (45); both with inputs that change from call to call, and 28 and 35 us where the call before left them in the last-level
// cache.  Few rows by latency: 7 rows 7.1 us, three trees of 7 nodes into the cache 9.4, of which a launch takes 4.4; hence
// fewer rows to a workgroup then.

#include <cmath>

#include "dip_decode_internal.h"

namespace dip {
namespace {

constexpr int kThreads = 256;
constexpr int kAngles = 2048;             // sines and cosines of a workgroup: its rows times the pairs of a head

struct Turn {
    const double* freq;
    int pairs;
    float scale;
};

// (scale cos, scale sin) of `rows` rows, [row][pair]
template <typename F>
__device__ __forceinline__ void angles(const Turn& t, int rows, F pos_of, float2* out) {
    for (int i = threadIdx.x; i < rows * t.pairs; i += kThreads) {
        const int r = i / t.pairs, x = i - r * t.pairs;
        double turns = (double)pos_of(r) * t.freq[x] * 0.15915494309189533577;
        turns -= rint(turns);
        float s, c;
        sincospif(2.f * (float)turns, &s, &c);
        out[i] = make_float2(c * t.scale, s * t.scale);
    }
}

template <typename E, int V>
struct Vec {
    typedef E type __attribute__((ext_vector_type(V)));
};
template <typename E>
struct Vec<E, 1> {
    typedef E type;
};
template <typename E, int V>
__device__ __forceinline__ void load(const E* from, float (&f)[V]) {
    const auto x = *(const typename Vec<E, V>::type*)from;
    if constexpr (V == 1) f[0] = (float)x;
    else
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = (float)x[i];
}
template <typename E, int V>
__device__ __forceinline__ void store(E* to, const float (&f)[V]) {
    typename Vec<E, V>::type x;
    if constexpr (V == 1) x = (E)f[0];
    else
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (E)f[i];
    *(typename Vec<E, V>::type*)to = x;
}

// A head goes in pieces of V elements (the most that its pairs come in side by side, 16 bytes where that fits); a unit is
// two of them that belong together (half) or one (interleaved), and behind the turned dims one that passes through.
template <typename E, int V, bool INTER>
struct Units {
    static_assert(!INTER || V >= 2, "a pair lies within a piece");
    __device__ __forceinline__ static int turned(int pairs) { return INTER ? 2 * pairs / V : pairs / V; }
    __device__ __forceinline__ static int of_head(int pairs, int dims) { return turned(pairs) + (dims - 2 * pairs) / V; }
    // unit x of a head; cs: sines and cosines of its row, null: copied
    __device__ __forceinline__ static void go(const E* from, E* to, int x, int pairs, const float2* cs) {
        float a[V], b[V];
        if (x >= turned(pairs)) {
            const int at = 2 * pairs + (x - turned(pairs)) * V;
            load<E, V>(from + at, a);
            store<E, V>(to + at, a);
        } else if constexpr (INTER) {
            load<E, V>(from + x * V, a);
            if (cs) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float2 t = cs[(x * V + i) / 2];
                    b[i] = a[i] * t.x - a[i + 1] * t.y;
                    b[i + 1] = a[i] * t.y + a[i + 1] * t.x;
                }
                store<E, V>(to + x * V, b);
            } else {
                store<E, V>(to + x * V, a);
            }
        } else {
            load<E, V>(from + x * V, a);
            load<E, V>(from + pairs + x * V, b);
            if (cs) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float2 t = cs[x * V + i];
                    const float y = a[i] * t.x - b[i] * t.y;
                    b[i] = a[i] * t.y + b[i] * t.x;
                    a[i] = y;
                }
            }
            store<E, V>(to + x * V, a);
            store<E, V>(to + pairs + x * V, b);
        }
    }
};

struct RotateParams {
    Turn t;
    const char* x;
    char* out;
    int64_t x_stride;         // bytes
    int64_t out_stride;
    const int32_t* positions;
    int n_rows, n_heads, head_dim;
    int rows_per_wg;
};
template <typename E, int V, bool INTER>
__global__ void __launch_bounds__(kThreads) rotate_kernel(const RotateParams p) {
    __shared__ float2 s_cs[kAngles];
    typedef Units<E, V, INTER> U;
    const int r0 = blockIdx.x * p.rows_per_wg, rows = min(p.rows_per_wg, p.n_rows - r0);
    angles(p.t, rows, [&](int r) { return p.positions[r0 + r]; }, s_cs);
    __syncthreads();
    const int units = U::of_head(p.t.pairs, p.head_dim), wide = min(units, kThreads), side = kThreads / wide;
    const int mine = threadIdx.x / wide, n = mine < side ? rows * p.n_heads : 0;
    for (int x = threadIdx.x - mine * wide; x < units; x += wide)
        for (int i = mine; i < n; i += side) {
            const int r = i / p.n_heads, h = i - r * p.n_heads;
            U::go((const E*)(p.x + (int64_t)(r0 + r) * p.x_stride) + (int64_t)h * p.head_dim,
                  (E*)(p.out + (int64_t)(r0 + r) * p.out_stride) + (int64_t)h * p.head_dim, x, p.t.pairs, s_cs + r * p.t.pairs);
        }
}

struct AppendRotaryParams {
    KvView c;                 // k and v already at the layer
    BatchView b;
    const int32_t* parents;   // nullable
    Turn t;
    const char* q;
    char* q_out;
    const char* k_new;
    const char* v_new;
    int64_t q_stride;         // bytes
    int64_t q_out_stride;
    int64_t row_stride;
    int n_q_heads, head_dim;
    int rows_per_wg;
};
constexpr int kRows = 16;                 // most rows of a workgroup
template <typename E, int V, bool INTER>
__global__ void __launch_bounds__(kThreads) append_rotary_kernel(const AppendRotaryParams p) {
    __shared__ float2 s_cs[kAngles];
    __shared__ uint64_t s_tree[64];
    __shared__ int64_t s_place[kRows];
    typedef Units<E, V, INTER> U;
    const EntryRows er = entry_rows(p.b, blockIdx.x);
    const int t0 = blockIdx.y * p.rows_per_wg;
    if (t0 >= er.rows) return;
    const int seq = entry_seq(p.b, p.c, blockIdx.x);
    if (seq < 0) return;
    const int len = entry_len(p.c, seq), rows = min(p.rows_per_wg, er.rows - t0);
    const int32_t* table = p.c.table + (size_t)seq * p.c.max_pages;
    if (p.parents) {
        if (threadIdx.x < 64) tree_masks(p.parents + er.first, er.rows, s_tree);
        __syncthreads();
    }
    angles(p.t, rows, [&](int r) { return len + (p.parents ? max(0, (int)__popcll(s_tree[t0 + r]) - 1) : t0 + r); }, s_cs);
    const bool lacks = __syncthreads_or(lacks_room<kThreads>(p.c, table, len, er.rows));
    if (!lacks && (int)threadIdx.x < rows) {
        const int pos = len + t0 + threadIdx.x;
        s_place[threadIdx.x] = (table[pos >> p.c.page_shift] * p.c.page_stride + (pos & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride) * 16;
    }
    __syncthreads();
    const int heads = p.n_q_heads + (lacks ? 0 : 2 * p.c.n_heads);
    const int units = U::of_head(p.t.pairs, p.head_dim), wide = min(units, kThreads), side = kThreads / wide;
    const int mine = threadIdx.x / wide, n = mine < side ? rows * heads : 0;
    for (int x = threadIdx.x - mine * wide; x < units; x += wide)
        for (int i = mine; i < n; i += side) {
            const int r = i / heads;
            int h = i - r * heads;
            const int64_t row = er.first + t0 + r;
            const char* from;
            char* to;
            const float2* cs = s_cs + r * p.t.pairs;
            if (h < p.n_q_heads) {
                from = p.q + row * p.q_stride;
                to = p.q_out + row * p.q_out_stride + (int64_t)h * p.head_dim * (int)sizeof(E);
            } else {
                h -= p.n_q_heads;
                const bool value = h >= p.c.n_heads;
                if (value) {
                    h -= p.c.n_heads;
                    cs = nullptr;
                }
                from = (value ? p.v_new : p.k_new) + row * p.row_stride;
                to = (value ? p.c.v : p.c.k) + s_place[r] + h * p.c.head_stride * 16;
            }
            U::go((const E*)from + (int64_t)h * p.head_dim, (E*)to, x, p.t.pairs, cs);
        }
}

// The widest pieces that a head's pairs come in: 16 bytes, or as many elements as divide what lies side by side.
int piece_of(int dtype, int layout, int dims) {
    const int side = layout == DIP_ROTARY_HALF ? dims / 2 : dims;
    int v = dtype == DIP_F32 ? 4 : 8;
    while (side % v) v >>= 1;
    return v;
}
// Calls go(E(), V, INTER) as compile-time constants.
template <typename E, typename F>
hipError_t with_piece(int v, bool inter, F go) {
    using std::integral_constant;
    const auto pick = [&](auto width) {
        if (inter) {
            if constexpr (decltype(width)::value >= 2) return go(width, std::true_type());
        }
        return go(width, std::false_type());
    };
    if constexpr (sizeof(E) == 2)
        if (v == 8) return pick(integral_constant<int, 8>());
    if (v == 4) return pick(integral_constant<int, 4>());
    if (v == 2) return pick(integral_constant<int, 2>());
    return pick(integral_constant<int, 1>());
}

int32_t validate_rotary(const dip_rotary* r, int head_dim) {
    if (!r || !r->freq) return fail(DIP_ERR_INVALID_ARG, "rotary: null pointer");
    if (r->reserved) return fail(DIP_ERR_INVALID_ARG, "rotary: reserved must be 0");
    if (r->layout != DIP_ROTARY_HALF && r->layout != DIP_ROTARY_INTERLEAVED) return fail(DIP_ERR_INVALID_ARG, "rotary: layout %d", r->layout);
    if (r->dims < 2 || r->dims % 2 || r->dims > head_dim)
        return fail(DIP_ERR_INVALID_ARG, "rotary: dims must be even, in [2, %d], got %d", head_dim, r->dims);
    if (r->dims > DIP_MAX_ROTARY_DIMS) return fail(DIP_ERR_UNSUPPORTED, "rotary: more than %d dims", DIP_MAX_ROTARY_DIMS);
    if (!std::isfinite(r->scale)) return fail(DIP_ERR_INVALID_ARG, "rotary: scale must be finite");
    if (reinterpret_cast<uintptr_t>(r->freq) % 8) return fail(DIP_ERR_UNSUPPORTED, "rotary: freq must be 8-byte aligned");
    return DIP_OK;
}
// rows of a workgroup: 16 where that leaves enough workgroups for the chip, else fewer, and no more than LDS holds angles of
int rows_of(int64_t n_rows, int pairs) {
    int rows = kRows;
    while (rows > 1 && (n_rows / rows < 1024 || rows * pairs > kAngles)) rows >>= 1;
    return rows;
}

}  // namespace
}  // namespace dip

using namespace dip;

extern "C" {

int32_t dip_rotary_frequencies(int32_t dims, double base, const dip_rotary_scaling* scaling, double* freq) {
    if (!freq) return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: null pointer");
    if (dims < 2 || dims % 2) return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: dims must be even and >= 2");
    if (!std::isfinite(base) || base <= 0.0) return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: base must be finite and > 0");
    const int kind = scaling ? scaling->kind : DIP_SCALING_NONE;
    if (kind < DIP_SCALING_NONE || kind > DIP_SCALING_LIST) return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: scaling %d", kind);
    if (scaling && scaling->reserved) return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: reserved must be 0");
    const bool by_factor = kind == DIP_SCALING_LINEAR || kind == DIP_SCALING_BASE || kind == DIP_SCALING_PARTS;
    if (by_factor && !(std::isfinite(scaling->factor) && scaling->factor > 0.0))
        return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: factor must be finite and > 0");
    if (kind == DIP_SCALING_BASE && dims == 2) return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: a base is scaled by more than one pair");
    if (kind == DIP_SCALING_PARTS &&
        !(scaling->slow >= 0.0 && scaling->slow < scaling->fast && std::isfinite(scaling->fast) && scaling->original_len > 0.0 && std::isfinite(scaling->original_len)))
        return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: 0 <= slow < fast and original_len > 0 are needed");
    if (kind == DIP_SCALING_LIST) {
        if (!scaling->factors) return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: no list of factors");
        for (int i = 0; i < dims / 2; ++i)
            if (!(std::isfinite(scaling->factors[i]) && scaling->factors[i] > 0.0))
                return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: factor %d must be finite and > 0", i);
    }
    if (kind == DIP_SCALING_BASE) base *= std::pow(scaling->factor, (double)dims / (dims - 2));
    const auto angle = [&](int i) {
        double f = std::pow(base, -2.0 * i / dims);
        if (kind == DIP_SCALING_LINEAR) f /= scaling->factor;
        if (kind == DIP_SCALING_LIST) f /= scaling->factors[i];
        if (kind == DIP_SCALING_PARTS) {
            const double turns = scaling->original_len * f / 6.28318530717958647693;
            double m = (turns - scaling->slow) / (scaling->fast - scaling->slow);
            m = m < 0.0 ? 0.0 : m > 1.0 ? 1.0 : m;
            f = f * m + f / scaling->factor * (1.0 - m);
        }
        return f;
    };
    bool fits = std::isfinite(base) && base > 0.0;
    for (int i = 0; i < dims / 2; ++i) fits &= std::isfinite(angle(i));
    if (!fits) return fail(DIP_ERR_INVALID_ARG, "rotary_frequencies: base and scaling lead beyond the finite numbers");
    for (int i = 0; i < dims / 2; ++i) freq[i] = angle(i);
    return DIP_OK;
}

int32_t dip_rotate_rows(const dip_rotary* rot, const void* x, int64_t x_stride, const int32_t* positions, int32_t n_rows,
                        int32_t n_heads, int32_t head_dim, int32_t dtype, void* out, int64_t out_stride, void* stream) {
    if (!x || !positions || !out) return fail(DIP_ERR_INVALID_ARG, "rotate_rows: null pointer");
    if (dtype != DIP_F32 && dtype != DIP_BF16) return fail(DIP_ERR_UNSUPPORTED, "rotate_rows: dtype %d", dtype);
    const int es = elem_bytes(dtype), per = 16 / es;
    if (n_rows < 1 || n_heads < 1 || head_dim < 1) return fail(DIP_ERR_INVALID_ARG, "rotate_rows: sizes must be >= 1");
    if (n_rows >= 1 << 24 || n_heads > 65535 || head_dim > 65536)
        return fail(DIP_ERR_UNSUPPORTED, "rotate_rows: 2^24 rows, more than 65535 heads or 65536 dims");
    if (head_dim % per) return fail(DIP_ERR_UNSUPPORTED, "rotate_rows: head_dim must be a multiple of %d", per);
    int32_t st = validate_rotary(rot, head_dim);
    if (st) return st;
    const int64_t width = (int64_t)n_heads * head_dim;
    if (x_stride < width || out_stride < width) return fail(DIP_ERR_INVALID_ARG, "rotate_rows: strides smaller than a row");
    if (x_stride % per || out_stride % per || !aligned16(x) || !aligned16(out))
        return fail(DIP_ERR_UNSUPPORTED, "rotate_rows: rows must start on 16-byte boundaries");
    if (!(x == out && (x_stride == out_stride || n_rows == 1)) && rows_overlap(x, x_stride * es, width * es, out, out_stride * es, width * es, n_rows))
        return fail(DIP_ERR_INVALID_ARG, "rotate_rows: out overlaps x without being it");
    RotateParams p;
    p.t = {rot->freq, rot->dims / 2, rot->scale};
    p.x = (const char*)x;
    p.out = (char*)out;
    p.x_stride = x_stride * es;
    p.out_stride = out_stride * es;
    p.positions = positions;
    p.n_rows = n_rows;
    p.n_heads = n_heads;
    p.head_dim = head_dim;
    p.rows_per_wg = rows_of(n_rows, p.t.pairs);
    const dim3 grid((unsigned)((n_rows + p.rows_per_wg - 1) / p.rows_per_wg));
    const int v = piece_of(dtype, rot->layout, rot->dims);
    const bool inter = rot->layout == DIP_ROTARY_INTERLEAVED;
    const auto go = [&](auto e) {
        typedef decltype(e) E;
        return with_piece<E>(v, inter, [&](auto width, auto is_inter) {
            return launch_timed(rotate_kernel<E, decltype(width)::value, decltype(is_inter)::value>, grid, dim3(kThreads), (hipStream_t)stream,
                                DIP_KERNEL_ROTARY, p);
        });
    };
    return check_hip(dtype == DIP_F32 ? go(float()) : go(__bf16()), "rotate_rows launch");
}

int32_t dip_kv_append_rotary(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const int32_t* parents,
                             const dip_rotary* rot, const void* q, int64_t q_stride, int32_t n_q_heads, void* q_out,
                             int64_t q_out_stride, const void* k_new, const void* v_new, int64_t row_stride, void* stream) {
    int32_t st = validate_kv(cache);
    if (!st) st = validate_batch(batch, true);
    if (!st) st = validate_rotary(rot, cache->head_dim);
    if (st) return st;
    if (layer < 0 || layer >= cache->n_layers) return fail(DIP_ERR_INVALID_ARG, "append_rotary: layer %d of %d", layer, cache->n_layers);
    if (!k_new || !v_new) return fail(DIP_ERR_INVALID_ARG, "append_rotary: null rows");
    if (n_q_heads < 0 || (n_q_heads > 0) != (q != nullptr) || (n_q_heads > 0) != (q_out != nullptr))
        return fail(DIP_ERR_INVALID_ARG, "append_rotary: q, q_out and n_q_heads go together");
    if (n_q_heads > 65535) return fail(DIP_ERR_UNSUPPORTED, "append_rotary: more than 65535 query heads");
    if (parents && rows_bound(batch) > DIP_MAX_TREE) return fail(DIP_ERR_UNSUPPORTED, "append_rotary: a tree has at most %d nodes", DIP_MAX_TREE);
    const int es = elem_bytes(cache->dtype), per = 16 / es;
    const int64_t q_width = (int64_t)n_q_heads * cache->head_dim, width = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (row_stride < width || (n_q_heads && (q_stride < q_width || q_out_stride < q_width)))
        return fail(DIP_ERR_INVALID_ARG, "append_rotary: strides smaller than a row");
    if (row_stride % per || !aligned16(k_new) || !aligned16(v_new) || (n_q_heads && (q_stride % per || q_out_stride % per || !aligned16(q) || !aligned16(q_out))))
        return fail(DIP_ERR_UNSUPPORTED, "append_rotary: rows must start on 16-byte boundaries");
    const auto meets = [&](const void* x, int64_t stride, int64_t w) {
        return rows_overlap(x, stride * es, w * es, q_out, q_out_stride * es, q_width * es, batch->n_rows);
    };
    if (n_q_heads && !(q == q_out && (q_stride == q_out_stride || batch->n_rows == 1)) && meets(q, q_stride, q_width))
        return fail(DIP_ERR_INVALID_ARG, "append_rotary: q_out overlaps q without being it");
    if (n_q_heads && (meets(k_new, row_stride, width) || meets(v_new, row_stride, width)))
        return fail(DIP_ERR_INVALID_ARG, "append_rotary: q_out overlaps the new keys or values");
    AppendRotaryParams p;
    p.c = view_of(cache);
    p.c.k += p.c.layer_stride * layer * 16;
    p.c.v += p.c.layer_stride * layer * 16;
    p.b = view_of(batch);
    p.parents = parents;
    p.t = {rot->freq, rot->dims / 2, rot->scale};
    p.q = (const char*)q;
    p.q_out = (char*)q_out;
    p.k_new = (const char*)k_new;
    p.v_new = (const char*)v_new;
    p.q_stride = q_stride * es;
    p.q_out_stride = q_out_stride * es;
    p.row_stride = row_stride * es;
    p.n_q_heads = n_q_heads;
    p.head_dim = cache->head_dim;
    p.rows_per_wg = rows_of(batch->n_rows, p.t.pairs);
    const int64_t blocks = (p.b.max_rows + p.rows_per_wg - 1) / p.rows_per_wg;
    if (blocks > 65535) return fail(DIP_ERR_UNSUPPORTED, "append_rotary: max_rows is too large for one call");
    const dim3 grid(batch->n_batch, (unsigned)blocks);
    const int v = piece_of(cache->dtype, rot->layout, rot->dims);
    const bool inter = rot->layout == DIP_ROTARY_INTERLEAVED;
    const auto go = [&](auto e) {
        typedef decltype(e) E;
        return with_piece<E>(v, inter, [&](auto width, auto is_inter) {
            return launch_timed(append_rotary_kernel<E, decltype(width)::value, decltype(is_inter)::value>, grid, dim3(kThreads),
                                (hipStream_t)stream, DIP_KERNEL_ROTARY, p);
        });
    };
    return check_hip(cache->dtype == DIP_F32 ? go(float()) : go(__bf16()), "append_rotary launch");
}

}  // extern "C"
