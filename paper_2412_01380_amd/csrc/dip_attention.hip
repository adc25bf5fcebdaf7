// Attention over a paged key/value cache: dip_window_attention, dip_tree_attention.
//
// The rows of an entry that share a key/value head -- its tokens or nodes times the query heads of the
// group -- form blocks of 16, 32 or 64; a workgroup takes a block and a share of the keys that it sees.

#include <cmath>

#include "dip_attn_device.h"

namespace dip {
namespace attn {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kIds = 1024;                // page numbers of a share, in LDS
constexpr int kRing = 2;                  // tiles of a wavefront in LDS: one in use, one on its way

// Every wavefront streams tiles of its own through LDS (no barrier in the loop) and keeps a softmax of its
// own; they are joined in LDS at the end.
template <typename E, int D, int NB>
__global__ void __launch_bounds__(kThreads, 1) attn_rows_kernel(const AttnParams p) {
    typedef Geo<E, D> G;
    typedef Core<E, D, NB> C;
    constexpr int KEYS = G::KEYS, TILE = KEYS * G::ROWB, LOADS = TILE / 1024, ROWS = 16 * NB;
    static_assert(TILE % 1024 == 0, "whole loads");
    __shared__ __align__(1024) char s_ring[kWaves * kRing * 2 * TILE];
    __shared__ int s_ids[kIds];
    __shared__ uint64_t s_tree[64];
    __shared__ float s_m[kWaves][ROWS], s_l[kWaves][ROWS];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int split = blockIdx.x % p.splits;
    const int block = blockIdx.x / p.splits;             // (entry, head, block of rows)
    const int rb = block % p.row_blocks;
    const int head = block / p.row_blocks % p.c.n_heads;
    const int e = block / p.row_blocks / p.c.n_heads;

    const EntryRows er = entry_rows(p.b, e);
    const int r0 = rb * ROWS, n_rows = min(ROWS, er.rows * p.group - r0);
    if (n_rows <= 0) return;
    const int seq = entry_seq(p.b, p.c, e);
    const int len = seq >= 0 ? min(entry_len(p.c, seq), p.max_len) : 0;
    Range range = key_range<KEYS>(p, len, er.rows, r0 / p.group, (r0 + n_rows - 1) / p.group);
    if (seq < 0) range.tiles = 0;
    const int shares = (range.tiles + p.tiles_per_split - 1) / p.tiles_per_split;
    const int begin = split * p.tiles_per_split, end = min(range.tiles, begin + p.tiles_per_split);
    if (begin >= end && split > 0) return;

    // the share's page numbers, `per` of a tile
    const int shift = p.c.page_shift;
    const int per = max(1, KEYS >> shift);
    for (int i = tid; i < (end - begin) * per; i += kThreads) {
        const int vt = i / per;
        const int at = ((tile_at(range, begin + vt) * KEYS) >> shift) + (i - vt * per);
        int page = at < p.c.max_pages ? p.c.table[(size_t)seq * p.c.max_pages + at] : 0;
        s_ids[i] = (unsigned)page < (unsigned)p.c.n_pages ? page : 0;
    }
    if (p.parents && wave == 0) tree_masks(p.parents + er.first, er.rows, s_tree);
    __syncthreads();

    C core;
    RowSees row[NB];
    bool alive[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = r0 + 16 * nb + (lane & 15);
        const bool is = r < r0 + n_rows;
        const int t = is ? r / p.group : 0;
        row[nb] = row_sees(p, len, t, s_tree);
        alive[nb] = is && (row[nb].hi > 0 || row[nb].tree);
        core.load_q(nb, is ? p.q + (int64_t)(er.first + t) * p.q_stride + (int64_t)(head * p.group + r % p.group) * (D * G::ES) : nullptr);
    }
    Softmax<E, D, NB> soft;
    soft.start(core);

    const char* kbase = p.c.k + p.c.head_stride * head * 16;
    const char* vbase = p.c.v + p.c.head_stride * head * 16;
    const lds_char* ring = (const lds_char*)s_ring + wave * (kRing * 2 * TILE);
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_offset(s_ring) + wave * (kRing * 2 * TILE));
    const int mine = max(0, (end - begin - wave + kWaves - 1) / kWaves);

    auto fetch = [&](int i) {
        const int vt = begin + wave + kWaves * i, j0 = tile_at(range, vt) * KEYS;
        const uint32_t to = ring_at + (i & (kRing - 1)) * (2 * TILE);
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int at = x * 64 + lane, r = at / G::CPR;
            const int pos = min(j0 + r, range.end - 1);
            const int page = s_ids[(vt - begin) * per + ((pos >> shift) - (j0 >> shift))];
            const int64_t off = (page * p.c.page_stride + (pos & ((1 << shift) - 1)) * p.c.slot_stride + G::piece(r, at % G::CPR)) * 16;
            load_to_lds(kbase + off, to + x * 1024);
            load_to_lds(vbase + off, to + TILE + x * 1024);
        }
    };
    // V's pieces that are not finite become zero, for a weight of zero to take them out; the keys' bits
    auto take_out = [&](lds_char* v) {
        uint32_t bad = 0;
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            auto* at = (__attribute__((address_space(3))) u32x4*)(v + x * 1024 + lane * 16);
            const u32x4 w = *at;
            bool inf = false;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                if constexpr (sizeof(E) == 4) inf |= (w[y] & 0x7f800000u) == 0x7f800000u;
                else inf |= (w[y] & 0x7f800000u) == 0x7f800000u || (w[y] & 0x7f80u) == 0x7f80u;
            }
            if (inf) {
                *at = u32x4{0, 0, 0, 0};
                bad |= 1u << ((x * 64 + lane) / G::CPR);
            }
        }
        if (__any(bad))
            for (int off = 1; off < 64; off <<= 1) bad |= __shfl_xor(bad, off);
        asm volatile("" ::: "memory");
        return bad;
    };

    if (mine > 0) fetch(0);
    if (mine > 1) fetch(1);
    for (int i = 0; i < mine; ++i) {
        if (i + 1 < mine) wait_loads<2 * LOADS>(); else wait_loads<0>();
        const int j0 = tile_at(range, begin + wave + kWaves * i) * KEYS;
        const lds_char* kt = ring + (i & (kRing - 1)) * (2 * TILE);
        f32x4 s[NB][C::MT];
        core.scores(kt, s);
        const bool whole = j0 + KEYS <= range.sure && (j0 >= range.from || j0 + KEYS <= p.sinks);
        if (!whole) {
            const uint32_t bad = take_out((lds_char*)kt + TILE);
            const int g = lane >> 4;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int x = 0; x < 4 * C::MT; ++x) {
                    const int key = 16 * (x >> 2) + 4 * g + (x & 3);
                    float z = (bad >> key) & 1 ? NAN : s[nb][x >> 2][x & 3];
                    if (!sees(row[nb], j0 + key, p.sinks, len)) z = -INFINITY;
                    s[nb][x >> 2][x & 3] = z;
                }
        }
        soft.step(core, s, p.scale_log2);
        core.template add_values<true>(kt + TILE, s);
        if (i + kRing < mine) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (everything read from the tile that goes)
            fetch(i + kRing);
        }
    }

    // join the wavefronts
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const float l = column_sum(soft.l[nb]);
        if (lane < 16) {
            s_m[wave][16 * nb + lane] = alive[nb] ? soft.m[nb] : -INFINITY;
            s_l[wave][16 * nb + lane] = alive[nb] ? l : 0.f;
        }
    }
    __syncthreads();                                      // (and every wavefront is done with its tiles)
    constexpr int QUADS = D / 4;
    float* s_o = (float*)s_ring;                          // [wave][row][quad, rotated by the row][4]
    static_assert(kWaves * ROWS * D * 4 <= (int)sizeof(s_ring), "the joined rows fit the ring");
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = 16 * nb + (lane & 15);
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
        const float a = s_m[wave][r] == -INFINITY ? 0.f : fast_exp2(s_m[wave][r] - top);
#pragma unroll
        for (int y = 0; y < C::OB; ++y) {
            const int quad = C::quad_dim(y) / 4;
            *(f32x4*)(s_o + ((wave * ROWS + r) * QUADS + (quad + r) % QUADS) * 4) = core.quad(nb, y) * a;
        }
    }
    __syncthreads();
    for (int i = tid; i < n_rows * QUADS; i += kThreads) {
        const int r = i / QUADS, quad = i % QUADS;
        float top = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) l += s_m[w][r] == -INFINITY ? (s_l[w][r] == 0.f ? 0.f : s_l[w][r]) : s_l[w][r] * fast_exp2(s_m[w][r] - top);
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) o += *(const f32x4*)(s_o + ((w * ROWS + r) * QUADS + (quad + r) % QUADS) * 4);
        if (shares > 1) {
            const size_t at = ((size_t)block * p.splits + split) * ROWS + r;
            *(f32x4*)(p.part_o + at * D + quad * 4) = o;
            if (quad == 0) p.part_ml[at] = make_float2(top, l);
        } else {
            const int t = (r0 + r) / p.group, h = head * p.group + (r0 + r) % p.group;
            const f32x4 zero = {0, 0, 0, 0};
            store_quad<E>(p.out + (int64_t)(er.first + t) * p.out_stride + (int64_t)h * (D * G::ES), quad * 4, l == 0.f ? zero : o / l);
        }
    }
}

// Shares of one row joined: 8 rows of a block to a workgroup of 256, four dims to a thread.
constexpr int kJoinRows = 8;
template <typename E, int D, int KEYS>
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnParams p, const int rows_of_block) {
    constexpr int QUADS = D / 4;
    const int block = blockIdx.x;
    const int rb = block % p.row_blocks;
    const int head = block / p.row_blocks % p.c.n_heads;
    const int e = block / p.row_blocks / p.c.n_heads;
    const EntryRows er = entry_rows(p.b, e);
    const int r0 = rb * rows_of_block, n_rows = min(rows_of_block, er.rows * p.group - r0);
    if (n_rows <= (int)blockIdx.y * kJoinRows) return;
    const int seq = entry_seq(p.b, p.c, e);
    if (seq < 0) return;
    const int len = min(entry_len(p.c, seq), p.max_len);
    const Range range = key_range<KEYS>(p, len, er.rows, r0 / p.group, (r0 + n_rows - 1) / p.group);
    const int shares = (range.tiles + p.tiles_per_split - 1) / p.tiles_per_split;
    if (shares <= 1) return;
    for (int i = threadIdx.x; i < kJoinRows * QUADS; i += 256) {
        const int r = blockIdx.y * kJoinRows + i / QUADS, quad = i % QUADS;
        if (r >= n_rows) break;
        const size_t at = (size_t)block * p.splits * rows_of_block + r;
        float top = -INFINITY;
        for (int s = 0; s < shares; ++s) top = fmaxf(top, p.part_ml[at + (size_t)s * rows_of_block].x);
        f32x4 o = {0, 0, 0, 0};
        float l = 0.f;
#pragma unroll 4
        for (int s = 0; s < shares; ++s) {
            const float2 ml = p.part_ml[at + (size_t)s * rows_of_block];
            const f32x4 x = *(const f32x4*)(p.part_o + (at + (size_t)s * rows_of_block) * D + quad * 4);
            const float a = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - top);
            if (ml.x != -INFINITY || ml.y != 0.f) {
                l += ml.x == -INFINITY ? ml.y : ml.y * a;
                o += x * a;
            }
        }
        const int t = (r0 + r) / p.group, h = head * p.group + (r0 + r) % p.group;
        const f32x4 zero = {0, 0, 0, 0};
        store_quad<E>(p.out + (int64_t)(er.first + t) * p.out_stride + (int64_t)h * (D * (int)sizeof(E)), quad * 4, l == 0.f ? zero : o / l);
    }
}

// ---- launch plan ----------------------------------------------------------------------------------
struct Plan {
    int nb, row_blocks, splits, tiles_per_split;
    int64_t blocks;
    size_t off_ml, total;
};
int reach(const dip_kv_cache* c, const dip_batch* b) {
    const int fit = c->max_pages * c->page_size;
    return b->max_len && b->max_len < fit ? b->max_len : fit;
}
Plan plan_attention(const dip_kv_cache* c, const dip_batch* b, int n_q_heads, int window, int sinks) {
    Plan pl;
    const int keys = c->dtype == DIP_F32 ? 16 : 32;
    const int64_t rows = (int64_t)rows_bound(b) * (n_q_heads / c->n_kv_heads);
    pl.nb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    pl.row_blocks = (int)((rows + 16 * pl.nb - 1) / (16 * pl.nb));
    pl.blocks = (int64_t)b->n_batch * c->n_kv_heads * pl.row_blocks;
    // most tiles that a block of rows sees
    const int64_t all = ((int64_t)reach(c, b) + keys - 1) / keys;
    int64_t tiles = all;
    if (window) {
        const int64_t w = ((int64_t)sinks + keys - 1) / keys + ((int64_t)window + rows_bound(b)) / keys + 2;
        if (w < tiles) tiles = w;
    }
    // enough workgroups for the chip, but no share under two tiles a wavefront, and none with more page
    // numbers than LDS holds
    int64_t want = (512 + pl.blocks - 1) / pl.blocks;
    int64_t per = (tiles + want - 1) / want;
    if (per < 2 * kWaves) per = 2 * kWaves;
    per = (per + kWaves - 1) / kWaves * kWaves;
    const int ids = keys / c->page_size > 1 ? keys / c->page_size : 1;
    if (per > kIds / ids) per = kIds / ids;
    pl.tiles_per_split = (int)per;
    pl.splits = (int)((tiles + per - 1) / per);
    if (pl.splits < 1) pl.splits = 1;
    size_t o = 0;
    if (pl.splits > 1) {
        const size_t rows_all = (size_t)pl.blocks * pl.splits * 16 * pl.nb;
        o = align_up(rows_all * c->head_dim * sizeof(float), 256);
        pl.off_ml = o;
        o += align_up(rows_all * sizeof(float2), 256);
    } else {
        pl.off_ml = 0;
    }
    pl.total = o < 256 ? 256 : o;
    return pl;
}

template <typename E, int D>
int32_t launch(const AttnParams& p, const Plan& pl, hipStream_t stream) {
    const dim3 grid((unsigned)(pl.blocks * pl.splits));
    hipError_t err;
    if (pl.nb == 1) err = launch_timed(attn_rows_kernel<E, D, 1>, grid, dim3(kThreads), stream, DIP_KERNEL_ATTENTION, p);
    else if (pl.nb == 2) err = launch_timed(attn_rows_kernel<E, D, 2>, grid, dim3(kThreads), stream, DIP_KERNEL_ATTENTION, p);
    else err = launch_timed(attn_rows_kernel<E, D, 4>, grid, dim3(kThreads), stream, DIP_KERNEL_ATTENTION, p);
    int32_t st = check_hip(err, "attention launch");
    if (st || pl.splits == 1) return st;
    hipEvent_t e0, e1;
    const dim3 jgrid((unsigned)pl.blocks, 16 * pl.nb / kJoinRows);
    if (prof_next(DIP_KERNEL_ATTENTION_JOIN, &e0, &e1))
        hipExtLaunchKernelGGL((attn_join_kernel<E, D, Geo<E, D>::KEYS>), jgrid, dim3(256), 0, stream, e0, e1, 0, p, 16 * pl.nb);
    else
        hipLaunchKernelGGL((attn_join_kernel<E, D, Geo<E, D>::KEYS>), jgrid, dim3(256), 0, stream, p, 16 * pl.nb);
    return check_hip(hipGetLastError(), "attention join launch");
}
template <typename E>
int32_t launch_dim(const AttnParams& p, const Plan& pl, int head_dim, hipStream_t stream) {
    if (head_dim == 64) return launch<E, 64>(p, pl, stream);
    if (head_dim == 96) return launch<E, 96>(p, pl, stream);
    return launch<E, 128>(p, pl, stream);
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
    const int64_t rows = (int64_t)rows_bound(b) * (n_q_heads / c->n_kv_heads);
    if (rows >= 1 << 30) return fail(DIP_ERR_UNSUPPORTED, "attention: too many rows of one entry");
    const Plan pl = plan_attention(c, b, n_q_heads, window, sinks);
    if (pl.blocks * pl.splits >= (int64_t)1 << 31) return fail(DIP_ERR_UNSUPPORTED, "attention: too many rows for one call");
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
    const Plan pl = plan_attention(c, b, n_q_heads, window, sinks);
    st = validate_ws(ws, ws_bytes, pl.total);
    if (st) return st;
    AttnParams p;
    p.c = view_of(c);
    p.c.k += p.c.layer_stride * layer * 16;
    p.c.v += p.c.layer_stride * layer * 16;
    p.b = view_of(b);
    p.parents = parents;
    p.q = (const char*)q;
    p.out = (char*)out;
    p.q_stride = q_stride * es;
    p.out_stride = out_stride * es;
    p.n_q_heads = n_q_heads;
    p.group = n_q_heads / c->n_kv_heads;
    p.scale_log2 = scale * 1.44269504088896340736f;
    p.window = window;
    p.sinks = sinks;
    p.max_len = reach(c, b);
    p.splits = pl.splits;
    p.tiles_per_split = pl.tiles_per_split;
    p.row_blocks = pl.row_blocks;
    p.part_o = (float*)ws;
    p.part_ml = (float2*)((char*)ws + pl.off_ml);
    return c->dtype == DIP_F32 ? launch_dim<float>(p, pl, c->head_dim, (hipStream_t)stream)
                               : launch_dim<uint16_t>(p, pl, c->head_dim, (hipStream_t)stream);
}

}  // namespace
}  // namespace attn
}  // namespace dip

using namespace dip;

extern "C" {

size_t dip_attention_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch, int32_t n_q_heads, int32_t window, int32_t sinks) {
    if (attn::check_attention(cache, batch, n_q_heads, window, sinks)) return 0;
    return attn::plan_attention(cache, batch, n_q_heads, window, sinks).total;
}

int32_t dip_window_attention(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const void* q, int64_t q_stride,
                             int32_t n_q_heads, float scale, int32_t window, int32_t sinks, void* out, int64_t out_stride, void* ws,
                             size_t ws_bytes, void* stream) {
    return attn::attend(cache, layer, batch, nullptr, q, q_stride, n_q_heads, scale, window, sinks, out, out_stride, ws, ws_bytes, stream);
}

int32_t dip_tree_attention(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const int32_t* parents, const void* q,
                           int64_t q_stride, int32_t n_q_heads, float scale, int32_t window, int32_t sinks, void* out,
                           int64_t out_stride, void* ws, size_t ws_bytes, void* stream) {
    if (!parents) return fail(DIP_ERR_INVALID_ARG, "tree_attention: null parents");
    if (batch && batch->max_rows > DIP_MAX_TREE && batch->n_rows > DIP_MAX_TREE)
        return fail(DIP_ERR_UNSUPPORTED, "tree_attention: a tree has at most %d nodes", DIP_MAX_TREE);
    return attn::attend(cache, layer, batch, parents, q, q_stride, n_q_heads, scale, window, sinks, out, out_stride, ws, ws_bytes, stream);
}

}  // extern "C"
