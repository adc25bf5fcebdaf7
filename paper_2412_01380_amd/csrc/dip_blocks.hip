// Attention over chosen blocks of a long context: bounds of the blocks' keys (dip_kv_block_bounds), the choice
// (dip_select_blocks), and the attention itself (dip_block_attention).
//
// A block's smallest and largest key, channel by channel, bound q . k for all its keys: sum_d max(q_d lo_d, q_d hi_d).  With
// q+ = max(q, 0), q- = max(-q, 0) this is q+ . hi - q- . lo.  Which blocks are read hangs on the order of these sums, so
// that they are taken in fp64, where another order of adding moves them by 1e-16 and not by a block's rank.

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "dip_attn_device.h"

namespace dip {
namespace blocks {
namespace {

using attn::f32x4;
using attn::u32x4;

constexpr int kThreads = 256;

// What an entry's rows read of its past: [0, front), chosen blocks of [front, tail), [tail, len).
struct Parts {
    int front, tail;
};
__device__ __forceinline__ Parts parts_of(int len, int page_shift, int block_shift, int sinks, int recent) {
    Parts x;
    x.tail = (min(max(len - recent, 0), (len >> page_shift) << page_shift) >> block_shift) << block_shift;
    // (sinks near 2^31: compared before they are rounded up)
    x.front = sinks >= x.tail ? x.tail : ((sinks + (1 << block_shift) - 1) >> block_shift) << block_shift;
    return x;
}

template <typename E>
__device__ __forceinline__ void widen(u32x4 x, float (&f)[16 / sizeof(E)]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) {
            f[i] = __uint_as_float(x[i]);
        } else {
            f[2 * i] = __uint_as_float(x[i] << 16);
            f[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u);
        }
    }
}

// ---- bounds: grid (pages of a sequence, sequences, layers) ------------------------------------------------------------
// A thread takes 16 bytes of a head's channels through a block's slots, kFlight of them on their way at a time.
constexpr int kFlight = 8;
struct BoundsParams {
    KvView c;                 // k at the first layer
    const int32_t* seqs;
    int back;
    int block_shift;
    char* bounds;             // at the first layer
};
template <typename E>
__global__ void __launch_bounds__(kThreads) block_bounds_kernel(const BoundsParams p) {
    constexpr int N = 16 / sizeof(E);
    const int seq = p.seqs[blockIdx.y];
    if ((unsigned)seq >= (unsigned)p.c.n_seqs) return;
    const int len = entry_len(p.c, seq);
    const int j = (p.back ? max(len - p.back, 0) >> p.c.page_shift : 0) + (int)blockIdx.x;
    if (j >= len >> p.c.page_shift) return;
    const int page = p.c.table[(size_t)seq * p.c.max_pages + j];
    if (!is_page(p.c, page)) return;
    const int per_page = 1 << (p.c.page_shift - p.block_shift), slots = 1 << p.block_shift;
    const u32x4* k = (const u32x4*)p.c.k + (int64_t)blockIdx.z * p.c.layer_stride + page * p.c.page_stride;
    u32x4* out = (u32x4*)p.bounds + ((int64_t)blockIdx.z * p.c.n_pages + page) * p.c.n_heads * per_page * 2 * p.c.pieces;
    for (int64_t i = threadIdx.x; i < (int64_t)p.c.n_heads * per_page * p.c.pieces; i += kThreads) {
        const int64_t at = i / p.c.pieces;
        const int x = (int)(i - at * p.c.pieces), b = (int)(at & (per_page - 1));
        const u32x4* from = k + (at >> (p.c.page_shift - p.block_shift)) * p.c.head_stride + (int64_t)(b * slots) * p.c.slot_stride + x;
        float lo[N], hi[N];
#pragma unroll
        for (int e = 0; e < N; ++e) lo[e] = INFINITY, hi[e] = -INFINITY;
        for (int s = 0; s < slots; s += kFlight) {        // (16 slots at least)
            u32x4 v[kFlight];
#pragma unroll
            for (int f = 0; f < kFlight; ++f) v[f] = from[(s + f) * p.c.slot_stride];
#pragma unroll
            for (int f = 0; f < kFlight; ++f) {
                float y[N];
                widen<E>(v[f], y);
#pragma unroll
                for (int e = 0; e < N; ++e) lo[e] = fminf(lo[e], y[e]), hi[e] = fmaxf(hi[e], y[e]);
            }
        }
        const float most = sizeof(E) == 4 ? FLT_MAX : __uint_as_float(0x7f7f0000u);
        u32x4 a, z;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const bool none = lo[e] > hi[e];
            lo[e] = none ? 0.f : fmaxf(fminf(lo[e], most), -most);
            hi[e] = none ? 0.f : fmaxf(fminf(hi[e], most), -most);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (sizeof(E) == 4) {
                a[w] = __float_as_uint(lo[w]);
                z[w] = __float_as_uint(hi[w]);
            } else {                                      // (what came out of bf16 goes back without rounding)
                a[w] = __float_as_uint(lo[2 * w]) >> 16 | (__float_as_uint(lo[2 * w + 1]) & 0xffff0000u);
                z[w] = __float_as_uint(hi[2 * w]) >> 16 | (__float_as_uint(hi[2 * w + 1]) & 0xffff0000u);
            }
        }
        out[at * 2 * p.c.pieces + x] = a;
        out[(at * 2 + 1) * p.c.pieces + x] = z;
    }
}

// ---- scores: grid (chunks of blocks, key/value heads, entries) --------------------------------------------------------------
struct ChoiceParams {
    KvView c;
    BatchView b;
    const char* q;
    int64_t q_stride;         // bytes
    const char* bounds;       // at the layer
    float* scores;            // [row][head][most]
    int32_t* out;             // [row][head][n_select]
    int most;                 // blocks of a sequence that there may be
    int group;
    int block_shift;
    int n_select, sinks, recent, max_len;
};
// the blocks that an entry chooses from: first, first + 1, ..
struct Middle {
    int first, n;
};
__device__ __forceinline__ Middle middle_of(const ChoiceParams& p, int len) {
    const Parts x = parts_of(min(len, p.max_len), p.c.page_shift, p.block_shift, p.sinks, p.recent);
    return {x.front >> p.block_shift, (x.tail - x.front) >> p.block_shift};
}

// Lanes of a block: each holds 16 bytes of its bounds' channels.
template <typename E, int D>
struct Lanes {
    static constexpr int PIECES = D * sizeof(E) / 16, L = PIECES <= 8 ? 8 : PIECES <= 16 ? 16 : 32;
};
// sum over L neighbouring lanes, in the last of them
template <int L>
__device__ __forceinline__ double sum_of_lanes(double x) {
    const auto moved = [&](auto ctrl) {
        const uint64_t b = __double_as_longlong(x);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, decltype(ctrl)::value, 0xf, 0xf, true);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), decltype(ctrl)::value, 0xf, 0xf, true);
        return __longlong_as_double(((uint64_t)hi << 32) | lo);
    };
    x += moved(std::integral_constant<int, 0x111>());     // row_shr 1, 2, 4, 8
    x += moved(std::integral_constant<int, 0x112>());
    x += moved(std::integral_constant<int, 0x114>());
    if constexpr (L >= 16) x += moved(std::integral_constant<int, 0x118>());
    if constexpr (L == 32) x += __shfl_up(x, 16);
    return x;
}

constexpr int kBlocks = 4;                // of a group of lanes, in registers
constexpr int kHeads = 2;                 // query heads at a time
template <typename E, int D>
__global__ void __launch_bounds__(kThreads) block_scores_kernel(const ChoiceParams p) {
    typedef Lanes<E, D> X;
    constexpr int N = 16 / sizeof(E), GROUPS = kThreads / X::L, CHUNK = GROUPS * kBlocks;
    const int e = blockIdx.z, head = blockIdx.y, lane = threadIdx.x % X::L, g = threadIdx.x / X::L;
    const EntryRows er = entry_rows(p.b, e);
    const int seq = entry_seq(p.b, p.c, e);
    if (seq < 0 || er.rows == 0) return;
    const Middle m = middle_of(p, entry_len(p.c, seq));
    const int b0 = blockIdx.x * CHUNK;
    if (b0 >= m.n || m.n <= p.n_select) return;           // (all of them are chosen)
    const int32_t* table = p.c.table + (size_t)seq * p.c.max_pages;
    const int per_shift = p.c.page_shift - p.block_shift;
    const bool has = lane < X::PIECES;
    u32x4 lo[kBlocks], hi[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
        const int b = m.first + min(b0 + i * GROUPS + g, m.n - 1);
        const int named = table[b >> per_shift], page = is_page(p.c, named) ? named : 0;
        const int64_t at = (((int64_t)page * p.c.n_heads + head) << per_shift) + (b & ((1 << per_shift) - 1));
        const u32x4* from = (const u32x4*)p.bounds + at * 2 * X::PIECES + (has ? lane : 0);
        lo[i] = from[0];
        hi[i] = from[X::PIECES];
    }
    for (int t = 0; t < er.rows; ++t) {
        const char* q = p.q + (int64_t)(er.first + t) * p.q_stride + (int64_t)head * p.group * (D * (int)sizeof(E));
        double best[kBlocks];
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) best[i] = -(double)INFINITY;
        for (int h = 0; h < p.group; h += kHeads) {
            double up[kHeads][N], down[kHeads][N];        // q+, q-
#pragma unroll
            for (int y = 0; y < kHeads; ++y) {
                float f[N];
                // (an odd group's last head twice)
                widen<E>(*(const u32x4*)(q + min(h + y, p.group - 1) * (D * (int)sizeof(E)) + (has ? lane : 0) * 16), f);
#pragma unroll
                for (int d = 0; d < N; ++d) {
                    up[y][d] = !has ? 0.0 : f[d] > 0.f || f[d] != f[d] ? (double)f[d] : 0.0;
                    down[y][d] = has && f[d] < 0.f ? (double)f[d] : 0.0;      // (-q-)
                }
            }
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                float l[N], u[N];
                widen<E>(lo[i], l);
                widen<E>(hi[i], u);
                double s[kHeads];
#pragma unroll
                for (int y = 0; y < kHeads; ++y) s[y] = 0.0;
#pragma unroll
                for (int d = 0; d < N; ++d)
#pragma unroll
                    for (int y = 0; y < kHeads; ++y) s[y] = fma(down[y][d], (double)l[d], fma(up[y][d], (double)u[d], s[y]));
#pragma unroll
                for (int y = 0; y < kHeads; ++y) {
                    const double all = sum_of_lanes<X::L>(s[y]);
                    best[i] = all > best[i] ? all : best[i];
                }
            }
        }
        if (lane == X::L - 1) {
            float* out = p.scores + ((size_t)(er.first + t) * p.c.n_heads + head) * p.most;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                const int b = b0 + i * GROUPS + g;
                if (b < m.n) out[b] = (float)best[i];
            }
        }
    }
}

// ---- the choice: grid (rows of an entry, key/value heads, entries) ------------------------------------------------------------
// The n_select largest of a row's scores, equal ones in order: a radix selection of their keys, 11, 11 and 10 bits, and
// a pass that writes the chosen ones in order.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ int block_before(int x, int* waves, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(upto, off);
        if (lane >= off) upto += y;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    int before = upto - x, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    *total = all;
    return before;
}
constexpr int kDigits = 2048;
constexpr int kItems = 8;                 // neighbouring scores of a thread in the last pass
__global__ void __launch_bounds__(kThreads) block_choice_kernel(const ChoiceParams p) {
    __shared__ int s_hist[kDigits];
    __shared__ int s_waves[kThreads / 64];
    __shared__ int s_digit, s_left;
    const int e = blockIdx.z, head = blockIdx.y, tid = threadIdx.x;
    const EntryRows er = entry_rows(p.b, e);
    if ((int)blockIdx.x >= er.rows) return;
    const size_t row = (size_t)(er.first + blockIdx.x) * p.c.n_heads + head;
    int32_t* out = p.out + row * p.n_select;
    const int seq = entry_seq(p.b, p.c, e);
    const Middle m = seq >= 0 ? middle_of(p, entry_len(p.c, seq)) : Middle{0, 0};
    if (m.n <= p.n_select) {
        for (int i = tid; i < p.n_select; i += kThreads) out[i] = i < m.n ? m.first + i : -1;
        return;
    }
    const float* scores = p.scores + row * p.most;
    // the key that the last chosen one has, and how many of those that have it
    uint32_t prefix = 0;
    int left = p.n_select;
    for (int shift = 21; shift >= 0; shift -= shift == 21 ? 11 : 10) {
        const int bits = shift == 0 ? 10 : 11, digits = 1 << bits;
        for (int i = tid; i < digits; i += kThreads) s_hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < m.n; i += kThreads) {
            const uint32_t k = key_of(scores[i]);
            if ((uint64_t)(k ^ prefix) >> (shift + bits) == 0) atomicAdd(&s_hist[k >> shift & (digits - 1)], 1);
        }
        __syncthreads();
        // from the largest digit down: the one in which `left` are reached
        const int per = digits / kThreads;
        int mine = 0, total;
        for (int i = 0; i < per; ++i) mine += s_hist[digits - 1 - (tid * per + i)];
        int before = block_before(mine, s_waves, &total);
        if (before < left && before + mine >= left)
            for (int i = 0; i < per; ++i) {
                const int d = digits - 1 - (tid * per + i), n = s_hist[d];
                if (before < left && before + n >= left) {
                    s_digit = d;
                    s_left = left - before;
                }
                before += n;
            }
        __syncthreads();
        prefix |= (uint32_t)s_digit << shift;
        left = s_left;
        __syncthreads();
    }
    int given = 0, ties = 0;
    for (int i0 = 0; i0 < m.n; i0 += kThreads * kItems) {
        uint32_t k[kItems];
        int more = 0, same = 0;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int at = i0 + tid * kItems + i;
            k[i] = at < m.n ? key_of(scores[at]) : 0;
            more += at < m.n && k[i] > prefix;
            same += at < m.n && k[i] == prefix;
        }
        int all_more, all_same;
        const int more_before = block_before(more, s_waves, &all_more);
        const int same_before = ties + block_before(same, s_waves, &all_same);
        // of the ties in front of this thread's, `left` at most were taken
        int to = given + more_before + min(same_before, left) - min(ties, left), tie = same_before;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int at = i0 + tid * kItems + i;
            if (at >= m.n || k[i] < prefix) continue;
            if (k[i] > prefix || tie++ < left) out[to++] = m.first + at;
        }
        given += all_more + min(ties + all_same, left) - min(ties, left);
        ties += all_same;
    }
}

// ---- attention ---------------------------------------------------------------------------------------------------------------
// A unit is a row, a key/value head, up to 16 query heads of its group and a share of what the row reads, which comes
// in cells of 16 positions: those in front, those of the chosen blocks, those behind.  A cell lies within a page, so that it
// has one address; a tile of a product is two cells (bf16) or one (fp32), wherever they lie.  Each wavefront streams tiles of
// its own through LDS, as in attn_rows_kernel.
struct BlockAttnParams {
    attn::AttnParams a;       // window, sinks 0
    const int32_t* blocks;    // [row][head][n_select]
    int n_select;
    int block_shift;
    int front, recent;        // (front: sinks)
    int share_tiles;          // tiles of a share
    int shares;               // most shares of a unit
    int head_blocks;          // blocks of 16 query heads of a group
};
struct Cell {
    int64_t base;             // its first position, in pieces of 16 bytes from the start of the head
    uint32_t mask;            // which of its positions the row sees
    int last;                 // the last of its positions that is read
};
constexpr int kCells = 64;                // of a wavefront in LDS at a time

template <typename E, int D, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, 1) block_attn_kernel(const BlockAttnParams bp) {
    using namespace attn;
    typedef Geo<E, D> G;
    typedef Core<E, D, 1> C;
    constexpr int THREADS = WAVES * 64, RING = 2, ROWS = 16;
    constexpr int KEYS = G::KEYS, TILE = KEYS * G::ROWB, LOADS = TILE / 1024, CPT = KEYS / 16, SPAN = kCells / CPT;
    __shared__ __align__(1024) char s_ring[WAVES * RING * 2 * TILE];
    __shared__ Cell s_cells[WAVES][kCells];
    __shared__ uint64_t s_tree[64];
    __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS];
    __shared__ int s_last, s_entry;

    const AttnParams& p = bp.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int share = blockIdx.x % bp.shares;
    int unit = blockIdx.x / bp.shares;
    const int first_unit = unit;
    const int hb = unit % bp.head_blocks;
    unit /= bp.head_blocks;
    const int head = unit % p.c.n_heads, row = unit / p.c.n_heads;
    // the entry that the row is one of
    if (tid == 0) s_entry = -1;
    __syncthreads();
    for (int e = tid; e < p.b.n_batch; e += THREADS) {
        const EntryRows er = entry_rows(p.b, e);
        if (row >= er.first && row < er.first + er.rows) atomicMax(&s_entry, e);
    }
    __syncthreads();
    const int e = __builtin_amdgcn_readfirstlane(s_entry);
    if (e < 0) return;
    const EntryRows er = entry_rows(p.b, e);
    const int seq = entry_seq(p.b, p.c, e), len = seq >= 0 ? entry_len(p.c, seq) : 0, t = row - er.first;
    if (p.parents) {
        if (wave == 0) tree_masks(p.parents + er.first, er.rows, s_tree);
        __syncthreads();
    }
    const RowSees sees_own = row_sees(p, len, t, s_tree);
    const Parts parts = parts_of(min(len, p.max_len), p.c.page_shift, bp.block_shift, bp.front, bp.recent);
    // no row sees anything from `end` on
    const int end = min(p.parents ? len + er.rows : len + t + 1, p.max_len);
    const bool alive = seq >= 0 && (sees_own.hi > 0 || sees_own.tree) && end > 0;
    const int per_block = 1 << (bp.block_shift - 4);
    const int chosen = min(bp.n_select, (parts.tail - parts.front) >> bp.block_shift);
    const int front_cells = parts.front >> 4, chosen_cells = chosen << (bp.block_shift - 4);
    const int cells = alive ? front_cells + chosen_cells + (max(end - parts.tail, 0) + 15) / 16 : 0;
    const int tiles = (cells + CPT - 1) / CPT;
    const int shares = max(1, (tiles + bp.share_tiles - 1) / bp.share_tiles);
    if (share >= shares) return;
    const int begin = share * bp.share_tiles, stop = min(tiles, begin + bp.share_tiles);
    const int mine = max(0, (stop - begin - wave + WAVES - 1) / WAVES);
    const int32_t* list = bp.blocks + ((size_t)row * p.c.n_heads + head) * bp.n_select;
    const int32_t* table = p.c.table + (size_t)max(seq, 0) * p.c.max_pages;

    auto fill = [&](int i0) {                             // the cells of the wavefront's tiles from i0 on
        const int i = lane / CPT, at = (begin + wave + WAVES * (i0 + i)) * CPT + lane % CPT;
        Cell c = {0, 0, 0};
        if (i0 + i < mine && at < cells) {
            int pos = -1;
            uint32_t mask = 0xffff;
            if (at < front_cells) {
                pos = at << 4;
            } else if (at < front_cells + chosen_cells) {
                const int n = (at - front_cells) >> (bp.block_shift - 4), b = list[n];
                const bool rises = n == 0 || b > list[n - 1];
                if (rises && b >= parts.front >> bp.block_shift && b < parts.tail >> bp.block_shift)
                    pos = (b << bp.block_shift) + (((at - front_cells) & (per_block - 1)) << 4);
            } else {
                pos = parts.tail + ((at - front_cells - chosen_cells) << 4);
                mask = (uint32_t)sees(sees_own, pos, 0, len) & 0xffff;
            }
            if (pos < 0) {
                pos = 0;
                mask = 0;
            }
            const int named = table[pos >> p.c.page_shift], page = is_page(p.c, named) ? named : 0;
            c.base = page * p.c.page_stride + (pos & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride;
            c.mask = mask;
            c.last = min(15, end - 1 - pos);
        }
        s_cells[wave][lane] = c;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    if (mine > 0) fill(0);

    C core;
    const int r0 = hb * ROWS, n_rows = min(ROWS, p.group - r0);
    {
        const int r = lane & 15;
        core.load_q(0, r < n_rows ? p.q + (int64_t)row * p.q_stride + (int64_t)(head * p.group + r0 + r) * (D * G::ES) : nullptr);
    }
    Softmax<E, D, 1> soft;
    soft.start(core);
    const char* kbase = p.c.k + p.c.head_stride * head * 16;
    const char* vbase = p.c.v + p.c.head_stride * head * 16;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_offset(s_ring) + wave * (RING * 2 * TILE));
    auto fetch = [&](int i) {
        const uint32_t to = ring_at + (i & (RING - 1)) * (2 * TILE);
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int at = x * 64 + lane, r = at / G::CPR;
            const Cell& c = s_cells[wave][(i & (SPAN - 1)) * CPT + (r >> 4)];
            const int64_t off = (c.base + min(r & 15, c.last) * p.c.slot_stride + ((at % G::CPR) ^ G::twist(r))) * 16;
            load_to_lds<true>(kbase + off, to + x * 1024);
            load_to_lds<true>(vbase + off, to + TILE + x * 1024);
        }
    };
    // what the row sees of a tile, a bit per key
    auto mask_of = [&](int i) {
        uint32_t m = 0;
#pragma unroll
        for (int x = 0; x < CPT; ++x) m |= s_cells[wave][(i & (SPAN - 1)) * CPT + x].mask << (16 * x);
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
    };
    constexpr uint32_t ALL = CPT == 2 ? 0xffffffffu : 0xffffu;
    uint32_t masks[RING] = {0, 0};                        // of the tiles in the ring
    if (mine > 0) {
        masks[0] = mask_of(0);
        fetch(0);
    }
    if (mine > 1) {
        masks[1] = mask_of(1);
        fetch(1);
    }
    if (shares > 1 && tid == 0) ticket_open(p.tickets + (size_t)first_unit * kTicketStride, p.epoch);
    bool spoilt = false;
    for (int i = 0; i < mine; ++i) {
        if (i + 1 < mine) wait_loads<2 * LOADS>(); else wait_loads<0>();
        const uint32_t tile = ring_at + (i & (RING - 1)) * (2 * TILE), mask = masks[0];
        masks[0] = masks[1];
        f32x4 s[1][C::MT];
        core.scores(C::k_base(tile), s);
        if (mask != ALL) {
#pragma unroll
            for (int x = 0; x < LOADS; ++x) spoilt |= take_out<G>(tile + TILE, x);
            asm volatile("" ::: "memory");
            const uint32_t bits = mask >> (4 * (lane >> 4));
#pragma unroll
            for (int x = 0; x < 4 * C::MT; ++x) s[0][x >> 2][x & 3] = (bits >> (16 * (x >> 2) + (x & 3))) & 1 ? s[0][x >> 2][x & 3] : -INFINITY;
        }
        soft.step(core, s, p.scale_log2);
        typename C::Weights w;
        C::pack(s, 0, w);
        core.add_values(C::v_base(tile + TILE), 0, w);
        C::schedule_values();
        if (i + RING < mine) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (everything read from the tile that goes)
            if (((i + RING) & (SPAN - 1)) == 0) fill(i + RING);
            masks[1] = mask_of(i + RING);
            fetch(i + RING);
        }
    }
    // what was taken out of tiles, to the sums of a row that sees it
    if (__any(spoilt)) {
        for (int i = 0; i < mine; ++i) {
            if ((i & (SPAN - 1)) == 0) fill(i);
            const uint32_t mask = mask_of(i);
            if (mask == ALL) continue;
            for (uint32_t left = mask; left; left &= left - 1) {
                const int r = __ffs((int)left) - 1;
                const Cell& c = s_cells[wave][(i & (SPAN - 1)) * CPT + (r >> 4)];
                const char* from = vbase + (c.base + (r & 15) * p.c.slot_stride) * 16;
#pragma unroll
                for (int y = 0; y < C::OB; ++y) {
                    f32x4 v;
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const int dim = C::quad_dim(y) + d;
                        if constexpr (sizeof(E) == 4) v[d] = ((const float*)from)[dim];
                        else v[d] = __uint_as_float((uint32_t)((const uint16_t*)from)[dim] << 16);
                        v[d] = (__float_as_uint(v[d]) & 0x7f800000u) == 0x7f800000u ? v[d] : 0.f;
                    }
                    core.add_quad(0, y, v);
                }
            }
        }
    }

    // join the wavefronts
    {
        const float l = column_sum(soft.l[0]);
        if (lane < 16) {
            s_m[wave][lane] = mine > 0 ? soft.m[0] : -INFINITY;
            s_l[wave][lane] = mine > 0 ? l : 0.f;
        }
    }
    __syncthreads();                                      // (and every wavefront is done with its tiles)
    constexpr int QUADS = D / 4;
    float* s_o = (float*)s_ring;                          // [wave][row][quad, rotated by the row][4]
    static_assert(WAVES * ROWS * D * 4 <= (int)sizeof(s_ring), "the joined rows fit the ring");
    {
        const int r = lane & 15;
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, s_m[w][r]);
        const float a = join_weight(s_m[wave][r], top);
#pragma unroll
        for (int y = 0; y < C::OB; ++y) {
            const int quad = C::quad_dim(y) / 4;
            *(f32x4*)(s_o + ((wave * ROWS + r) * QUADS + (quad + r) % QUADS) * 4) = core.quad(0, y) * a;
        }
    }
    __syncthreads();
    const size_t part = (size_t)first_unit * bp.shares;
    for (int i = tid; i < n_rows * QUADS; i += THREADS) {
        const int r = i / QUADS, quad = i % QUADS;
        float top = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, s_m[w][r]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) l += s_m[w][r] == -INFINITY ? s_l[w][r] : s_l[w][r] * fast_exp2(s_m[w][r] - top);
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) o += *(const f32x4*)(s_o + ((w * ROWS + r) * QUADS + (quad + r) % QUADS) * 4);
        if (shares > 1) {
            const size_t at = (part + share) * ROWS + r;
            share_put(p.part_o + at * D + quad * 4, o);
            if (quad == 0)
                __hip_atomic_store((uint64_t*)(p.part_ml + at), ((uint64_t)__float_as_uint(l) << 32) | __float_as_uint(top),
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        } else {
            const f32x4 zero = {0, 0, 0, 0};
            store_quad<E>(p.out + (int64_t)row * p.out_stride + (int64_t)(head * p.group + r0 + r) * (D * G::ES), quad * 4,
                          l == 0.f ? zero : o * (1.f / l));
        }
    }
    if (shares <= 1) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s_last = ticket_last(p.tickets + (size_t)first_unit * kTicketStride, p.epoch, shares);
    __syncthreads();
    if (s_last) join_shares<E, D, ROWS, THREADS, true>(p, (int)part, shares, row, head, r0, 0, n_rows);
}

// ---- checks and launches ---------------------------------------------------------------------------------------------------
int32_t check_block(const dip_kv_cache* c, int32_t block) {
    if (block < 16 || block > c->page_size || (block & (block - 1)))
        return fail(DIP_ERR_UNSUPPORTED, "blocks: a block must be a power of two from 16 to the page size, got %d", block);
    return DIP_OK;
}
int reach(const dip_kv_cache* c, const dip_batch* b) {
    const int fit = c->max_pages * c->page_size;
    return b->max_len && b->max_len < fit ? b->max_len : fit;
}
int32_t check_rows(const dip_kv_cache* c, const dip_batch* b, int32_t n_q_heads, int32_t block) {
    int32_t st = validate_kv(c);
    if (!st) st = validate_batch(b, true);
    if (!st) st = check_block(c, block);
    if (st) return st;
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128)
        return fail(DIP_ERR_UNSUPPORTED, "blocks: head_dim %d is none of 64, 96, 128", c->head_dim);
    if (n_q_heads < 1 || n_q_heads % c->n_kv_heads)
        return fail(DIP_ERR_INVALID_ARG, "blocks: %d query heads are no multiple of %d", n_q_heads, c->n_kv_heads);
    if (n_q_heads > 65535) return fail(DIP_ERR_UNSUPPORTED, "blocks: more than 65535 query heads");
    return DIP_OK;
}
int32_t check_choice(int32_t n_select, int32_t sinks, int32_t recent) {
    if (n_select < 1) return fail(DIP_ERR_INVALID_ARG, "blocks: n_select must be >= 1");
    if (n_select > DIP_MAX_SELECT) return fail(DIP_ERR_UNSUPPORTED, "blocks: n_select must be at most %d", DIP_MAX_SELECT);
    if (sinks < 0 || recent < 0) return fail(DIP_ERR_INVALID_ARG, "blocks: sinks and recent must be >= 0");
    return DIP_OK;
}
int32_t check_q(const dip_kv_cache* c, int32_t layer, const void* q, int64_t q_stride, int32_t n_q_heads) {
    if (layer < 0 || layer >= c->n_layers) return fail(DIP_ERR_INVALID_ARG, "blocks: layer %d of %d", layer, c->n_layers);
    if (!q) return fail(DIP_ERR_INVALID_ARG, "blocks: null queries");
    if (q_stride < (int64_t)n_q_heads * c->head_dim) return fail(DIP_ERR_INVALID_ARG, "blocks: q_stride smaller than a row");
    if (q_stride * elem_bytes(c->dtype) % 16 || !aligned16(q)) return fail(DIP_ERR_UNSUPPORTED, "blocks: rows of q must start on 16-byte boundaries");
    return DIP_OK;
}
size_t layer_bounds(const dip_kv_cache* c, int32_t block) {
    return (size_t)c->n_pages * c->n_kv_heads * (c->page_size / block) * 2 * c->head_dim * elem_bytes(c->dtype);
}
// most blocks that a row may choose from
int64_t most_blocks(const dip_kv_cache* c, const dip_batch* b, int32_t block) { return reach(c, b) / block; }

template <typename E>
hipError_t launch_scores(const ChoiceParams& p, int head_dim, int n_batch, hipStream_t stream) {
    const auto go = [&](auto dim) {
        constexpr int D = decltype(dim)::value, CHUNK = kThreads / Lanes<E, D>::L * kBlocks;
        return launch_timed(block_scores_kernel<E, D>, dim3((p.most + CHUNK - 1) / CHUNK, p.c.n_heads, n_batch), dim3(kThreads), stream,
                            DIP_KERNEL_BLOCKS, p);
    };
    if (head_dim == 64) return go(std::integral_constant<int, 64>());
    if (head_dim == 96) return go(std::integral_constant<int, 96>());
    return go(std::integral_constant<int, 128>());
}

struct AttnPlan {
    int waves, head_blocks, share_tiles, shares;
    int64_t units;
    size_t off_ml, off_tickets, total;
};
AttnPlan plan_attention(const dip_kv_cache* c, const dip_batch* b, int n_q_heads, int block, int n_select, int sinks, int recent) {
    AttnPlan pl;
    const int keys = c->dtype == DIP_BF16 ? 32 : 16;
    pl.waves = 2;
    pl.head_blocks = (n_q_heads / c->n_kv_heads + 15) / 16;
    pl.units = (int64_t)b->n_rows * c->n_kv_heads * pl.head_blocks;
    // the most that a row can come to read, in tiles
    const int64_t all = reach(c, b);
    int64_t read = std::min((int64_t)sinks + block, all) + std::min((int64_t)n_select * block, all);
    read += std::min((int64_t)recent + c->page_size + block + rows_bound(b), all);
    const int64_t tiles = std::max<int64_t>(1, (std::min(read, all) + keys - 1) / keys + 2);
    const int64_t slots = 256 * ((160 * 1024 - 1024) / (pl.waves * 256 * c->head_dim + 6144));
    // one round of workgroups; a share has two tiles for each wavefront at least
    const int64_t shares = std::max<int64_t>(1, std::min(slots / pl.units, tiles / (2 * pl.waves)));
    pl.share_tiles = (int)((tiles + shares - 1) / shares);
    pl.shares = (int)((tiles + pl.share_tiles - 1) / pl.share_tiles);
    const size_t parts = pl.shares > 1 ? (size_t)pl.units * pl.shares : 0;
    size_t o = align_up(parts * 16 * c->head_dim * sizeof(float), 256);
    pl.off_ml = o;
    o += align_up(parts * 16 * sizeof(float2), 256);
    pl.off_tickets = o;
    if (pl.shares > 1) o += sizeof(uint64_t) * kTicketStride * pl.units;
    pl.total = o < 256 ? 256 : o;
    return pl;
}
template <typename E>
hipError_t launch_attention(const BlockAttnParams& p, const AttnPlan& pl, int head_dim, hipStream_t stream) {
    const dim3 grid((unsigned)(pl.units * pl.shares)), block(pl.waves * 64);
    const auto go = [&](auto kernel) { return launch_timed(kernel, grid, block, stream, DIP_KERNEL_BLOCKS, p); };
    if (head_dim == 64) return go(block_attn_kernel<E, 64, 2>);
    if (head_dim == 96) return go(block_attn_kernel<E, 96, 2>);
    return go(block_attn_kernel<E, 128, 2>);
}

int32_t check_attention(const dip_kv_cache* c, const dip_batch* b, int32_t n_q_heads, int32_t block, int32_t n_select, int32_t sinks,
                        int32_t recent) {
    int32_t st = check_rows(c, b, n_q_heads, block);
    if (!st) st = check_choice(n_select, sinks, recent);
    if (st) return st;
    const AttnPlan pl = plan_attention(c, b, n_q_heads, block, n_select, sinks, recent);
    if (pl.units * pl.shares * pl.waves * 64 >= (int64_t)1 << 32)    // threads of a launch
        return fail(DIP_ERR_UNSUPPORTED, "blocks: too many rows for one call");
    return DIP_OK;
}

}  // namespace
}  // namespace blocks
}  // namespace dip

using namespace dip;
using namespace dip::blocks;

extern "C" {

size_t dip_block_bounds_bytes(const dip_kv_cache* cache, int32_t block) {
    if (validate_kv(cache) || check_block(cache, block)) return 0;
    return layer_bounds(cache, block) * cache->n_layers;
}

int32_t dip_kv_block_bounds(const dip_kv_cache* cache, int32_t layer, int32_t n_layers, const int32_t* seqs, int32_t n, int32_t back,
                            int32_t block, void* bounds, void* stream) {
    int32_t st = validate_kv(cache);
    if (!st) st = check_block(cache, block);
    if (st) return st;
    if (layer < 0 || n_layers < 1 || n_layers > cache->n_layers || layer > cache->n_layers - n_layers)
        return fail(DIP_ERR_INVALID_ARG, "layers %d .. %d outside the cache's %d", layer, layer + n_layers - 1, cache->n_layers);
    if (!seqs || !bounds) return fail(DIP_ERR_INVALID_ARG, "block_bounds: null pointer");
    if (n < 1 || n > 65535) return fail(DIP_ERR_INVALID_ARG, "block_bounds: 1 .. 65535 sequences, got %d", n);
    if (back < 0) return fail(DIP_ERR_INVALID_ARG, "block_bounds: back must be >= 0");
    if (!aligned16(bounds)) return fail(DIP_ERR_UNSUPPORTED, "block_bounds: bounds must be 16-byte aligned");
    BoundsParams p;
    p.c = view_of(cache);
    p.c.k += p.c.layer_stride * layer * 16;
    p.seqs = seqs;
    p.back = back;
    p.block_shift = log2_of(block);
    p.bounds = (char*)bounds + layer_bounds(cache, block) * layer;
    const int64_t pages = back ? std::min<int64_t>(cache->max_pages, (int64_t)back / cache->page_size + 1) : cache->max_pages;
    if (pages * kThreads >= (int64_t)1 << 32) return fail(DIP_ERR_UNSUPPORTED, "block_bounds: too many pages for one call");
    const dim3 grid((unsigned)pages, n, n_layers);
    return check_hip(cache->dtype == DIP_F32 ? launch_timed(block_bounds_kernel<float>, grid, dim3(kThreads), (hipStream_t)stream, DIP_KERNEL_BLOCKS, p)
                                             : launch_timed(block_bounds_kernel<uint16_t>, grid, dim3(kThreads), (hipStream_t)stream, DIP_KERNEL_BLOCKS, p),
                     "block_bounds launch");
}

size_t dip_select_blocks_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch, int32_t n_q_heads, int32_t block) {
    if (check_rows(cache, batch, n_q_heads, block)) return 0;
    const size_t n = (size_t)batch->n_rows * cache->n_kv_heads * most_blocks(cache, batch, block) * sizeof(float);
    return n < 256 ? 256 : align_up(n, 256);
}

int32_t dip_select_blocks(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const void* q, int64_t q_stride,
                          int32_t n_q_heads, int32_t block, const void* bounds, int32_t n_select, int32_t sinks, int32_t recent,
                          int32_t* blocks, void* ws, size_t ws_bytes, void* stream) {
    int32_t st = check_rows(cache, batch, n_q_heads, block);
    if (!st) st = check_choice(n_select, sinks, recent);
    if (!st) st = check_q(cache, layer, q, q_stride, n_q_heads);
    if (st) return st;
    if (!bounds || !blocks) return fail(DIP_ERR_INVALID_ARG, "select_blocks: null pointer");
    if (!aligned16(bounds)) return fail(DIP_ERR_UNSUPPORTED, "select_blocks: bounds must be 16-byte aligned");
    if (rows_bound(batch) >= 1 << 24) return fail(DIP_ERR_UNSUPPORTED, "select_blocks: too many rows for one call");
    st = validate_ws(ws, ws_bytes, dip_select_blocks_workspace_bytes(cache, batch, n_q_heads, block));
    if (st) return st;
    ChoiceParams p;
    p.c = view_of(cache);
    p.b = view_of(batch);
    p.q = (const char*)q;
    p.q_stride = q_stride * elem_bytes(cache->dtype);
    p.bounds = (const char*)bounds + layer_bounds(cache, block) * layer;
    p.scores = (float*)ws;
    p.out = blocks;
    p.most = (int)most_blocks(cache, batch, block);
    p.group = n_q_heads / cache->n_kv_heads;
    p.block_shift = log2_of(block);
    p.n_select = n_select;
    p.sinks = sinks;
    p.recent = recent;
    p.max_len = reach(cache, batch);
    if (p.most > n_select) {
        st = check_hip(cache->dtype == DIP_F32 ? launch_scores<float>(p, cache->head_dim, batch->n_batch, (hipStream_t)stream)
                                               : launch_scores<uint16_t>(p, cache->head_dim, batch->n_batch, (hipStream_t)stream),
                       "block_scores launch");
        if (st) return st;
    }
    return check_hip(launch_timed(block_choice_kernel, dim3(p.b.max_rows, cache->n_kv_heads, batch->n_batch), dim3(kThreads),
                                  (hipStream_t)stream, DIP_KERNEL_BLOCKS, p), "block_choice launch");
}

size_t dip_block_attention_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch, int32_t n_q_heads, int32_t block,
                                           int32_t n_select, int32_t sinks, int32_t recent) {
    if (check_attention(cache, batch, n_q_heads, block, n_select, sinks, recent)) return 0;
    return blocks::plan_attention(cache, batch, n_q_heads, block, n_select, sinks, recent).total;
}

int32_t dip_block_attention(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const int32_t* parents,
                            const int32_t* blocks, int32_t n_select, int32_t block, const void* q, int64_t q_stride, int32_t n_q_heads,
                            float scale, int32_t sinks, int32_t recent, void* out, int64_t out_stride, void* ws, size_t ws_bytes,
                            void* stream) {
    int32_t st = check_attention(cache, batch, n_q_heads, block, n_select, sinks, recent);
    if (!st) st = check_q(cache, layer, q, q_stride, n_q_heads);
    if (st) return st;
    if (!blocks || !out) return fail(DIP_ERR_INVALID_ARG, "block_attention: null pointer");
    if (parents && rows_bound(batch) > DIP_MAX_TREE) return fail(DIP_ERR_UNSUPPORTED, "block_attention: a tree has at most %d nodes", DIP_MAX_TREE);
    if (!std::isfinite(scale) || scale <= 0.f) return fail(DIP_ERR_INVALID_ARG, "block_attention: scale must be finite and > 0");
    const int es = elem_bytes(cache->dtype);
    if (out_stride < (int64_t)n_q_heads * cache->head_dim) return fail(DIP_ERR_INVALID_ARG, "block_attention: out_stride smaller than a row");
    if (out_stride * es % 16 || !aligned16(out)) return fail(DIP_ERR_UNSUPPORTED, "block_attention: rows of out must start on 16-byte boundaries");
    const AttnPlan pl = dip::blocks::plan_attention(cache, batch, n_q_heads, block, n_select, sinks, recent);
    st = validate_ws(ws, ws_bytes, pl.total);
    if (st) return st;
    BlockAttnParams p;
    p.a.c = view_of(cache);
    p.a.c.k += p.a.c.layer_stride * layer * 16;
    p.a.c.v += p.a.c.layer_stride * layer * 16;
    p.a.b = view_of(batch);
    p.a.parents = parents;
    p.a.q = (const char*)q;
    p.a.out = (char*)out;
    p.a.q_stride = q_stride * es;
    p.a.out_stride = out_stride * es;
    p.a.group = n_q_heads / cache->n_kv_heads;
    p.a.scale_log2 = scale * 1.44269504088896340736f;
    p.a.window = 0;
    p.a.sinks = 0;
    p.a.max_len = reach(cache, batch);
    p.a.slots = p.a.grid = p.a.row_blocks = p.a.join_rows = 0;
    p.a.part_o = (float*)ws;
    p.a.part_ml = (float2*)((char*)ws + pl.off_ml);
    p.a.tickets = (uint64_t*)((char*)ws + pl.off_tickets);
    p.a.epoch = next_epoch();
    p.blocks = blocks;
    p.n_select = n_select;
    p.block_shift = log2_of(block);
    p.front = sinks;
    p.recent = recent;
    p.share_tiles = pl.share_tiles;
    p.shares = pl.shares;
    p.head_blocks = pl.head_blocks;
    return check_hip(cache->dtype == DIP_F32 ? launch_attention<float>(p, pl, cache->head_dim, (hipStream_t)stream)
                                             : launch_attention<uint16_t>(p, pl, cache->head_dim, (hipStream_t)stream),
                     "block_attention launch");
}

}  // extern "C"
