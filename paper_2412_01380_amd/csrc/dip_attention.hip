// Attention over a paged key/value cache: dip_window_attention, dip_tree_attention.
//
// The rows of an entry that share a key/value head -- its tokens or nodes times the query heads of the
// group -- form blocks, and a workgroup takes a block and a share of the keys that it sees:
//   up to 64 rows          attn_rows_kernel: blocks of 16, 32 or 64; wavefronts stream keys of their own
//   more                   attn_block_kernel: blocks of 64 (fp32), 128 or 256 whose wavefronts share the tiles
// Keys are read once for all query heads of a group and all rows of a block.  With few rows what bounds the
// call is reading them: 32 tokens of 40 heads on 10, a window of 2047, 73 us for the 332 MB of K and V (52 us
// at the rate of a plain read).  With many it is the matrix cores and, beside them, the softmax's plain
// instructions: a maximum, two multiply-adds, an exponential, a sum, a mask and two halves of a move and a conversion
// for every weight, whose products, P V with two terms, are 384 multiply-adds at 128 dims.

#include <algorithm>
#include <cmath>

#include "dip_attn_device.h"

namespace dip {
namespace attn {
namespace {

constexpr int kRing = 2;                  // tiles of a wavefront in LDS: one in use, one on its way
constexpr int kIds = 256;                 // page numbers of a wavefront in LDS at a time

// WAVES wavefronts, each of which streams tiles of its own through LDS (no barrier in the loop) and keeps a
// softmax of its own; they are joined in LDS at the end, and shares of a block by the last of its workgroups.
// LDS although no wavefront reads another's tile: a load to LDS holds no registers while it is on its way, and
// the products want rows of K and columns of V, which memory has neither of side by side.  Two tiles of 32 keys
// (16 in fp32) each: a third one costs a workgroup per compute unit.
// Measured (bf16, 128 dims): 2 x 700 keys 10.3 us, of which 4.4 any launch takes; 8 trees of 8 nodes, 4 heads on
// one, up to 8192 keys 46 us at 3.7 TB/s.  fp32, 3 trees of 7 nodes, 32 heads, 96 dims: 19 us.
template <typename E, int D, int NB, int WAVES, bool ONCE>
__global__ void __launch_bounds__(WAVES * 64, 1) attn_rows_kernel(const AttnParams p) {
    typedef Geo<E, D> G;
    typedef Core<E, D, NB> C;
    constexpr int THREADS = WAVES * 64;
    constexpr int KEYS = G::KEYS, TILE = KEYS * G::ROWB, LOADS = TILE / 1024, ROWS = 16 * NB;
    static_assert(TILE % 1024 == 0, "whole loads");
    __shared__ __align__(1024) char s_ring[WAVES * kRing * 2 * TILE];
    __shared__ int s_ids[WAVES][kIds];
    __shared__ uint64_t s_tree[64];
    __shared__ float s_m[WAVES][ROWS], s_l[WAVES][ROWS];
    __shared__ int s_last;
    __shared__ Unit s_unit;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (wave == 0) Units<KEYS, ROWS>(p, 2 * WAVES).find(blockIdx.x, &s_unit);
    __syncthreads();
    const Unit u = uniform(s_unit);
    if (u.rows == 0) return;
    const int seq = u.seq, len = u.len, r0 = u.r0, n_rows = u.n_rows, head = u.head;
    Range range = key_range<KEYS>(p, len, u.rows, r0 / p.group, (r0 + n_rows - 1) / p.group);
    if (seq < 0) range.tiles = 0;
    const int shares = u.cut(range.tiles);
    const int begin = u.share * u.size, end = u.end(range.tiles);
    if (begin >= end && u.share > 0) return;

    // the wavefront's tiles are begin + wave, + WAVES, ..; the page numbers of the next `span` of them are in LDS
    constexpr int KEYS_LOG2 = KEYS == 32 ? 5 : 4;
    const int per_log2 = max(0, KEYS_LOG2 - p.c.page_shift), per = 1 << per_log2, span = min(64, kIds >> per_log2);
    const int mine = max(0, (end - begin - wave + WAVES - 1) / WAVES);
    auto tile_of = [&](int i) { return tile_at(range, begin + wave + WAVES * i) * KEYS; };
    auto ids = [&](int i0) {
        for (int i = lane; i < min(span, mine - i0) * per; i += 64) {
            const int at = (tile_of(i0 + (i >> per_log2)) >> p.c.page_shift) + (i & (per - 1));
            const int page = at < p.c.max_pages ? p.c.table[(size_t)seq * p.c.max_pages + at] : 0;
            s_ids[wave][i] = (unsigned)page < (unsigned)p.c.n_pages ? page : 0;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    ids(0);
    if (p.parents && wave == 0) tree_masks(p.parents + u.first_row, u.rows, s_tree);
    if (p.parents) __syncthreads();

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
        core.load_q(nb, is ? p.q + (int64_t)(u.first_row + t) * p.q_stride + (int64_t)(head * p.group + r % p.group) * (D * G::ES) : nullptr);
    }
    Softmax<E, D, NB> soft;
    soft.start(core);

    const char* kbase = p.c.k + p.c.head_stride * head * 16;
    const char* vbase = p.c.v + p.c.head_stride * head * 16;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_offset(s_ring) + wave * (kRing * 2 * TILE));
    auto fetch = [&](int i) {
        if (i && (i & (span - 1)) == 0) ids(i);
        const int j0 = tile_of(i);
        const uint32_t to = ring_at + (i & (kRing - 1)) * (2 * TILE);
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int64_t off = piece_offset<G>(p.c, s_ids[wave] + (i & (span - 1)) * per, j0, range.end, x);
            load_to_lds<ONCE>(kbase + off, to + x * 1024);
            load_to_lds<ONCE>(vbase + off, to + TILE + x * 1024);
        }
    };

    if (mine > 0) fetch(0);
    if (mine > 1) fetch(1);
    if (shares > 1 && tid == 0) ticket_open(p.tickets + (size_t)u.first * kTicketStride, p.epoch);
    bool spoilt = false;                                  // (something was taken out of a tile)
    auto whole = [&](int j0) { return j0 + KEYS <= range.sure && (j0 >= range.from || j0 + KEYS <= p.sinks); };
    for (int i = 0; i < mine; ++i) {
        if (i + 1 < mine) wait_loads<2 * LOADS>(); else wait_loads<0>();
        const int j0 = tile_of(i);
        const uint32_t tile = ring_at + (i & (kRing - 1)) * (2 * TILE);
        f32x4 s[NB][C::MT];
        core.scores(C::k_base(tile), s);
        if (!whole(j0)) {
#pragma unroll
            for (int x = 0; x < LOADS; ++x) spoilt |= take_out<G>(tile + TILE, x);
            asm volatile("" ::: "memory");
            apply_sees(s, row, j0, p.sinks, len);
        }
        soft.step(core, s, p.scale_log2);
        typename C::Weights w;
        C::pack(s, 0, w);
        core.add_values(C::v_base(tile + TILE), 0, w);
        C::schedule_values();
        if (i + kRing < mine) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (everything read from the tile that goes)
            fetch(i + kRing);
        }
    }

    if (__any(spoilt))
        put_back<E, D, NB, KEYS>(p, core, row, vbase, seq, len, range.end, mine, [&](int i) { const int j0 = tile_of(i); return whole(j0) ? -1 : j0; });

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
    static_assert(WAVES * ROWS * D * 4 <= (int)sizeof(s_ring), "the joined rows fit the ring");
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = 16 * nb + (lane & 15);
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, s_m[w][r]);
        const float a = join_weight(s_m[wave][r], top);
#pragma unroll
        for (int y = 0; y < C::OB; ++y) {
            const int quad = C::quad_dim(y) / 4;
            *(f32x4*)(s_o + ((wave * ROWS + r) * QUADS + (quad + r) % QUADS) * 4) = core.quad(nb, y) * a;
        }
    }
    __syncthreads();
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
            const size_t at = (size_t)(u.first + u.share) * ROWS + r;
            share_put(p.part_o + at * D + quad * 4, o);
            if (quad == 0)
                __hip_atomic_store((uint64_t*)(p.part_ml + at), ((uint64_t)__float_as_uint(l) << 32) | __float_as_uint(top),
                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        } else {
            const int t = (r0 + r) / p.group, h = head * p.group + (r0 + r) % p.group;
            const f32x4 zero = {0, 0, 0, 0};
            store_quad<E>(p.out + (int64_t)(u.first_row + t) * p.out_stride + (int64_t)h * (D * G::ES), quad * 4, l == 0.f ? zero : o * (1.f / l));
        }
    }
    if (shares <= 1) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s_last = ticket_last(p.tickets + (size_t)u.first * kTicketStride, p.epoch, shares);
    __syncthreads();
    if (s_last) join_shares<E, D, ROWS, THREADS, true>(p, u.first, shares, u.first_row, head, r0, 0, n_rows);
}

// Rows enough to fill the matrix cores: the wavefronts of a workgroup, 16 NB rows each, share the tiles, one barrier
// a tile.  Four tiles of LDS: V of the last one, the current one, two on their way.
// An operand read from LDS serves NB products: with one block of 16 rows the reads (570 bytes/ns of a compute
// unit) take as long as the products, with two half; four do not fit the registers.  The softmax of a tile runs
// beside the products of its neighbours: P V lags one tile behind K Q, so both are at hand when a wavefront
// waits for exponentials.  What is left is that products and plain instructions of the two wavefronts of a SIMD
// overlap only by half (with one term: alone 485 and 515 us of a probe, together 880).
// Measured (bf16, 128 dims, 4 heads on one): 2 prompts of up to 4096 rows, window 2047: 470 us (630 TFLOP/s, 950 with the
// weights' second terms, of the 1152 of a large library product); 4 trees of 64 nodes over up to 49152 keys 226 us.
// With attn_rows_kernel: 868 and 472 us.
// bf16: 64 keys to a tile, eight wavefronts, one workgroup to a compute unit.
template <typename E>
struct Block {
    static constexpr int WAVES = 8, SUB = 2;
    static constexpr int per_simd(int) { return 2; }
};
// fp32: 16 keys, and small workgroups, several to a compute unit (its products take sixteen times as long: what
// counts is that some wavefront of a SIMD always has one).  Against attn_rows_kernel over the same rows: 2 x 100
// rows of 8 heads, 64 dims, 3000 keys 60 -> 37 us; 2048 rows, 4 heads on one, 128 dims 555 -> 412 us; 32 trees of 24
// nodes, 4 heads on one, 64 dims, 2000 keys 124 -> 84 us; 4 x 600 rows, 96 dims, 1000 keys before them 214 -> 210 us.
template <>
struct Block<float> {
    static constexpr int WAVES = 4, SUB = 1;
    static constexpr int per_simd(int dims) { return 6 - dims / 32; }
};
constexpr int kBlockRing = 4;
constexpr int kIdTiles = 64;              // tiles whose page numbers are in LDS at a time

template <typename E, int D, int NB, bool ONCE>
__global__ void __launch_bounds__(Block<E>::WAVES * 64, Block<E>::per_simd(D)) attn_block_kernel(const AttnParams p) {
    typedef Geo<E, D> G;
    typedef Core<E, D, NB> C;
    constexpr int WAVES = Block<E>::WAVES, THREADS = WAVES * 64, SUB = Block<E>::SUB;
    constexpr int KEYS = SUB * G::KEYS, TILE = KEYS * G::ROWB, LOADS = TILE / 1024, ROWS = 16 * NB * WAVES;
    constexpr int MINE = (LOADS + WAVES - 1) / WAVES;     // loads of a wavefront (some twice where uneven)
    constexpr int Q = SUB * C::MT;
    __shared__ __align__(1024) char s_ring[kBlockRing * 2 * TILE];
    __shared__ int s_ids[kIdTiles * KEYS];
    __shared__ uint64_t s_tree[64];
    __shared__ int s_spoilt;                              // something was taken out of a tile
    __shared__ Unit s_unit;

    // XCD x gets consecutive units, so that blocks of one head find its keys in their L2
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (wave == 0) {
        const Units<KEYS, ROWS> units(p, 8);
        const int per_xcd = (units.total + 7) / 8, at = blockIdx.x >> 3;
        units.find(at < per_xcd ? (int)(blockIdx.x & 7) * per_xcd + at : units.total, &s_unit);
    }
    __syncthreads();
    const Unit u = uniform(s_unit);
    if (u.rows == 0) return;
    const int seq = u.seq, len = u.len, r0 = u.r0, n_rows = u.n_rows, head = u.head;
    Range range = key_range<KEYS>(p, len, u.rows, r0 / p.group, (r0 + n_rows - 1) / p.group);
    if (seq < 0) range.tiles = 0;
    const int shares = u.cut(range.tiles);
    const int begin = u.share * u.size, n = max(0, u.end(range.tiles) - begin);
    if (n == 0 && u.share > 0) return;

    const int per = max(1, KEYS >> p.c.page_shift);
    page_ids<KEYS, THREADS>(p.c, seq, range, begin, min(n, kIdTiles), per, s_ids);
    if (p.parents && wave == 0) tree_masks(p.parents + u.first_row, u.rows, s_tree);
    if (tid == 0) s_spoilt = 0;
    __syncthreads();

    C core;
    const int w0 = wave * 16 * NB;                        // the wavefront's first row in the block
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = w0 + 16 * nb + (lane & 15), t = (r0 + r) / p.group;
        core.load_q(nb, r < n_rows ? p.q + (int64_t)(u.first_row + t) * p.q_stride + (int64_t)(head * p.group + (r0 + r) % p.group) * (D * G::ES) : nullptr);
    }
    // what the lane's rows see, worked out where it is asked for rather than kept in registers (`lane` from
    // fresh(): the compiler would keep it all the same)
    auto fresh = [&]() { int x = tid & 63; asm volatile("" : "+v"(x)); return x; };
    auto sees_of = [&](int lane, RowSees (&row)[NB]) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int r = w0 + 16 * nb + (lane & 15);
            row[nb] = row_sees(p, len, r < n_rows ? (r0 + r) / p.group : 0, s_tree);
        }
    };
    Softmax<E, D, NB> soft;
    soft.start(core);

    const char* kbase = p.c.k + p.c.head_stride * head * 16;
    const char* vbase = p.c.v + p.c.head_stride * head * 16;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(lds_offset(s_ring));
    auto tile_of = [&](int i) { return ring_at + (i & (kBlockRing - 1)) * (2 * TILE); };
    auto fetch = [&](int i) {
        const int j0 = tile_at(range, begin + i) * KEYS;
        const int* ids = s_ids + (i & (kIdTiles - 1)) * per;
        const uint32_t to = ring_at + (i & (kBlockRing - 1)) * (2 * TILE);
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
            const int x = (wave * MINE + m) % LOADS;
            const int64_t off = piece_offset<G>(p.c, ids, j0, range.end, x);
            load_to_lds<ONCE>(kbase + off, to + x * 1024);
            load_to_lds<ONCE>(vbase + off, to + TILE + x * 1024);
        }
    };
    auto barrier = [&]() {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    // tile i is there for everybody, tile i - 2 done with, and tile i + 2 on its way
    auto arrive = [&](int i) {
        if (i + 1 < n) wait_loads<2 * MINE>(); else wait_loads<0>();
        barrier();
        if (i + 2 < n) {
            if (((i + 2) & (kIdTiles - 1)) == 0) {
                page_ids<KEYS, THREADS>(p.c, seq, range, begin + i + 2, min(n - i - 2, kIdTiles), per, s_ids);
                barrier();
            }
            fetch(i + 2);
        }
    };
    auto scores = [&](int i, f32x4 (&s)[NB][Q]) { core.scores(C::k_base(tile_of(i)), s); };
    // What the wavefront's rows see lies below see_hi and, but for the sinks, from see_lo on.
    const int wt0 = (r0 + w0) / p.group, wt1 = (r0 + min(w0 + 16 * NB, n_rows) - 1) / p.group;
    const int see_hi = w0 >= n_rows ? 0 : p.parents ? range.end : min(range.end, len + wt1 + 1);
    const int see_lo = !p.window ? 0 : max(0, len + (p.parents ? 0 : wt0) - p.window + 1);
    // tiles that some row does not see all of
    auto edge = [&](int from, int to) {
        RowSees row[NB];
        sees_of(fresh(), row);
        for (int i = from; i < to; ++i) {
            arrive(i);
            bool bad = false;
#pragma unroll
            for (int m = 0; m < MINE; ++m) bad |= take_out<G>(tile_of(i) + TILE, (wave * MINE + m) % LOADS);
            if (bad) s_spoilt = 1;
            barrier();
            // (a wavefront that sees nothing of the tile only keeps the others' time)
            const int j0 = tile_at(range, begin + i) * KEYS;
            if (j0 >= see_hi || (j0 + KEYS <= see_lo && j0 >= p.sinks)) continue;
            f32x4 s[NB][Q];
            scores(i, s);
            apply_sees(s, row, j0, p.sinks, len);
            soft.step(core, s, p.scale_log2);
            const uint32_t v = C::v_base(tile_of(i) + TILE);
#pragma unroll
            for (int b = 0; b < SUB; ++b) {
                typename C::Weights w;
                C::pack(s, b * C::MT, w);
                core.add_values(v, b * G::KEYS, w);
            }
        }
    };
    // the others: the second product lags one tile behind the first, so that both are at hand together
    auto middle = [&](int from, int to) {
        if (w0 >= n_rows) {                               // a wavefront without rows keeps the others' time
            for (int i = from; i < to; ++i) arrive(i);
            return;
        }
        if (from >= to) return;
        f32x4 s[NB][Q];
        typename C::Weights w[SUB];
        auto weigh = [&]() {
            soft.step(core, s, p.scale_log2);
#pragma unroll
            for (int b = 0; b < SUB; ++b) C::pack(s, b * C::MT, w[b]);
        };
        auto values = [&](int i) {
            const uint32_t v = C::v_base(tile_of(i) + TILE);
#pragma unroll
            for (int b = 0; b < SUB; ++b) core.add_values(v, b * G::KEYS, w[b]);
        };
        arrive(from);
        scores(from, s);
        for (int i = from + 1; i < to; ++i) {
            arrive(i);
            weigh();
            scores(i, s);
            values(i - 1);
            C::template schedule_products<SUB>();
        }
        weigh();
        values(to - 1);
    };

    // [edge][middle][edge] of the share; the middle is what everybody sees all of
    const int mid0 = min(n, max(0, range.sink_tiles + max(0, (range.from + KEYS - 1) / KEYS - range.first) - begin));
    const int mid1 = min(n, max(mid0, range.sink_tiles + range.sure / KEYS - range.first - begin));
    if (n > 0) fetch(0);
    if (n > 1) fetch(1);
    edge(0, mid0);
    middle(mid0, mid1);
    edge(mid1, n);

    RowSees row[NB];
    sees_of(fresh(), row);
    if (s_spoilt)                                         // (set in front of a barrier that everybody has passed)
        put_back<E, D, NB, KEYS>(p, core, row, vbase, seq, len, range.end, n,
                                 [&](int i) { return i >= mid0 && i < mid1 ? -1 : tile_at(range, begin + i) * KEYS; });
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = 16 * nb + (lane & 15) + w0;
        const bool alive = row[nb].hi > 0 || row[nb].tree;
        const float l = alive ? column_sum(soft.l[nb]) : 0.f;
        if (r >= n_rows) continue;
        if (shares > 1) {
            const size_t at = (size_t)(u.first + u.share) * ROWS + r;
#pragma unroll
            for (int y = 0; y < C::OB; ++y) *(f32x4*)(p.part_o + at * D + C::quad_dim(y)) = core.quad(nb, y);
            if (lane < 16) p.part_ml[at] = make_float2(alive ? soft.m[nb] : -INFINITY, l);
        } else {
            const int t = (r0 + r) / p.group, h = head * p.group + (r0 + r) % p.group;
            char* out = p.out + (int64_t)(u.first_row + t) * p.out_stride + (int64_t)h * (D * G::ES);
            const f32x4 zero = {0, 0, 0, 0};
            const float inv = 1.f / l;
#pragma unroll
            for (int y = 0; y < C::OB; ++y) store_quad<E>(out, C::quad_dim(y), l == 0.f ? zero : core.quad(nb, y) * inv);
        }
    }
}

// The shares of attn_block_kernel's rows, spread over the chip: 9 us of 226 for wide trees, whose blocks have 256 rows of
// 20 shares; a workgroup that joins all of a block by itself takes 75 us longer.  At least kJoinRows rows to a
// workgroup, and no more than about kJoinGrid workgroups: each works out for itself what the blocks were cut into.
// 3 x 777 rows in fp32, of which nothing is cut: 111 us; with 9984 workgroups that find so 123; without the launch 107.
constexpr int kJoinRows = 8;
constexpr int kJoinGrid = 1024;
template <typename E, int D, int NB>
__global__ void __launch_bounds__(256) attn_join_kernel(const AttnParams p) {
    constexpr int ROWS = 16 * NB * Block<E>::WAVES;
    constexpr int KEYS = Block<E>::SUB * Geo<E, D>::KEYS;
    __shared__ Unit s_unit;
    const int join_rows = p.join_rows, parts = ROWS / join_rows, block = blockIdx.x / parts, part = blockIdx.x - block * parts;
    const int per_entry = p.row_blocks * p.c.n_heads;
    if (threadIdx.x < 64) Units<KEYS, ROWS>(p, 8).find_block(block / per_entry, block % per_entry, &s_unit);
    __syncthreads();
    const Unit u = uniform(s_unit);
    if (u.rows == 0 || u.seq < 0 || u.n_rows <= part * join_rows) return;
    const Range range = key_range<KEYS>(p, u.len, u.rows, u.r0 / p.group, (u.r0 + u.n_rows - 1) / p.group);
    const int shares = u.cut(range.tiles);
    if (shares > 1)
        join_shares<E, D, ROWS, 256, false>(p, u.first, shares, u.first_row, u.head, u.r0, part * join_rows, min(u.n_rows, (part + 1) * join_rows));
}

// ---- launch plan ----------------------------------------------------------------------------------
struct Plan {
    bool shared;              // attn_block_kernel
    int nb, rows, waves, row_blocks, slots, join_rows;
    int64_t blocks, grid;
    bool cut;                 // blocks may be cut into shares (slots > 0)
    bool once;                // keys and values pass by the caches
    size_t off_ml, off_tickets, total;
};
int reach(const dip_kv_cache* c, const dip_batch* b) {
    const int fit = c->max_pages * c->page_size;
    return b->max_len && b->max_len < fit ? b->max_len : fit;
}
// Non-temporal loads of keys and values from here on (bytes of a call), where one block of rows is all that reads
// them.  At 170 MB and more of bf16: 49.3 -> 45.9 us (8 trees of 8 nodes), 78.4 -> 74.8 (32 tokens), 224 -> 210
// (32 tokens over 12000 keys).  Less may still be in the last-level cache (256 MB) when it is read again, and what
// several blocks read should stay there: 39 MB 19.4 -> 20.1 us, 4 MB 10.6 -> 11.0.  (Of two
// kernels: asking for each load costs more than it gains, 2 to 4 %.  fp32 blocks wait for their products: 184 us and 184.)
constexpr double kOnceBytes = 64 << 20;
Plan plan_attention(const dip_kv_cache* c, const dip_batch* b, int n_q_heads, int window, int sinks) {
    Plan pl;
    const int64_t rows = (int64_t)rows_bound(b) * (n_q_heads / c->n_kv_heads);
    const bool bf16 = c->dtype == DIP_BF16;
    const int block_waves = bf16 ? Block<uint16_t>::WAVES : Block<float>::WAVES;
    pl.shared = rows > 64;
    pl.nb = pl.shared ? (!bf16 || rows <= 16 * block_waves ? 1 : 2) : rows <= 16 ? 1 : rows <= 32 || (!bf16 && c->head_dim == 128) ? 2 : 4;
    // (fp32 at 128 dims: four blocks of 16 rows do not fit the registers)
    pl.rows = 16 * pl.nb * (pl.shared ? block_waves : 1);
    pl.row_blocks = (int)((rows + pl.rows - 1) / pl.rows);
    pl.blocks = (int64_t)b->n_batch * c->n_kv_heads * pl.row_blocks;
    // Four wavefronts to a workgroup, as many workgroups to a compute unit as their rings of tiles leave room for;
    // where the blocks alone are more than that, two: the start and the end of one workgroup, when it streams
    // nothing, then lie beside another's middle (32 tokens over up to 12000 keys 201 us, with four 262; 8 trees of 8
    // nodes 44 us with four, 54 with two).
    const auto fit = [&](int waves) { return 256 * ((160 * 1024 - 1024) / (waves * 256 * c->head_dim + 6144)); };
    pl.waves = pl.shared ? block_waves : pl.blocks <= fit(4) ? 4 : 2;
    pl.slots = !pl.shared ? fit(pl.waves) : bf16 ? 256 : 256 * (160 * 1024 / (512 * c->head_dim + 5120));
    // attn_block_kernel's shares are joined by a launch of its own, which costs 4 us even where there turn out to be
    // none: with far more blocks than the chip holds at a time none are made (2 x 4096 rows 467 us, else 471; but uncut, 4
    // trees of 64 nodes take 1685 us, 2 x 100 rows 175 instead of 37)
    pl.cut = !pl.shared || pl.blocks < 4 * pl.slots;
    if (!pl.cut) pl.slots = 0;
    int64_t keys = reach(c, b);
    if (window) keys = std::min(keys, (int64_t)window + sinks + rows_bound(b));
    pl.once = pl.row_blocks == 1 && (double)keys * b->n_batch * c->n_kv_heads * c->head_dim * 2 * elem_bytes(c->dtype) >= kOnceBytes;
    pl.join_rows = pl.rows;
    while (pl.join_rows > kJoinRows && pl.blocks * (pl.rows / pl.join_rows) < kJoinGrid) pl.join_rows /= 2;
    pl.grid = pl.blocks > pl.slots ? pl.blocks : pl.slots;
    size_t o = 0;
    // (only a cut into at most `slots` units has shares)
    const size_t units = (size_t)pl.slots;
    o = align_up(units * pl.rows * c->head_dim * sizeof(float), 256);
    pl.off_ml = o;
    o += align_up(units * pl.rows * sizeof(float2), 256);
    pl.off_tickets = o;
    if (!pl.shared) o += sizeof(uint64_t) * kTicketStride * units;
    pl.total = o < 256 ? 256 : o;
    return pl;
}

template <typename E, int D, int NB>
hipError_t launch_rows(const AttnParams& p, const Plan& pl, hipStream_t stream) {
    const dim3 grid((unsigned)p.grid), block(pl.waves * 64);
    const auto go = [&](auto kernel) { return launch_timed(kernel, grid, block, stream, DIP_KERNEL_ATTENTION, p); };
    if (pl.waves == 4) return pl.once ? go(attn_rows_kernel<E, D, NB, 4, true>) : go(attn_rows_kernel<E, D, NB, 4, false>);
    return pl.once ? go(attn_rows_kernel<E, D, NB, 2, true>) : go(attn_rows_kernel<E, D, NB, 2, false>);
}
template <typename E, int D, int NB>
hipError_t launch_block(const AttnParams& p, const Plan& pl, hipStream_t stream) {
    const dim3 grid((unsigned)((p.grid + 7) / 8 * 8));
    const auto go = [&](auto kernel) { return launch_timed(kernel, grid, dim3(Block<E>::WAVES * 64), stream, DIP_KERNEL_ATTENTION, p); };
    hipError_t err;
    if constexpr (sizeof(E) == 2) err = pl.once ? go(attn_block_kernel<E, D, NB, true>) : go(attn_block_kernel<E, D, NB, false>);
    else err = go(attn_block_kernel<E, D, NB, false>);
    if (err != hipSuccess || !pl.cut) return err;
    const dim3 join((unsigned)(pl.blocks * (pl.rows / p.join_rows)));
    return launch_timed(attn_join_kernel<E, D, NB>, join, dim3(256), stream, DIP_KERNEL_ATTENTION, p);
}
template <typename E, int D>
int32_t launch(const AttnParams& p, const Plan& pl, hipStream_t stream) {
    hipError_t err;
    if (pl.shared) {
        if (pl.nb == 1) err = launch_block<E, D, 1>(p, pl, stream);
        else if constexpr (sizeof(E) == 2) err = launch_block<E, D, 2>(p, pl, stream);
        else return fail(DIP_ERR_UNSUPPORTED, "attention: no kernel for this shape");
        return check_hip(err, "attention launch");
    }
    if (pl.nb == 1) err = launch_rows<E, D, 1>(p, pl, stream);
    else if (pl.nb == 2) err = launch_rows<E, D, 2>(p, pl, stream);
    else if constexpr (sizeof(E) == 2 || D < 128) err = launch_rows<E, D, 4>(p, pl, stream);
    else return fail(DIP_ERR_UNSUPPORTED, "attention: no kernel for this shape");
    return check_hip(err, "attention launch");
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
    if ((pl.grid + 8) * pl.waves * 64 >= (int64_t)1 << 32)    // threads of a launch
        return fail(DIP_ERR_UNSUPPORTED, "attention: too many rows for one call");
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
    p.group = n_q_heads / c->n_kv_heads;
    p.scale_log2 = scale * 1.44269504088896340736f;
    p.window = window;
    p.sinks = sinks;
    p.max_len = reach(c, b);
    p.slots = pl.slots;
    p.grid = (int)pl.grid;
    p.row_blocks = pl.row_blocks;
    p.join_rows = pl.join_rows;
    p.part_o = (float*)ws;
    p.part_ml = (float2*)((char*)ws + pl.off_ml);
    p.tickets = (uint64_t*)((char*)ws + pl.off_tickets);
    p.epoch = next_epoch();
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
