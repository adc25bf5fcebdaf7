// What the attention kernels share: which keys a block of rows sees, key/value tiles in LDS, the two
// matrix-core products of a tile and the running softmax between them.
//
// For a block of rows r (n = r % 16 the column of a product) and the keys m of a tile
//     S^T = K Q^T          [keys x rows]     16x16 products, K from LDS, Q^T in registers
//     P^T = exp2(c S^T - max)                in the registers that S^T came out in
//     O^T = O^T + V^T P^T  [dims x rows]     V^T from LDS
// A lane (column n = lane % 16, g = lane / 16) gets S^T of keys 4 g + i, i < 4, of each 16 keys, and that is
// what the second product takes from it if V's keys come in the same order: P never leaves its lane.  A row's
// maximum is one value per column, so rescaling O^T is a product with a lane's own number.
#ifndef DIP_ATTN_DEVICE_H_
#define DIP_ATTN_DEVICE_H_

#include <type_traits>

#include "dip_decode_internal.h"

namespace dip {
namespace attn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

struct AttnParams {
    KvView c;                 // k and v already at the layer
    BatchView b;
    const int32_t* parents;   // null: window attention
    const char* q;
    char* out;
    int64_t q_stride;         // bytes
    int64_t out_stride;
    int group;                // query heads of a key/value head
    float scale_log2;         // scale * log2(e)
    int window;               // 0: no bound
    int sinks;
    int max_len;
    int slots;                // workgroups that the chip holds at a time, or what to pretend it does
    int grid;                 // most units there can be
    int row_blocks;           // most blocks of rows of an entry and key/value head
    int join_rows;            // of a workgroup of attn_join_kernel
    float* part_o;            // [unit][rows of a block][D], not normalised
    float2* part_ml;          // [unit][rows of a block]: maximum (times scale_log2), sum
    uint64_t* tickets;        // a word per unit, kTicketStride apart, whatever they hold
    uint64_t epoch;           // this launch's tag in them
};

// ---- which keys a block of rows sees -----------------------------------------------------------
struct Range {
    int tiles;                // tiles of KEYS positions that some row sees: the sinks' first ...
    int sink_tiles;
    int first;                // ... then those from here on
    int end;                  // no row sees position `end` or anything behind it
    int sure;                 // every row sees all positions below `sure` ...
    int from;                 // ... from `from` on, and the sinks
};
template <int KEYS>
__device__ __forceinline__ Range key_range(const AttnParams& p, int len, int rows, int t0, int t1) {
    Range r;
    int lo;                   // first position behind the sinks that some row sees
    if (p.parents) {          // rows stand at len + depth, 0 <= depth < rows
        r.end = len + rows;
        r.sure = len;
        lo = p.window ? max(0, len - p.window + 1) : 0;
        r.from = p.window ? max(0, len + rows - p.window) : 0;
    } else {
        r.end = len + t1 + 1;
        r.sure = len + t0 + 1;
        lo = p.window ? max(0, len + t0 - p.window + 1) : 0;
        r.from = p.window ? max(0, len + t1 - p.window + 1) : 0;
    }
    r.end = min(r.end, p.max_len);
    r.sure = min(r.sure, p.max_len);
    const int last = (r.end + KEYS - 1) / KEYS;
    if (p.sinks >= lo) {
        r.sink_tiles = 0;
        r.first = 0;
    } else {
        r.sink_tiles = (min(p.sinks, r.end) + KEYS - 1) / KEYS;
        r.first = max(lo / KEYS, r.sink_tiles);
    }
    r.tiles = r.sink_tiles + max(0, last - r.first);
    return r;
}
__device__ __forceinline__ int tile_at(const Range& r, int vt) { return vt < r.sink_tiles ? vt : r.first + vt - r.sink_tiles; }

// what one row sees
struct RowSees {
    int lo, hi;               // positions [lo, hi) and sinks below hi ...
    uint64_t tree;            // ... and nodes of its tree
};
// As a bit for each of the 64 positions from j0 on.
__device__ __forceinline__ uint64_t below(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }
__device__ __forceinline__ uint64_t sees(const RowSees& r, int j0, int sinks, int len) {
    uint64_t bits = below(r.hi - j0) & (~below(r.lo - j0) | below(sinks - j0));
    const int at = len - j0;                              // of node 0
    if (at > -64 && at < 64) bits |= at >= 0 ? r.tree << at : r.tree >> -at;
    return bits;
}

// The ancestors of every node of an entry's tree, itself among them (0: the node is absent), into LDS by
// one wavefront: pointers jump 1, 2, 4 .. steps up.
__device__ __forceinline__ void tree_masks(const int32_t* parents, int rows, uint64_t* out) {
    const int lane = threadIdx.x & 63;
    int up = lane < rows ? parents[lane] : -2;
    if (up < -1 || up >= lane) up = -2;
    uint64_t mask = 1ull << lane;
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        const int at = up < 0 ? lane : up;
        const uint32_t lo = __shfl((uint32_t)mask, at), hi = __shfl((uint32_t)(mask >> 32), at);
        const int next = __shfl(up, at);
        if (up >= 0) {
            mask |= ((uint64_t)hi << 32) | lo;
            up = next;
        }
    }
    out[lane] = up == -1 ? mask : 0;
}

// (Nothing from max_len on: a tile that it cuts holds other positions' keys there.)
__device__ __forceinline__ RowSees row_sees(const AttnParams& p, int len, int t, const uint64_t* masks) {
    RowSees r;
    int pos = len + t;
    r.tree = 0;
    if (p.parents) {
        r.tree = masks[t];
        pos = len + __popcll(r.tree) - 1;
        r.hi = r.tree ? len : 0;
        r.tree &= below(p.max_len - len);
    } else {
        r.hi = pos + 1;
    }
    r.hi = min(r.hi, p.max_len);
    r.lo = p.window ? max(0, pos - p.window + 1) : 0;
    return r;
}

// ---- units of work ---------------------------------------------------------------------------
// A unit is a block of rows (of an entry and key/value head) and a share of the tiles that it sees.  How long the
// sequences are is known on the device alone, so every workgroup cuts the work up for itself, all alike:
// shares of `size` tiles, the smallest size that makes no more units than the chip holds at a time -- one
// round, of units as alike as can be whatever the lengths.  (With blocks enough for that, a block is a unit.)
struct Unit {
    int entry, first_row, rows, seq, len;      // rows == 0: no unit
    int head, r0, n_rows;                      // its rows: r0 .. r0 + n_rows - 1 of rows x group
    int first;                                 // unit of the block's first share
    int share, shares, size;                   // this one begins at tile share * size, the last takes all that is left
    // how many shares a block that sees `tiles` tiles is cut into, and where this one ends
    __device__ __forceinline__ int cut(int tiles) const { return min(shares, (tiles + size - 1) / size); }
    __device__ __forceinline__ int end(int tiles) const { return share + 1 >= cut(tiles) ? tiles : min(tiles, (share + 1) * size); }
};
// (the same for all lanes: into scalar registers)
__device__ __forceinline__ Unit uniform(const Unit& u) {
    Unit x;
    constexpr int N = sizeof(Unit) / sizeof(int);
    int raw[N];
    __builtin_memcpy(raw, &u, sizeof(u));
#pragma unroll
    for (int i = 0; i < N; ++i) raw[i] = __builtin_amdgcn_readfirstlane(raw[i]);
    __builtin_memcpy(&x, raw, sizeof(x));
    return x;
}
template <int KEYS, int ROWS>
struct Units {
    struct Entry {
        int first, rows, seq, len, row_blocks, blocks, tiles;
    };
    const AttnParams& p;
    Entry cached;
    int size;
    float per_size;
    int total;
    __device__ __forceinline__ Entry entry(int e) const {
        Entry x = {0, 0, -1, 0, 0, 0, 0};
        if (e >= p.b.n_batch) return x;
        const EntryRows er = entry_rows(p.b, e);
        x.first = er.first;
        x.rows = er.rows;
        x.seq = entry_seq(p.b, p.c, e);
        x.len = x.seq >= 0 ? entry_len(p.c, x.seq) : 0;
        const int all = er.rows * p.group;
        x.row_blocks = (all + ROWS - 1) / ROWS;
        x.blocks = x.row_blocks * p.c.n_heads;
        if (all > 0) {            // (about as many as any of its blocks sees; one that sees nothing is a unit all the same)
            const Range r = key_range<KEYS>(p, x.len, er.rows, max(0, all - ROWS) / p.group, er.rows - 1);
            x.tiles = x.seq >= 0 ? max(1, r.tiles) : 1;
        }
        return x;
    }
    __device__ __forceinline__ Entry at(int chunk) const { return chunk == 0 ? cached : entry(chunk * 64 + (int)(threadIdx.x & 63)); }
    // (a share more or less does not matter, as long as everybody says the same: the last one takes what is left)
    __device__ __forceinline__ int shares_of(const Entry& x) const { return max(1, (int)ceilf((float)x.tiles * per_size)); }
    __device__ __forceinline__ int units_of(const Entry& x) const { return x.blocks * shares_of(x); }
    // running sums over the lanes in data-parallel moves within rows of 16, then the rows' sums by scalar
    __device__ __forceinline__ static int running(int x) {
        x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);      // row_shr 1, 2, 4, 8
        x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
        const int a = __builtin_amdgcn_readlane(x, 15), b = __builtin_amdgcn_readlane(x, 31), c = __builtin_amdgcn_readlane(x, 47);
        const int row = (threadIdx.x & 63) >> 4;
        return x + (row > 0 ? a : 0) + (row > 1 ? b : 0) + (row > 2 ? c : 0);
    }
    __device__ __forceinline__ static int sum(int x) { return __builtin_amdgcn_readlane(running(x), 63); }
    __device__ __forceinline__ static float sum_of(float x) {
        const auto from = [](float y, auto ctrl) {
            return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(y), decltype(ctrl)::value, 0xf, 0xf, true));
        };
        x += from(x, std::integral_constant<int, 0x111>());
        x += from(x, std::integral_constant<int, 0x112>());
        x += from(x, std::integral_constant<int, 0x114>());
        x += from(x, std::integral_constant<int, 0x118>());
        const auto row = [&](int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane)); };
        return (row(15) + row(31)) + (row(47) + row(63));
    }
    __device__ __forceinline__ static int least_of(int x) {
        x = min(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
        x = min(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
        x = min(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
        x = min(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
        return min(min(__builtin_amdgcn_readlane(x, 15), __builtin_amdgcn_readlane(x, 31)),
                   min(__builtin_amdgcn_readlane(x, 47), __builtin_amdgcn_readlane(x, 63)));
    }
    // one wavefront; all its lanes get the answer
    __device__ __forceinline__ Units(const AttnParams& params, int least) : p(params) {
        cached = entry(threadIdx.x & 63);
        const int chunks = (p.b.n_batch + 63) / 64;
        float work = 0.f;                                  // (the same bits for everybody: that is all it takes)
        int most = -1;
        total = 0;
        for (int c = 0; c < chunks; ++c) {
            const Entry x = at(c);
            total += sum(x.blocks);
            most = max(most, -least_of(-x.tiles));
            work += sum_of((float)x.blocks * (float)x.tiles);
        }
        whole(max(1, most));
        if (total >= p.slots) return;
        int next = max(least, (int)(work / (float)p.slots));
        while (next < most) {
            set(next);
            // the units there would be, and the next size at which some entry has a share less
            int units = 0, step = most;
            for (int c = 0; c < chunks; ++c) {
                const Entry x = at(c);
                units += sum(units_of(x));
                const int k = shares_of(x);
                step = min(step, least_of(k > 1 ? (int)ceilf((float)x.tiles / (float)(k - 1)) : most));
            }
            if (units <= p.slots) {
                total = units;
                return;
            }
            next = max(next + 1 + (next >> 5), step);
        }
        whole(max(1, most));
    }
    __device__ __forceinline__ void set(int n) {
        size = n;
        per_size = 1.f / (float)n;
    }
    __device__ __forceinline__ void whole(int most) {      // every block one unit, to the letter
        size = most;
        per_size = 0.f;
    }
    // the unit `w`, or the first one of block `b` of entry `e`
    __device__ __forceinline__ void find(int w, Unit* out) const {
        const int lane = threadIdx.x & 63;
        int before = 0;
        for (int c = 0; c * 64 < p.b.n_batch; ++c) {
            const Entry x = at(c);
            const int upto = running(units_of(x));
            const int mine = before + upto - units_of(x);
            if (w >= mine && w < before + upto) fill(x, c * 64 + lane, mine, w - mine, out);
            before += __builtin_amdgcn_readlane(upto, 63);
            if (w < before) return;
        }
        if (lane == 0) out->rows = 0;
    }
    __device__ __forceinline__ void find_block(int e, int block, Unit* out) const {
        const int lane = threadIdx.x & 63;
        int before = 0;
        for (int c = 0; c * 64 <= e; ++c) {
            const Entry x = at(c);
            const int mine = c * 64 + lane < e ? units_of(x) : 0;
            before += sum(mine);
            if (c * 64 + lane == e) {
                const int shares = shares_of(x);
                if (block < x.blocks) fill(x, e, -1, block * shares, out);
                else out->rows = 0;
            }
        }
        if (lane == (e & 63) && out->rows) out->first += before + 1;
    }
    __device__ __forceinline__ void fill(const Entry& x, int e, int at_unit, int local, Unit* out) const {
        const int shares = shares_of(x), block = local / shares;
        out->entry = e;
        out->first_row = x.first;
        out->rows = x.rows;
        out->seq = x.seq;
        out->len = x.len;
        out->head = block / x.row_blocks;
        out->r0 = (block - out->head * x.row_blocks) * ROWS;
        out->n_rows = min(ROWS, x.rows * p.group - out->r0);
        out->first = at_unit + block * shares;
        out->share = local - block * shares;
        out->shares = shares;
        out->size = size;
    }
};

// The page numbers of `tiles` tiles from virtual tile `from` on, `per` of each, by the threads of a workgroup or
// of a wavefront (numbers that are none become page 0).
template <int KEYS, int THREADS>
__device__ __forceinline__ void page_ids(const KvView& c, int seq, const Range& range, int from, int tiles, int per, int* ids) {
    for (int i = threadIdx.x & (THREADS - 1); i < tiles * per; i += THREADS) {
        const int vt = i / per;
        const int at = ((tile_at(range, from + vt) * KEYS) >> c.page_shift) + (i - vt * per);
        const int page = at < c.max_pages ? c.table[(size_t)seq * c.max_pages + at] : 0;
        ids[i] = (unsigned)page < (unsigned)c.n_pages ? page : 0;
    }
}

// ---- tiles in LDS --------------------------------------------------------------------------------
// KEYS rows of D elements, 16-byte pieces swizzled so that 16 rows' pieces of one dim (a K operand) and
// the 16 pieces of a row (a V operand) both fall on different banks.  Filled by loads that go to LDS
// directly, each lane fetching the piece that belongs at its place.
template <typename E, int D>
struct Geo {
    static constexpr int ES = sizeof(E);
    static constexpr int ROWB = D * ES;
    static constexpr int CPR = ROWB / 16;                  // pieces of a row
    static constexpr int KEYS = ES == 2 ? 32 : 16;         // of one step of the products
    static constexpr int ROT = CPR == 12 ? 4 : CPR == 8 || CPR == 24 ? 8 : 16;
    // piece c of a row lies at c ^ twist(row): the low bits only, in which a row's start has none
    __device__ static __forceinline__ int twist(int row) {
        static_assert(CPR == 8 || CPR == 12 || CPR == 16 || CPR == 24 || CPR == 32, "row length");
        return ROT == 16 ? row & 15 : ROT == 8 ? (row >> 1) & 7 : (row >> 2) & 3;
    }
    // Where piece c + l of the rows row + 16 x (l < 4 a lane's part, c a multiple of 4, or l < 2 and of 2) lies, from
    // base = row_at(row, l): one register for all c and x.
    __device__ static __forceinline__ uint32_t row_at(int row, int l) { return row * ROWB + ((l ^ twist(row)) << 4); }
    __device__ static __forceinline__ const lds_char* at(uint32_t base, int c, int rows) {
        return (const lds_char*)(size_t)((base ^ ((c & (ROT - 1)) * 16)) + (c & ~(ROT - 1)) * 16 + rows * ROWB);
    }
};

__device__ __forceinline__ uint32_t lds_offset(const void* p) { return (uint32_t)(size_t)(const lds_char*)p; }

// 64 x 16 bytes from the lanes' addresses to LDS at `to` + 16 * lane.  Written in assembly because the
// compiler would make every later LDS read wait for all of them; nothing but the counter says that they are
// there, so readers wait with wait_loads().  (The load writes no register; m0 is put back.)  ONCE: non-temporal.
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const char* from, uint32_t to) {
    uint32_t m0;
    if constexpr (ONCE)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0) : "v"(from), "s"(to) : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0) : "v"(from), "s"(to) : "memory");
}
// This lane's 16 bytes of load x of a tile: `off` from the start of the head.  ids: the tile's page numbers.
template <typename G>
__device__ __forceinline__ int64_t piece_offset(const KvView& c, const int* ids, int j0, int end, int x) {
    const int at = x * 64 + (threadIdx.x & 63), r = at / G::CPR;
    const int pos = min(j0 + r, end - 1), shift = c.page_shift;
    const int page = ids[(pos >> shift) - (j0 >> shift)];
    return (page * c.page_stride + (pos & ((1 << shift) - 1)) * c.slot_stride + ((at % G::CPR) ^ G::twist(r))) * 16;
}
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Load x of a V tile in LDS: what is not finite in this lane's piece becomes zero, so that a weight of zero takes it
// out; whether there was any.  (Only tiles that some row does not see all of are looked through: in the others what
// is not finite belongs in the results.)
template <typename G>
__device__ __forceinline__ bool take_out(uint32_t v, int x) {
    const int lane = threadIdx.x & 63;
    auto* at = (__attribute__((address_space(3))) u32x4*)(lds_char*)(size_t)(v + x * 1024 + lane * 16);
    u32x4 w = *at;
    bool inf = false;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        inf |= (w[y] & 0x7f800000u) == 0x7f800000u;
        if constexpr (G::ES == 2) inf |= (w[y] & 0x7f80u) == 0x7f80u;
    }
    if (!inf) return false;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        if ((w[y] & 0x7f800000u) == 0x7f800000u) w[y] &= G::ES == 2 ? 0xffffu : 0u;
        if constexpr (G::ES == 2)
            if ((w[y] & 0x7f80u) == 0x7f80u) w[y] &= 0xffff0000u;
    }
    *at = w;
    return true;
}
// ---- the two products ----------------------------------------------------------------------------
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// maximum / sum over the four lanes of a column (lane ^ 16, lane ^ 32)
__device__ __forceinline__ float column_max(float x) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float column_sum(float x) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// NB blocks of 16 rows of one wavefront.
template <typename E, int D, int NB>
struct Core;

template <int D, int NB>
struct Core<uint16_t, D, NB> {
    typedef Geo<uint16_t, D> G;
    static constexpr int KEYS = 32, MT = 2, OB = D / 16, QS = D / 32;
    bf16x8 q[NB][QS];
    f32x4 o[NB][OB];

    __device__ __forceinline__ void load_q(int nb, const char* row) {      // row: the lane's column, or null
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            u32x4 x = {0, 0, 0, 0};
            if (row) x = *(const u32x4*)(row + (4 * s + ((threadIdx.x & 63) >> 4)) * 16);
            q[nb][s] = __builtin_bit_cast(bf16x8, x);
        }
    }
    // where a lane's reads of K and of V start in a tile; opaque, so that what is added to them is added where it is
    // used instead of being kept in a register each
    __device__ __forceinline__ static uint32_t k_base(uint32_t tile) {
        uint32_t x = tile + G::row_at(threadIdx.x & 15, (threadIdx.x & 63) >> 4);
        asm volatile("" : "+v"(x));
        return x;
    }
    __device__ __forceinline__ static uint32_t v_base(uint32_t tile) {
        const int i = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
        uint32_t x = tile + G::row_at(4 * g + (i >> 2), (i & 3) >> 1) + (i & 1) * 8;
        asm volatile("" : "+v"(x));
        return x;
    }
    // scores of a tile of 16 Q keys: s[nb][x][i] is key 16 x + 4 g + i.  The blocks of 16 keys go side by side, so that
    // a product does not wait for the one before it.
    template <int Q>
    __device__ __forceinline__ void scores(uint32_t k, f32x4 (&s)[NB][Q]) const {
#pragma unroll
        for (int st = 0; st < QS; ++st)
#pragma unroll
            for (int x = 0; x < Q; ++x) {
                const bf16x8 a = *(const __attribute__((address_space(3))) bf16x8*)G::at(k, 4 * st, 16 * x);
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    s[nb][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[nb][st], st ? s[nb][x] : f32x4{0, 0, 0, 0}, 0, 0, 0);
            }
    }
    // The weights of KEYS keys as the second product takes them: two bf16 terms, the upper half of the fp32 number and
    // what that leaves, rounded: 2^-15 of a weight.  With one term, off by up to 2^-8 where a few keys carry a row, a
    // call's relative error is 0.0023, with two 0.0017, which the rounding of its output alone is (prompts 389 us instead
    // of 479, trees of 64 nodes 180 instead of 227).  What is left of a weight above zero counts as at least 2^-23 of it, so
    // that an infinite value times either term has its sign and never meets a zero.
    struct Weights {
        bf16x8 w[NB], rest[NB];
    };
    __device__ __forceinline__ static float upper(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
    template <int Q>
    __device__ __forceinline__ static void pack(const f32x4 (&p)[NB][Q], int at, Weights& x) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float a = p[nb][at + (e >> 2)][e & 3], b = p[nb][at + (e >> 2)][(e & 3) + 1];
                const bf16x2 both = __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u));
                x.w[nb][e] = both[0];
                x.w[nb][e + 1] = both[1];
                x.rest[nb][e] = (__bf16)fmaf(a, 1.f + 0x1p-23f, -upper(a));
                x.rest[nb][e + 1] = (__bf16)fmaf(b, 1.f + 0x1p-23f, -upper(b));
            }
    }
    __device__ __forceinline__ void add_values(uint32_t v, int key, const Weights& p) {
#pragma unroll
        for (int db = 0; db < OB; ++db) {
            // four keys at this lane's dim each: the transposing read hands lane i column i of 4 rows x 16 dims
            bf16x8 a;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)G::at(v, 2 * db, key + 16 * half));
                const bf16x4 y = __builtin_bit_cast(bf16x4, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) a[4 * half + e] = y[e];
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p.w[nb], o[nb][db], 0, 0, 0);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) o[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p.rest[nb], o[nb][db], 0, 0, 0);
        }
    }
    // Behind a tile's two products (SUB KEYS keys): reads run FLIGHT operands ahead of the products that take them.
    // An operand of K serves NB products, one of V, with two terms, 2 NB.
    // (Left to itself the compiler reads each right before its use, to save registers: prompts 560 us instead of 484.)
    template <int SUB>
    __device__ __forceinline__ static void schedule_products() {
        constexpr int KF = SUB * MT * QS, VF = SUB * OB, FLIGHT = 4;       // operands of K, of V (two reads each)
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
        for (int f = FLIGHT; f < KF; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x8, NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x8, NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
#pragma unroll
        for (int f = FLIGHT; f < VF; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x8, 2 * NB, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, FLIGHT * 2 * NB, 0);
    }
    // Behind a tile's second product alone.
    __device__ __forceinline__ static void schedule_values() {
        constexpr int FLIGHT = 4;
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
#pragma unroll
        for (int f = FLIGHT; f < OB; ++f) {
            __builtin_amdgcn_sched_group_barrier(0x8, 2 * NB, 1);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, 2 * FLIGHT * NB, 1);
    }
    // first dim of the four that o[nb][x] .. hold: quad y of them, y < OB
    __device__ __forceinline__ static int quad_dim(int y) { return 16 * y + 4 * ((threadIdx.x & 63) >> 4); }
    __device__ __forceinline__ f32x4 quad(int nb, int y) const { return o[nb][y]; }
    __device__ __forceinline__ void add_quad(int nb, int y, f32x4 x) { o[nb][y] += x; }
};

template <int D, int NB>
struct Core<float, D, NB> {
    typedef Geo<float, D> G;
    static constexpr int KEYS = 16, MT = 1, OB = D / 16, QS = D / 16;
    static constexpr int VE = D % 64 == 0 ? 4 : 2;         // dims of a lane's V read
    f32x4 q[NB][QS];
    f32x4 o[NB][OB];

    __device__ __forceinline__ void load_q(int nb, const char* row) {
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            q[nb][s] = f32x4{0, 0, 0, 0};
            if (row) q[nb][s] = *(const f32x4*)(row + (4 * s + ((threadIdx.x & 63) >> 4)) * 16);
        }
    }
    __device__ __forceinline__ static uint32_t k_base(uint32_t tile) {
        uint32_t x = tile + G::row_at(threadIdx.x & 15, (threadIdx.x & 63) >> 4);
        asm volatile("" : "+v"(x));
        return x;
    }
    __device__ __forceinline__ static uint32_t v_base(uint32_t tile) {     // (the rows of a V read are no constants)
        uint32_t x = tile;
        asm volatile("" : "+v"(x));
        return x;
    }
    template <int Q>
    __device__ __forceinline__ void scores(uint32_t k, f32x4 (&s)[NB][Q]) const {
#pragma unroll
        for (int st = 0; st < QS; ++st)
#pragma unroll
            for (int x = 0; x < Q; ++x) {
                const f32x4 a = *(const __attribute__((address_space(3))) f32x4*)G::at(k, 4 * st, 16 * x);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        s[nb][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], q[nb][st][e], st + e ? s[nb][x] : f32x4{0, 0, 0, 0}, 0, 0, 0);
            }
    }
    struct Weights {
        f32x4 w[NB];
    };
    template <int Q>
    __device__ __forceinline__ static void pack(const f32x4 (&p)[NB][Q], int at, Weights& x) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) x.w[nb] = p[nb][at];
    }
    __device__ __forceinline__ void add_values(uint32_t v, int key, const Weights& p) {
        const int m = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
#pragma unroll
        for (int b = 0; b < OB / VE; ++b) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 4 * g + i;
                const uint32_t at = v + (key + row) * G::ROWB;
                float a[VE];
                if constexpr (VE == 4) {
                    const f32x4 x = *(const __attribute__((address_space(3))) f32x4*)(const lds_char*)(size_t)(at + ((16 * b + m) ^ G::twist(row)) * 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[e] = x[e];
                } else {
                    const f32x2 x = *(const __attribute__((address_space(3))) f32x2*)(const lds_char*)(size_t)(at + ((8 * b + (m >> 1)) ^ G::twist(row)) * 16 + (m & 1) * 8);
                    a[0] = x[0];
                    a[1] = x[1];
                }
#pragma unroll
                for (int e = 0; e < VE; ++e)
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
                        o[nb][b * VE + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], p.w[nb][i], o[nb][b * VE + e], 0, 0, 0);
            }
        }
    }
    template <int SUB>
    __device__ __forceinline__ static void schedule_products() {}
    __device__ __forceinline__ static void schedule_values() {}
    // o[nb][b * VE + e][i] is dim 16 VE b + VE (4 g + i) + e: four neighbours are e = 0 .. 3 of one i, or
    // e = 0, 1 of two
    __device__ __forceinline__ static int quad_dim(int y) {
        const int b = y / VE, x = y % VE, g = (threadIdx.x & 63) >> 4;
        return VE == 4 ? 64 * b + 4 * (4 * g + x) : 32 * b + 2 * (4 * g + 2 * x);
    }
    __device__ __forceinline__ f32x4 quad(int nb, int y) const {
        const int b = y / VE, x = y % VE;
        if constexpr (VE == 4) return f32x4{o[nb][4 * b][x], o[nb][4 * b + 1][x], o[nb][4 * b + 2][x], o[nb][4 * b + 3][x]};
        else return f32x4{o[nb][2 * b][2 * x], o[nb][2 * b + 1][2 * x], o[nb][2 * b][2 * x + 1], o[nb][2 * b + 1][2 * x + 1]};
    }
    __device__ __forceinline__ void add_quad(int nb, int y, f32x4 v) {
        const int b = y / VE, x = y % VE;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (VE == 4) o[nb][4 * b + e][x] += v[e];
            else o[nb][2 * b + (e & 1)][2 * x + (e >> 1)] += v[e];
        }
    }
};

// The running softmax of a wavefront's columns: m the maximum of c S so far, l this lane's share of the sum.
// m may lag behind the maximum by up to kSlack: weights up to 2^kSlack instead of 1 -- fp32 numbers, and two terms that
// keep 15 bits of them, whatever their size -- spare the rescaling that some of 32 rows would ask for with nearly every
// tile (2 x 4096 rows 494 -> 468 us, 4 trees of 64 nodes 237 -> 225, 8 trees of 8 46.9 -> 44.2).
constexpr float kSlack = 8.f;
template <typename E, int D, int NB>
struct Softmax {
    typedef Core<E, D, NB> C;
    float m[NB], l[NB];
    __device__ __forceinline__ void start(C& core) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb] = -INFINITY;
            l[nb] = 0.f;
#pragma unroll
            for (int b = 0; b < C::OB; ++b) core.o[nb][b] = f32x4{0, 0, 0, 0};
        }
    }
    // scores -> weights, everything before them rescaled to the new maximum
    template <int Q>
    __device__ __forceinline__ void step(C& core, f32x4 (&s)[NB][Q], float c) {
        float top[NB];
        bool more = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            float x = s[nb][0][0];
#pragma unroll
            for (int e = 1; e < 4 * Q; ++e) x = fmaxf(x, s[nb][e >> 2][e & 3]);
            top[nb] = fmaxf(m[nb], column_max(x) * c);
            more |= top[nb] > m[nb] + kSlack;
        }
        if (__any(more)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const float old = top[nb] > m[nb] ? fast_exp2(m[nb] - top[nb]) : 1.f;
                m[nb] = top[nb];
                l[nb] *= old;
#pragma unroll
                for (int b = 0; b < C::OB; ++b) core.o[nb][b] *= old;
            }
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const float base = m[nb] == -INFINITY ? 0.f : m[nb];
#pragma unroll
            for (int e = 0; e < 4 * Q; ++e) {
                const float w = fast_exp2(fmaf(s[nb][e >> 2][e & 3], c, -base));
                s[nb][e >> 2][e & 3] = w;
                l[nb] += w;
            }
        }
    }
};

// Scores of a tile from position j0 on that some row does not see all of: what a row does not see counts for
// nothing.
template <int NB, int Q>
__device__ __forceinline__ void apply_sees(f32x4 (&s)[NB][Q], const RowSees (&row)[NB], int j0, int sinks, int len) {
    const int g4 = 4 * ((threadIdx.x & 63) >> 4);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const uint64_t bits = sees(row[nb], j0, sinks, len) >> g4;
#pragma unroll
        for (int x = 0; x < 4 * Q; ++x)
            s[nb][x >> 2][x & 3] = (bits >> (16 * (x >> 2) + (x & 3))) & 1 ? s[nb][x >> 2][x & 3] : -INFINITY;
    }
}
// What take_out took out of tiles, to the sums of the rows that see it, when these are done: a weight is above zero, so
// what is not finite comes through as it is.  Values come from the cache again, KEYS of them from position j0_of(i) on, i < n
// (none where that is negative).
template <typename E, int D, int NB, int KEYS, typename F>
__device__ __forceinline__ void put_back(const AttnParams& p, Core<E, D, NB>& core, const RowSees (&row)[NB], const char* vbase, int seq,
                                         int len, int end, int n, F j0_of) {
    for (int i = 0; i < n; ++i) {
        const int j0 = j0_of(i);
        for (int m = 0; j0 >= 0 && m < KEYS && j0 + m < end; ++m) {
            const int pos = j0 + m, named = p.c.table[(size_t)seq * p.c.max_pages + (pos >> p.c.page_shift)];
            const int page = (unsigned)named < (unsigned)p.c.n_pages ? named : 0;
            const char* from = vbase + (page * p.c.page_stride + (pos & ((1 << p.c.page_shift) - 1)) * p.c.slot_stride) * 16;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const bool seen = (sees(row[nb], pos, p.sinks, len) & 1) != 0;
#pragma unroll
                for (int y = 0; y < Core<E, D, NB>::OB; ++y) {
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int dim = Core<E, D, NB>::quad_dim(y) + e;
                        if constexpr (sizeof(E) == 4) v[e] = ((const float*)from)[dim];
                        else v[e] = __uint_as_float((uint32_t)((const uint16_t*)from)[dim] << 16);
                        v[e] = seen && (__float_as_uint(v[e]) & 0x7f800000u) == 0x7f800000u ? v[e] : 0.f;
                    }
                    core.add_quad(nb, y, v);
                }
            }
        }
    }
}

template <typename E>
__device__ __forceinline__ void store_quad(char* row, int dim, f32x4 x) {
    if constexpr (sizeof(E) == 4) {
        *(f32x4*)(row + dim * 4) = x;
    } else {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)x[e];
        *(bf16x4*)(row + dim * 2) = y;
    }
}

// ---- shares of one block of rows -------------------------------------------------------------------
// They travel through agent-scope accesses, which the L2s of all dies agree on.
__device__ __forceinline__ void share_put(float* to, f32x4 x) {
    const uint64_t a = ((uint64_t)__float_as_uint(x[1]) << 32) | __float_as_uint(x[0]);
    const uint64_t b = ((uint64_t)__float_as_uint(x[3]) << 32) | __float_as_uint(x[2]);
    __hip_atomic_store((uint64_t*)to, a, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store((uint64_t*)to + 1, b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 share_pair(const float* from) {
    const uint64_t a = __hip_atomic_load((const uint64_t*)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)(a >> 32)));
}
// What a sum with maximum m weighs when joined under the maximum `top` (no key at all: m is -inf, l 0)
__device__ __forceinline__ float join_weight(float m, float top) { return m == -INFINITY ? 0.f : fast_exp2(m - top); }

// The shares of rows [from, to) of a block: a quad of a row by one thread.  AGENT: written in this launch.
template <bool AGENT>
__device__ __forceinline__ float2 share_get(const float* from) {
    if constexpr (AGENT) return share_pair(from);
    else return *(const float2*)from;
}
template <typename E, int D, int ROWS, int THREADS, bool AGENT>
__device__ __forceinline__ void join_shares(const AttnParams& p, int first, int shares, int first_row, int head, int r0, int from, int to) {
    constexpr int QUADS = D / 4, FLIGHT = 8;
    const size_t base = (size_t)first * ROWS;
    for (int i = threadIdx.x; i < (to - from) * QUADS; i += THREADS) {
        const int r = from + i / QUADS, quad = i % QUADS;
        // running maximum over the shares, FLIGHT of them on their way at a time
        float top = -INFINITY, l = 0.f;
        f32x4 o = {0, 0, 0, 0};
        for (int s0 = 0; s0 < shares; s0 += FLIGHT) {
            float2 ml[FLIGHT], a[FLIGHT], b[FLIGHT];
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f) {
                ml[f] = make_float2(-INFINITY, 0.f);
                a[f] = b[f] = make_float2(0.f, 0.f);
                if (s0 + f < shares) {
                    const size_t at = base + (size_t)(s0 + f) * ROWS + r;
                    ml[f] = share_get<AGENT>((const float*)(p.part_ml + at));
                    a[f] = share_get<AGENT>(p.part_o + at * D + quad * 4);
                    b[f] = share_get<AGENT>(p.part_o + at * D + quad * 4 + 2);
                }
            }
            float next = top;
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f) next = fmaxf(next, ml[f].x);
            const float old = join_weight(top, next);
            l *= old;
            o *= old;
            top = next;
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f) {
                if (ml[f].y == 0.f) continue;             // (nothing seen: its sums may be anything)
                const float w = join_weight(ml[f].x, top);
                l += ml[f].x == -INFINITY ? ml[f].y : ml[f].y * w;
                o += f32x4{a[f].x, a[f].y, b[f].x, b[f].y} * w;
            }
        }
        const int t = (r0 + r) / p.group, h = head * p.group + (r0 + r) % p.group;
        const f32x4 zero = {0, 0, 0, 0};
        store_quad<E>(p.out + (int64_t)(first_row + t) * p.out_stride + (int64_t)h * (D * (int)sizeof(E)), quad * 4, l == 0.f ? zero : o * (1.f / l));
    }
}

}  // namespace attn
}  // namespace dip

#endif  // DIP_ATTN_DEVICE_H_
