// Attention over chosen blocks of a long context: bounds of the blocks' keys (dip_kv_block_bounds), the choice
// (dip_select_blocks), and the attention itself (dip_block_attention).
//
// A block's smallest and largest key, channel by channel, bound q . k for all its keys: sum_d max(q_d lo_d, q_d hi_d).  With
// q+ = max(q, 0), q- = max(-q, 0) this is q+ . hi - q- . lo.  Which blocks are read must not hang on the order in which a sum
// is taken: the choice is that of the sums in fp64, where another order moves them by 1e-16 and not by a block's rank.

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>

#include "dip_attn_device.h"
#include "dip_vocab_device.h"

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
// A thread takes 16 bytes of a head's channels through a block's slots, kFlight of them on their way at a time.  Bound by bytes: 98304
// positions of 10 heads of 128 dims, bf16, two layers, 535 MB read and written in 80 us, which a plain read takes too.
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

// ---- scores: grid (parts, key/value heads, entries) --------------------------------------------------------------
// In fp32 on the matrix cores: [blocks x 2 D] times [2 D x columns], the bounds hi and lo times q+ and -q- of 16 columns (rows of the
// entry times the heads of the group).  A lane loads 16 bytes of a block's bounds, 16 blocks and 64 bytes of each at a time, straight
// into the product's operands, and they serve all columns: the call waits for memory (16 tokens over up to 64k positions, blocks of
// 32: 92 MB).  In fp64 without the matrix cores it took 44 us, and 24 for trees.
// The same sums with |hi| + |lo| and |q|, T, bound what rounding does to a score: half of its products are zero, the others are D
// roundings of 2^-23 T at most, in whatever order they are added up.  The choice settles in fp64 what lies nearer to its border than that.
// 28 us at 3.3 TB/s (25 where the last-level cache has them); a workgroup per 64 blocks, which has to look up entry, length, pages and queries for 32 KB of bounds, took 36.
struct ChoiceParams {
    KvView c;
    BatchView b;
    const char* q;
    int64_t q_stride;         // bytes
    const char* bounds;       // at the layer
    float* scores;            // [row][head][most]
    float4* stats;            // [entry][head][part]: least and most score, error bound (inf: none known)
    int32_t* out;             // [row][head][n_select]
    int most;                 // blocks of a sequence that there may be, a multiple of 4
    int parts;                // workgroups that share an entry's blocks of a head
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
// a block's bounds of a head
__device__ __forceinline__ const char* bounds_of(const ChoiceParams& p, const int32_t* table, int head, int b) {
    const int per_shift = p.c.page_shift - p.block_shift;
    const int named = table[b >> per_shift], page = is_page(p.c, named) ? named : 0;
    const int64_t at = (((int64_t)page * p.c.n_heads + head) << per_shift) + (b & ((1 << per_shift) - 1));
    return p.bounds + at * 2 * p.c.pieces * 16;
}

constexpr int kChunk = kThreads / 64 * 16;               // blocks at a time, 16 of a wavefront
// one 16-byte piece of 16 blocks times the same of 16 columns
template <typename E>
__device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (sizeof(E) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(attn::bf16x8, a), __builtin_bit_cast(attn::bf16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
        return c;
    }
}
// numbers above 0, below 0, and without their signs
template <typename E>
__device__ __forceinline__ void split(u32x4 x, u32x4& up, u32x4& down, u32x4& size) {
    constexpr uint32_t SIGN = sizeof(E) == 2 ? 0x80008000u : 0x80000000u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t below = sizeof(E) == 2 ? ((x[i] >> 15) & 0x00010001u) * 0xffffu : (uint32_t)((int32_t)x[i] >> 31);
        up[i] = x[i] & ~below;
        down[i] = x[i] & below;
        size[i] = x[i] & ~SIGN;
    }
}
template <typename E>
__device__ __forceinline__ u32x4 sizes(u32x4 x) {
    u32x4 up, down, size;
    split<E>(x, up, down, size);
    return size;
}
template <typename E>
__device__ __forceinline__ float largest(u32x4 size) {
    uint32_t m = 0;                                       // (numbers without signs are in order of their bits)
#pragma unroll
    for (int i = 0; i < 4; ++i) m = sizeof(E) == 2 ? max(m, max(size[i] & 0xffff0000u, size[i] << 16)) : max(m, size[i]);
    return __uint_as_float(m);
}

template <typename E, int D>
__global__ void __launch_bounds__(kThreads, sizeof(E) == 2 ? 4 : 3) block_scores_kernel(const ChoiceParams p) {
    constexpr int ES = sizeof(E), STEPS = D * ES / 64, PIECES = D * ES / 16, WAVES = kThreads / 64;
    __shared__ float s_tile[WAVES][16][20];               // [column][block]
    __shared__ float s_stat[3][WAVES];
    const int e = blockIdx.z, head = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const EntryRows er = entry_rows(p.b, e);
    const int seq = entry_seq(p.b, p.c, e);
    if (seq < 0 || er.rows == 0) return;
    const Middle m = middle_of(p, entry_len(p.c, seq));
    if ((int)blockIdx.x * kChunk >= m.n || m.n <= p.n_select) return;     // (all of them are chosen)
    const int32_t* table = p.c.table + (size_t)seq * p.c.max_pages;
    const int n = lane & 15, g = lane >> 4;
    float least = INFINITY, most = -INFINITY, error = 0.f;
    const int side = p.group < 16 ? 16 / p.group : 1;     // rows side by side in the columns
    const auto block_at = [&](int c) { return m.first + min(c * kChunk + wave * 16 + n, m.n - 1); };
    u32x4 lo[STEPS], hi[STEPS], x[STEPS];
    const auto load = [&](const char* at) {
        const u32x4* from = (const u32x4*)at + g;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) lo[s] = from[4 * s];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) hi[s] = from[PIECES + 4 * s];
    };
    // the queries of column n: row t0 + r, head h of the group
    const auto load_q = [&](int t0, int h0) {
        const int r = p.group < 16 ? n / p.group : 0, h = p.group < 16 ? n - r * p.group : h0 + n;
        const bool has = r < side && t0 + r < er.rows && h < p.group;
        const u32x4* q = (const u32x4*)(p.q + (int64_t)(er.first + t0 + (has ? r : 0)) * p.q_stride + (int64_t)(head * p.group + (has ? h : 0)) * (D * ES)) + g;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            x[s] = q[4 * s];
            if (!has) x[s] = u32x4{0, 0, 0, 0};
        }
    };
    const bool once = er.rows <= side && p.group <= 16;   // one set of columns: it stays in registers
    load(bounds_of(p, table, head, block_at(blockIdx.x)));
    if (once) load_q(0, 0);
    const char* next = bounds_of(p, table, head, block_at(blockIdx.x + gridDim.x));
    for (int c = blockIdx.x; c * kChunk < m.n; c += gridDim.x) {
        const int b0 = c * kChunk + wave * 16;
        for (int t0 = 0; t0 < er.rows; t0 += side) {
            float best[4];                                // of (row, block) lane + 64 i of side x 16
#pragma unroll
            for (int i = 0; i < 4; ++i) best[i] = -INFINITY;
            for (int h0 = 0; h0 < p.group; h0 += 16) {
                if (!once) load_q(t0, h0);
                f32x4 sum = {0, 0, 0, 0}, bound = {0, 0, 0, 0};
                float q_most = 0.f;
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    u32x4 up, down, size;
                    split<E>(x[s], up, down, size);
                    q_most = fmaxf(q_most, largest<E>(size));
                    sum = product<E>(hi[s], up, sum);
                    bound = product<E>(sizes<E>(hi[s]), size, bound);
                    sum = product<E>(lo[s], down, sum);
                    bound = product<E>(sizes<E>(lo[s]), size, bound);
                }
                // (should products flush what is below the normal numbers, each of them is off by the query times 2^-126)
                error = fmaxf(error, q_most <= FLT_MAX ? q_most * 0x1p-117f : INFINITY);
                float tall = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) tall = tall <= FLT_MAX && bound[i] <= FLT_MAX ? fmaxf(tall, bound[i]) : INFINITY;
                error = fmaxf(error, tall * ((D + 8) * 0x1p-23f));
                if (t0 + side >= er.rows && h0 + 16 >= p.group && (c + (int)gridDim.x) * kChunk < m.n) {
                    load(next);                           // (the chunk's last product is done with them)
                    next = bounds_of(p, table, head, block_at(c + 2 * (int)gridDim.x));
                }
                *(f32x4*)&s_tile[wave][n][4 * g] = sum;
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                const int heads = min(16, p.group - h0);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int y = lane + 64 * i, row = y >> 4;
                    if (row >= side) continue;
                    for (int k = 0; k < heads; ++k) best[i] = fmaxf(best[i], s_tile[wave][row * p.group + k][y & 15]);
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int y = lane + 64 * i, row = t0 + (y >> 4), b = b0 + (y & 15);
                if ((y >> 4) >= side || row >= er.rows || b >= m.n) continue;
                p.scores[((size_t)(er.first + row) * p.c.n_heads + head) * p.most + b] = best[i];
                least = fminf(least, best[i]);
                most = fmaxf(most, best[i]);
            }
        }
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) {
        least = fminf(least, __shfl_xor(least, off));
        most = fmaxf(most, __shfl_xor(most, off));
        error = fmaxf(error, __shfl_xor(error, off));
    }
    if (lane == 0) {
        s_stat[0][wave] = least;
        s_stat[1][wave] = most;
        s_stat[2][wave] = error;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < WAVES; ++w) {
            least = fminf(least, s_stat[0][w]);
            most = fmaxf(most, s_stat[1][w]);
            error = fmaxf(error, s_stat[2][w]);
        }
        p.stats[((size_t)e * p.c.n_heads + head) * p.parts + blockIdx.x] = make_float4(least, most, error, 0.f);
    }
}

// ---- the choice: grid (rows of an entry, key/value heads, entries) ------------------------------------------------------------
// One histogram of the fp32 scores finds the range that the border lies in.  What lies above it by more than three times the
// error is chosen, what lies below it by as much is not, and the few between are scored again in fp64 (unless all of them
// are wanted) and ranked, equal ones by number.  Where that leaves more than kNear, or no error bound is known (queries that are
// not finite, scores beyond fp32), all are scored in fp64 and selected by the digits of their keys.  Ranges and error are those of all
// rows of the entry and head together, so a few scores far from the others widen them: 16 tokens over up to 64k positions take 36 us for
// scores and choice, 67 with one block of each sequence three times as large as the others and 475 with one ten times, and three
// trees of seven nodes 23, or 460 where one node's queries are a hundred times the others'.
// Bound by latency, a chain of loads, barriers and LDS: 16 tokens of 10 heads, up to 2030 blocks, 11.6 us, two tokens 8.3 (256 threads
// 17.4 and 10.6, 1024 threads 13.3 and 9.1, and 17.2 instead of 11.4 for three trees of 32 heads).
constexpr int kChoiceThreads = 512;
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ int block_before(int x, int* waves, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, upto = running(x);
    __syncthreads();
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    int before = upto - x, all = 0;
#pragma unroll
    for (int w = 0; w < kChoiceThreads / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    *total = all;
    return before;
}
// A block's score in fp64, rounded once, by a wavefront.
template <typename E>
__device__ __forceinline__ float exact_score(const ChoiceParams& p, const int32_t* table, const char* q, int head, int b) {
    const int lane = threadIdx.x & 63, dims = p.c.pieces * (16 / (int)sizeof(E));      // (at most 128)
    const char* at = bounds_of(p, table, head, b);
    const auto number = [](const char* from, int i) {
        if constexpr (sizeof(E) == 4) return ((const float*)from)[i];
        else return __uint_as_float((uint32_t)((const uint16_t*)from)[i] << 16);
    };
    float lo[2], hi[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int d = min(lane + 64 * i, dims - 1);
        lo[i] = number(at, d);
        hi[i] = number(at, dims + d);
    }
    constexpr int HEADS = 4;
    double best = -(double)INFINITY;
    for (int h0 = 0; h0 < p.group; h0 += HEADS) {
        float x[HEADS][2];
#pragma unroll
        for (int h = 0; h < HEADS; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) x[h][i] = lane + 64 * i < dims ? number(q, min(h0 + h, p.group - 1) * dims + lane + 64 * i) : 0.f;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < 2; ++i) s += lane + 64 * i < dims ? (double)x[h][i] * (double)(x[h][i] > 0.f ? hi[i] : lo[i]) : 0.0;
            s = wave_sum(s);
            best = s > best ? s : best;                   // (a sum that is NaN is none)
        }
    }
    return (float)best;
}

constexpr int kDigits = 1024;
constexpr int kItems = 4;                 // neighbouring scores of a thread
constexpr int kNear = 128;
// kItems scores from i0 on, of n (a row of scores is whole 16 bytes)
__device__ __forceinline__ void load_scores(const float* scores, int i0, int n, float (&x)[kItems]) {
#pragma unroll
    for (int i = 0; i < kItems; i += 4) {
        const f32x4 y = i0 + i < n ? *(const f32x4*)(scores + i0 + i) : f32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) x[i + k] = y[k];
    }
}
struct ChoiceShared {
    int hist[kDigits];
    int waves[kChoiceThreads / 64];
    float stat[3][kChoiceThreads / 64];
    int digit, before;
    int n_near, n_sure;
    int near[kNear];
    float near_score[kNear];
    int near_taken[kNear];
};
// the first place in hist, from `n` of them, at which their running sum comes to `need`: s.digit, and the sum in front of it s.before
__device__ __forceinline__ void first_to(ChoiceShared& s, int n, int need) {
    const int per = n >= kChoiceThreads ? n / kChoiceThreads : (int)threadIdx.x < n, tid = threadIdx.x;
    int mine = 0, total, each[kDigits / kChoiceThreads];
#pragma unroll
    for (int i = 0; i < kDigits / kChoiceThreads; ++i) mine += each[i] = i < per ? s.hist[tid * per + i] : 0;
    int before = block_before(mine, s.waves, &total);
    if (before < need && before + mine >= need)
#pragma unroll
        for (int i = 0; i < kDigits / kChoiceThreads; ++i) {
            const int x = each[i];
            if (before < need && before + x >= need) {
                s.digit = tid * per + i;
                s.before = before;
            }
            before += x;
        }
    __syncthreads();
}
template <typename E>
__global__ void __launch_bounds__(kChoiceThreads) block_choice_kernel(const ChoiceParams p) {
    __shared__ ChoiceShared s;
    const int e = blockIdx.z, head = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
    const EntryRows er = entry_rows(p.b, e);
    if ((int)blockIdx.x >= er.rows) return;
    const size_t row = (size_t)(er.first + blockIdx.x) * p.c.n_heads + head;
    int32_t* out = p.out + row * p.n_select;
    const int seq = entry_seq(p.b, p.c, e);
    const Middle m = seq >= 0 ? middle_of(p, entry_len(p.c, seq)) : Middle{0, 0};
    if (m.n <= p.n_select) {
        for (int i = tid; i < p.n_select; i += kChoiceThreads) out[i] = i < m.n ? m.first + i : -1;
        return;
    }
    float* scores = p.scores + row * p.most;
    const int32_t* table = p.c.table + (size_t)seq * p.c.max_pages;
    const char* q = p.q + (int64_t)(er.first + blockIdx.x) * p.q_stride + (int64_t)head * p.group * p.c.pieces * 16;

    // up to kChoiceThreads * kItems scores stay in registers
    const bool one = m.n <= kChoiceThreads * kItems;
    float x[kItems];
    if (one) load_scores(scores, tid * kItems, m.n, x);
    float least = INFINITY, most = -INFINITY, error = 0.f;
    const float4* stats = p.stats + ((size_t)e * p.c.n_heads + head) * p.parts;
    for (int c = tid; c < p.parts && (int64_t)c * kChunk < m.n; c += kChoiceThreads) {
        const float4 y = stats[c];
        least = fminf(least, y.x);
        most = fmaxf(most, y.y);
        error = fmaxf(error, y.z);
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) {
        least = fminf(least, __shfl_xor(least, off));
        most = fmaxf(most, __shfl_xor(most, off));
        error = fmaxf(error, __shfl_xor(error, off));
    }
    if (lane == 0) {
        s.stat[0][tid >> 6] = least;
        s.stat[1][tid >> 6] = most;
        s.stat[2][tid >> 6] = error;
    }
    for (int i = tid; i < kDigits; i += kChoiceThreads) s.hist[i] = 0;
    if (tid == 0) s.n_near = s.n_sure = 0;
    __syncthreads();
    for (int w = 0; w < kChoiceThreads / 64; ++w) {
        least = fminf(least, s.stat[0][w]);
        most = fmaxf(most, s.stat[1][w]);
        error = fmaxf(error, s.stat[2][w]);
    }
    const float span = most - least;
    bool known = error <= FLT_MAX && span <= FLT_MAX && span >= 0.f;
    float above = 0.f, under = 0.f;                       // chosen: above `above`; not chosen: below `under`
    int need = 0;                                         // of those between
    if (known) {
        // ranges from the largest score down
        const float per = span > 0.f ? (kDigits - 1) / span : 0.f, width = span / (kDigits - 1);
        known = per <= FLT_MAX;
        for (int i0 = tid * kItems; i0 < m.n; i0 += kChoiceThreads * kItems) {
            if (!one) load_scores(scores, i0, m.n, x);
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (i0 + i < m.n) atomicAdd(&s.hist[min(kDigits - 1, (int)((most - x[i]) * per))], 1);
        }
        __syncthreads();
        first_to(s, kDigits, p.n_select);
        // (the range's limits, and what rounding leaves of them)
        const float slack = 3.f * error + span * 0x1p-18f;
        above = most - (float)s.digit * width + slack;
        under = most - (float)(s.digit + 1) * width - slack;
        int sure = 0;
        for (int i0 = tid * kItems; i0 < m.n; i0 += kChoiceThreads * kItems) {
            if (!one) load_scores(scores, i0, m.n, x);
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                if (i0 + i >= m.n) continue;
                sure += x[i] > above;
                if (x[i] > above || x[i] < under) continue;
                const int at = atomicAdd(&s.n_near, 1);
                if (at < kNear) s.near[at] = i0 + i;
            }
        }
#pragma unroll
        for (int off = 32; off; off >>= 1) sure += __shfl_xor(sure, off);
        if (lane == 0 && sure) atomicAdd(&s.n_sure, sure);
        __syncthreads();
        need = p.n_select - s.n_sure;
        if (s.n_near > kNear && s.n_near != need) known = false;
    }
    const int near = s.n_near;
    if (known && near != need) {
        for (int i = tid >> 6; i < near; i += kChoiceThreads / 64) {
            const float y = exact_score<E>(p, table, q, head, m.first + s.near[i]);
            if (lane == 0) s.near_score[i] = y;
        }
        __syncthreads();
        if (tid < near) {
            const uint32_t mine = key_of(s.near_score[tid]);
            int ahead = 0;
            for (int i = 0; i < near; ++i) {
                const uint32_t k = key_of(s.near_score[i]);
                ahead += k > mine || (k == mine && s.near[i] < s.near[tid]);
            }
            s.near_taken[tid] = ahead < need;
        }
        __syncthreads();
    }
    uint32_t prefix = 0;
    int left = p.n_select;
    if (!known) {
        // all of them in fp64, unless no product was anything but zero (queries of zeros: every score is, to the letter); the
        // key that the last chosen one has, and how many of those that have it
        for (int i = error == 0.f ? m.n : tid >> 6; i < m.n; i += kChoiceThreads / 64) {
            const float y = exact_score<E>(p, table, q, head, m.first + i);
            if (lane == 0) scores[i] = y;
        }
        for (int shift = 24; shift >= 0; shift -= 8) {
            constexpr int bits = 8, digits = 1 << bits;
            __syncthreads();
            for (int i = tid; i < digits; i += kChoiceThreads) s.hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < m.n; i += kChoiceThreads) {
                const uint32_t k = key_of(scores[i]);
                if ((uint64_t)(k ^ prefix) >> (shift + bits) == 0) atomicAdd(&s.hist[digits - 1 - (k >> shift & (digits - 1))], 1);
            }
            __syncthreads();
            first_to(s, digits, left);                    // from the largest digit down
            prefix |= (uint32_t)(digits - 1 - s.digit) << shift;
            left -= s.before;
        }
    }
    // the chosen ones, in order
    int given = 0, ties = 0;
    for (int i0 = 0; i0 < m.n; i0 += kChoiceThreads * kItems) {
        uint32_t take = 0, tie = 0;
        if (!one || !known) load_scores(scores, i0 + tid * kItems, m.n, x);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int at = i0 + tid * kItems + i;
            if (at >= m.n) continue;
            if (!known) {
                const uint32_t k = key_of(x[i]);
                take |= k > prefix ? 1u << i : 0u;
                tie |= k == prefix ? 1u << i : 0u;
            } else if (x[i] > above) {
                take |= 1u << i;
            } else if (x[i] >= under) {
                bool in = near == need;
                for (int y = 0; !in && y < near; ++y) in = s.near[y] == at && s.near_taken[y];
                take |= in ? 1u << i : 0u;
            }
        }
        int all, same;
        if (!known) {                                     // (uniform)
            int before = ties + block_before(__popc(tie), s.waves, &same);
            for (uint32_t rest = tie; rest; rest &= rest - 1)
                if (before++ < left) take |= rest & -rest;
            ties += same;
        }
        int to = given + block_before(__popc(take), s.waves, &all);
        for (uint32_t rest = take; rest; rest &= rest - 1) out[to++] = m.first + i0 + tid * kItems + __ffs((int)rest) - 1;
        given += all;
    }
}

// ---- attention ---------------------------------------------------------------------------------------------------------------
// A unit is a row, a key/value head, up to 16 query heads of its group and a share of what the row reads, which comes
// in cells of 16 positions: those in front, those of the chosen blocks, those behind.  A cell lies within a page, so that it
// has one address; a tile of a product is two cells (bf16) or one (fp32), wherever they lie.  Each wavefront streams tiles of
// its own through LDS, as in attn_rows_kernel.  Bound by reading what was chosen: 16 tokens of 40 heads on 10, bf16, 64 blocks of 32
// and 512 recent positions of up to 64k, 213 MB in 43 us (33 at the rate of a large read, 6.42 TB/s); three trees of up to 7 nodes, 32
// heads, 96 dims, fp32, 24 blocks of 32, 343 MB in 81 us (53); two tokens 10 us, latency.
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
    // the first entries of the row's list, on their way before it is known what is in range
    const int32_t* list = bp.blocks + ((size_t)row * p.c.n_heads + head) * bp.n_select;
    const int named0 = lane < bp.n_select ? list[lane] : -1, named1 = 64 + lane < bp.n_select ? list[64 + lane] : -1;
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
    // Entries of the list that are read: in range, and above the one before.  In a list of dip_select_blocks these are its first ones; where
    // a caller's has others between them (`gaps`), the n-th is looked for by number.  (A list is gone through whole: 0.3 us of 17.6 for
    // choice and attention by 128 entries, 5 of 113 by 4000.)
    const int from = parts.front >> bp.block_shift, upto = parts.tail >> bp.block_shift;
    const auto is_read = [&](int b, int before) { return b >= from && b < upto && b > before; };
    int chosen = 0, behind = 0, last = INT_MIN;           // (the entry before)
    const auto count = [&](int c, int x) {                // 64 entries (-1, behind the last one, is in no range)
        const int before = __builtin_amdgcn_update_dpp(last, x, 0x138, 0xf, 0xf, false);     // (of the lane before)
        const uint64_t read = __ballot(is_read(x, before));
        last = __builtin_amdgcn_readlane(x, 63);
        chosen += __popcll(read);
        if (read) behind = c + 64 - __clzll((long long)read);
    };
    count(0, named0);
    if (bp.n_select > 64) count(64, named1);
    constexpr int FLIGHT = 16;                            // on their way at a time
    for (int c = 128; c < bp.n_select; c += 64 * FLIGHT) {
        int named[FLIGHT];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) named[f] = list[min(c + 64 * f + lane, bp.n_select - 1)];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) count(c + 64 * f, c + 64 * f + lane < bp.n_select ? named[f] : -1);
    }
    const bool gaps = behind != chosen;
    const auto nth = [&](int n) {                         // (by all lanes)
        int at = 0, before = 0;
        for (int c = 0; c < bp.n_select; c += 64) {
            const int i = min(c + lane, bp.n_select - 1);
            uint64_t read = __ballot(c + lane == i && is_read(list[i], i ? list[i - 1] : INT_MIN));
            const int have = __popcll(read);
            if (n >= before && n < before + have) {
                for (int y = before; y < n; ++y) read &= read - 1;
                at = c + __ffsll((unsigned long long)read) - 1;
            }
            before += have;
        }
        return at;
    };
    const int front_cells = parts.front >> 4, chosen_cells = chosen << (bp.block_shift - 4);
    const int cells = alive ? front_cells + chosen_cells + (max(end - parts.tail, 0) + 15) / 16 : 0;
    const int tiles = (cells + CPT - 1) / CPT;
    // (a list that names blocks again and again may come to more tiles than the shares were made for)
    const int share_tiles = max(bp.share_tiles, (tiles + bp.shares - 1) / bp.shares);
    const int shares = max(1, (tiles + share_tiles - 1) / share_tiles);
    if (share >= shares) return;
    const int begin = share * share_tiles, stop = min(tiles, begin + share_tiles);
    const int mine = max(0, (stop - begin - wave + WAVES - 1) / WAVES);
    const int32_t* table = p.c.table + (size_t)max(seq, 0) * p.c.max_pages;

    auto fill = [&](int i0) {                             // the cells of the wavefront's tiles from i0 on
        const int i = lane / CPT, at = (begin + wave + WAVES * (i0 + i)) * CPT + lane % CPT;
        Cell c = {0, 0, 0};
        int n = (at - front_cells) >> (bp.block_shift - 4);
        if (gaps) n = nth(n);
        if (i0 + i < mine && at < cells) {
            int pos;
            uint32_t mask = 0xffff;
            if (at < front_cells) {
                pos = at << 4;
            } else if (at < front_cells + chosen_cells) {
                pos = (list[n] << bp.block_shift) + (((at - front_cells) & (per_block - 1)) << 4);
            } else {
                pos = parts.tail + ((at - front_cells - chosen_cells) << 4);
                mask = (uint32_t)sees(sees_own, pos, 0, len) & 0xffff;
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
int64_t most_blocks(const dip_kv_cache* c, const dip_batch* b, int32_t block) { return (reach(c, b) / block + 3) / 4 * 4; }

template <typename E>
hipError_t launch_choice(const ChoiceParams& p, int head_dim, int n_batch, hipStream_t stream) {
    const auto scores = [&](auto dim) {
        return launch_timed(block_scores_kernel<E, decltype(dim)::value>, dim3(p.parts, p.c.n_heads, n_batch), dim3(kThreads), stream, DIP_KERNEL_BLOCKS, p);
    };
    if (p.most > p.n_select) {
        const hipError_t err = head_dim == 64 ? scores(std::integral_constant<int, 64>()) : head_dim == 96 ? scores(std::integral_constant<int, 96>())
                                                                                                 : scores(std::integral_constant<int, 128>());
        if (err != hipSuccess) return err;
    }
    return launch_timed(block_choice_kernel<E>, dim3(p.b.max_rows, p.c.n_heads, n_batch), dim3(kChoiceThreads), stream, DIP_KERNEL_BLOCKS, p);
}
// Workgroups of block_scores_kernel that share an entry and head: about kScoreGrid in all
constexpr int kScoreGrid = 1280;
int parts_of(const dip_kv_cache* c, const dip_batch* b, int32_t block) {
    const int64_t chunks = (most_blocks(c, b, block) + kChunk - 1) / kChunk, fair = kScoreGrid / ((int64_t)c->n_kv_heads * b->n_batch);
    return (int)std::max<int64_t>(1, std::min(chunks, fair));
}
size_t score_bytes(const dip_kv_cache* c, const dip_batch* b, int32_t block) {
    return align_up((size_t)b->n_rows * c->n_kv_heads * most_blocks(c, b, block) * sizeof(float), 256);
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
    // one round of workgroups; a share has two tiles for each wavefront at least (two rounds: 49.7 instead of 43.9 us for 16
    // tokens over up to 64k positions, 95 instead of 80 for three trees in fp32)
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
    const size_t n = score_bytes(cache, batch, block) + (size_t)batch->n_batch * cache->n_kv_heads * parts_of(cache, batch, block) * sizeof(float4);
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
    if (rows_bound(batch) >= 1 << 23) return fail(DIP_ERR_UNSUPPORTED, "select_blocks: too many rows for one call");
    st = validate_ws(ws, ws_bytes, dip_select_blocks_workspace_bytes(cache, batch, n_q_heads, block));
    if (st) return st;
    ChoiceParams p;
    p.c = view_of(cache);
    p.b = view_of(batch);
    p.q = (const char*)q;
    p.q_stride = q_stride * elem_bytes(cache->dtype);
    p.bounds = (const char*)bounds + layer_bounds(cache, block) * layer;
    p.scores = (float*)ws;
    p.stats = (float4*)((char*)ws + score_bytes(cache, batch, block));
    p.out = blocks;
    p.parts = parts_of(cache, batch, block);
    p.most = (int)most_blocks(cache, batch, block);
    p.group = n_q_heads / cache->n_kv_heads;
    p.block_shift = log2_of(block);
    p.n_select = n_select;
    p.sinks = sinks;
    p.recent = recent;
    p.max_len = reach(cache, batch);
    return check_hip(cache->dtype == DIP_F32 ? launch_choice<float>(p, cache->head_dim, batch->n_batch, (hipStream_t)stream)
                                             : launch_choice<uint16_t>(p, cache->head_dim, batch->n_batch, (hipStream_t)stream),
                     "select_blocks launch");
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
