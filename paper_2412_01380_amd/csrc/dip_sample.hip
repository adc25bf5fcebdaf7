// From logits to tokens and probabilities (dip_sample).
//
// The kept words are the first ones in order of (logit, number), so every rule is a cut in one order: behind the top_k-th word,
// behind the word at which the weights pass top_p of their sum, in front of the first word below min_p.  A cut is a logit and
// a number among the words that have it.  It is found without sorting:
//   sample_scan_kernel   a workgroup per chunk of a row: its maximum, and a histogram of count and weight over bins an eighth
//                        of a nat wide, aligned to a grid that all chunks share (bin = floor(8 l / T)); the row's last
//                        workgroup adds the histograms up and says which bins the cut lies in -- or, where no rule
//                        applies, draws
//   sample_cut_kernel    the words in these bins (a few in a hundred) go into a list; the row's last workgroup narrows
//                        the cut down to a logit by histograms of 1024 key ranges over the list, and draws
//   sample_probs_kernel  the probabilities
// A weight is exp(-bin / 8) times a factor in (0.88, 1], which is held as an integer in units of 2^-30: sums over a bin are
// integer sums, the same in any order, and 2^-27 accurate relative to the weight itself however small it is.  8 l / T and its place
// in its bin are fp64 (2^-50 |l / T| more): of an fp32 quotient 2^-24 is lost, which at 30 nats is a weight off by 2 in 10^6.

#include <cmath>

#include "dip_vocab_device.h"

namespace dip {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = kThreads * kPer;
constexpr int kTiles = 2;                 // of a chunk, in registers
constexpr int kChunk = kTiles * kTile;
constexpr int kMaxChunks = (1 << 24) / kChunk;
constexpr int kBins = 512;                // the last one: all that lies 64 nats and more below the maximum
constexpr int kRest = kBins - 1;
constexpr int kList = 8192;               // words of a row's list; where more qualify the row itself is gone through again
constexpr int kRanges = 1024;             // key ranges of a step of narrowing down
constexpr uint32_t kOne = 1u << 30;       // weight 1 within a bin
constexpr int kCountShift = 44;           // a histogram word: count, weight
constexpr uint64_t kWeightMask = (1ull << kCountShift) - 1;
constexpr uint32_t kNothing = 0x007fffffu;    // key of -inf

enum : int { kEmpty = 0, kDone = 1, kCut = 2 };

// ---- words of a row ---------------------------------------------------------------------------------
// a larger number has a larger key; -0 is 0
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ ((int32_t)k < 0 ? 0x80000000u : 0xffffffffu)); }

__device__ __forceinline__ bool infinite(double x) { return x == (double)INFINITY; }
// 8 x / T (inv8 = 8 / T, 0 for an infinite temperature)
__device__ __forceinline__ double scaled(float x, double inv8) { return x == INFINITY ? (double)INFINITY : (double)x * inv8; }

// Where a word above -inf lies below `top`, the grid line of a maximum, and its weight within the bin.
struct Place {
    int bin;
    uint32_t weight;
};
__device__ __forceinline__ Place place_of(float x, double inv8, double top) {
    if (infinite(top)) return x == INFINITY ? Place{0, kOne} : Place{kRest, 0};
    const double z = scaled(x, inv8), line = floor(z), below = top - line;
    if (!(below < (double)kRest)) return {kRest, 0};
    // exp((part - 1) / 8) - 1, by its series: the first term left out is 1e-10
    const float t = ((float)(z - line) - 1.f) * 0.125f;
    float q = fmaf(t, 1.f / 720.f, 1.f / 120.f);
    q = fmaf(t, q, 1.f / 24.f);
    q = fmaf(t, q, 1.f / 6.f);
    q = fmaf(t, q, 0.5f);
    q = fmaf(t, q, 1.f);
    q *= t;
    return {(int)below, (uint32_t)((int)kOne + (int)rintf(q * (float)kOne))};
}
// what bins weigh: exp(-bin / 8) for weights in units of 2^-30, nothing behind the last
__device__ __forceinline__ void bin_scales(double* out) {
    for (int b = threadIdx.x; b < kBins; b += kThreads) out[b] = b == kRest ? 0.0 : exp(-0.125 * b) * 0x1p-30;
}

// ---- workspace -----------------------------------------------------------------------------------------
struct alignas(32) Chunk {
    double top;               // grid line of its maximum
    double weight;            // of its words, in units of exp((top + 1) / 8)
    uint64_t max_at;          // key of the maximum, ~number of the first word that has it
    uint64_t count;           // words above -inf
};
struct alignas(128) Row {
    double top;
    double inv8;
    double total;             // of the kept words, in units of exp((top + 1) / 8)
    double part;              // top_p's share
    uint32_t key;             // kept: a larger key, or this one and a number up to
    int32_t at;
    int32_t state;
    int32_t greedy;
    int32_t lo, hi;           // bins that the cut lies in
    int32_t k;                // words up to top_k's cut, 0: no such rule
    int32_t by_part;          // top_p cuts
    uint32_t min_key;         // min_p's cut, 0: no such rule
    int32_t listed;           // words in these bins: in the list, or too many for it
    uint32_t n;               // words in the list so far
    uint32_t least, most;     // their keys
    float best;               // the largest logit
};

struct SampleParams {
    const char* logits;
    int64_t stride;           // bytes
    int n_vocab, chunks;
    const float* temperature; // these four: nullable
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;           // nullable with token
    int32_t* token;           // nullable
    char* probs;              // nullable
    int64_t probs_stride;     // bytes
    Chunk* sums;              // [row][chunk]
    uint64_t* hist;           // [row][chunk][kBins]
    Row* rows;
    uint64_t* list;           // [row][kList]: key, number
    uint64_t* tickets;        // a word per row, kTicketStride apart; another of the second kernel behind them
    uint64_t epoch;
};

__device__ __forceinline__ void put64(void* to, uint64_t x) { __hip_atomic_store((uint64_t*)to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint64_t get64(const void* from) { return __hip_atomic_load((const uint64_t*)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ uint32_t get32(const uint32_t* from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

template <typename E>
__device__ __forceinline__ void load_logits(const char* row, int x, int end, float (&f)[kPer]) {
    load_entries<E>(row, x, end, f);
#pragma unroll
    for (int i = 0; i < kPer; ++i) f[i] = x + i < end && f[i] == f[i] ? f[i] : -INFINITY;
}

// exclusive sum over the workgroup, in order of the threads; *total: of all
template <typename T>
__device__ __forceinline__ T block_before(T x, T* waves, T* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T upto = x;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const T y = __shfl_up(upto, off);
        if (lane >= off) upto += y;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    T before = upto - x, all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    *total = all;
    return before;
}
__device__ __forceinline__ uint64_t block_max(uint64_t x, uint64_t* waves) {
#pragma unroll
    for (int off = 32; off; off >>= 1) {
        const uint64_t y = __shfl_xor((unsigned long long)x, off);
        x = y > x ? y : x;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) x = waves[w] > x ? waves[w] : x;
    return x;
}

struct Shared {
    double scale[kBins];
    double chunk[kMaxChunks];             // weights of the chunks' kept words
    union {
        struct {
            uint32_t count[kRanges];
            unsigned long long weight[kRanges];
        } range;
        struct {
            double weight[kBins];
            uint32_t count[kBins];
            int below[kMaxChunks];        // grid lines that a chunk's maximum lies below the row's
        } row;
        unsigned long long fixed[kMaxChunks];     // chunk weights of the listed words
    };
    double waves_d[kThreads / 64];
    uint64_t waves_u[kThreads / 64];
    uint32_t waves_i[kThreads / 64];
    double target;
    double total;
    uint64_t found;
    int at, last, flag;
    double got_weight;
    uint32_t got_count, got_key, got_here;
    double got_each;
};

// ---- the draw -----------------------------------------------------------------------------------------------
// s.chunk holds what each chunk's kept words weigh; kept: a key above `key`, or `key` and a number up to `at`.
// Returns the sum of all; the token is thread 0's to write.
template <typename E>
__device__ double draw(const SampleParams& p, int row, double top, double inv8, uint32_t key, int at, Shared& s) {
    const int tid = threadIdx.x;
    __syncthreads();
    // running sums over the chunks, contiguous ones to a thread
    const int per = (p.chunks + kThreads - 1) / kThreads;
    double mine = 0.0;
    for (int c = tid * per; c < min(p.chunks, (tid + 1) * per); ++c) mine += s.chunk[c];
    double total;
    const double before = block_before(mine, s.waves_d, &total);
    if (!p.token) return total;
    const double target = (double)p.u[row] * total;
    if (tid == 0) s.at = 0x7fffffff, s.last = -1, s.target = 0.0;
    __syncthreads();
    double run = before;
    int first = 0x7fffffff, some = -1;
    for (int c = tid * per; c < min(p.chunks, (tid + 1) * per); ++c) {
        run += s.chunk[c];
        if (s.chunk[c] > 0.0) {
            some = c;
            if (run > target) first = min(first, c);
        }
    }
    if (first != 0x7fffffff) atomicMin(&s.at, first);
    if (some >= 0) atomicMax(&s.last, some);
    __syncthreads();
    // (rounding may leave no chunk past the target: then the last one that holds anything)
    const int c = s.at != 0x7fffffff ? s.at : s.last;
    if (c < 0) {
        if (tid == 0) p.token[row] = -1;
        return total;
    }
    if (tid == c / per) {
        double sum = before;
        for (int i = tid * per; i < c; ++i) sum += s.chunk[i];
        s.target = target - sum;
    }
    __syncthreads();
    const double left = s.target;
    if (tid == 0) s.at = 0x7fffffff, s.last = -1;
    __syncthreads();
    const char* logits = p.logits + row * p.stride;
    double ahead = 0.0;
    for (int x0 = c * kChunk; x0 < min((c + 1) * kChunk, p.n_vocab); x0 += kTile) {
        const int x = x0 + tid * kPer;
        float f[kPer];
        load_logits<E>(logits, x, p.n_vocab, f);
        double w[kPer], sum = 0.0;
        int some_word = -1;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t k = key_of(f[i]);
            w[i] = 0.0;
            if (f[i] > -INFINITY && (k > key || (k == key && x + i <= at))) {
                const Place pl = place_of(f[i], inv8, top);
                w[i] = (double)pl.weight * s.scale[pl.bin];
                if (w[i] > 0.0) some_word = x + i;
            }
            sum += w[i];
        }
        double tile;
        double run_sum = ahead + block_before(sum, s.waves_d, &tile);
        int found = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            run_sum += w[i];
            if (w[i] > 0.0 && run_sum > left) found = min(found, x + i);
        }
        if (found != 0x7fffffff) atomicMin(&s.at, found);
        if (some_word >= 0) atomicMax(&s.last, some_word);
        ahead += tile;
        __syncthreads();
        if (s.at != 0x7fffffff) break;
    }
    if (tid == 0) p.token[row] = s.at != 0x7fffffff ? s.at : s.last;
    return total;
}

// ---- chunks, and what a row is to be cut at: grid (chunks, rows) ------------------------------------------------
template <typename E>
__global__ void __launch_bounds__(kThreads) sample_scan_kernel(const SampleParams p) {
    __shared__ Shared s;
    __shared__ unsigned long long s_hist[kBins];
    const int row = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x;
    const float T = p.temperature ? p.temperature[row] : 1.f;
    const bool greedy = !(T > 0.f);
    const double inv8 = greedy ? 0.0 : 8.0 / (double)T;
    const int k = p.top_k ? p.top_k[row] : 0;
    const float part = p.top_p ? p.top_p[row] : 1.f;
    float least = p.min_p ? p.min_p[row] : 0.f;
    least = isinf(T) || !(least > 0.f) ? 0.f : fminf(least, 1.f);
    const bool cuts = !greedy && ((k > 0 && k < p.n_vocab) || part < 1.f || least > 0.f);
    uint64_t* ticket = p.tickets + (size_t)row * kTicketStride;
    if (tid == 0) ticket_open(ticket, p.epoch);

    float f[kTiles][kPer];
    uint64_t best = 0;
    uint32_t n = 0;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int x = chunk * kChunk + t * kTile + tid * kPer;
        load_logits<E>(p.logits + row * p.stride, x, min(p.n_vocab, (chunk + 1) * kChunk), f[t]);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const bool is = f[t][i] > -INFINITY;
            n += is;
            const uint64_t at = is ? ((uint64_t)key_of(f[t][i]) << 32) | (uint32_t)~(x + i) : 0;
            best = at > best ? at : best;
        }
    }
    bin_scales(s.scale);
    for (int b = tid; b < kBins; b += kThreads) s_hist[b] = 0;
    best = block_max(best, s.waves_u);
    uint32_t count;
    block_before(n, s.waves_i, &count);
    const double top = best ? floor(scaled(of_key((uint32_t)(best >> 32)), inv8)) : -(double)INFINITY;
    double weight = 0.0;
    if (!greedy && best) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (f[t][i] > -INFINITY) {
                    const Place pl = place_of(f[t][i], inv8, top);
                    atomicAdd(&s_hist[pl.bin], (1ull << kCountShift) | pl.weight);
                }
        __syncthreads();
        for (int b = tid; b < kBins; b += kThreads) weight += (double)(s_hist[b] & kWeightMask) * s.scale[b];
        double all;
        block_before(weight, s.waves_d, &all);
        weight = all;
    }
    if (cuts) {
        uint64_t* out = p.hist + ((size_t)row * p.chunks + chunk) * kBins;
        for (int b = tid; b < kBins; b += kThreads) put64(out + b, s_hist[b]);
    }
    Chunk* sum = p.sums + (size_t)row * p.chunks + chunk;
    if (tid == 0) {
        put((double*)&sum->top, top);
        put((double*)&sum->weight, weight);
        put64(&sum->max_at, best);
        put64(&sum->count, count);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s.flag = ticket_last(ticket, p.epoch, p.chunks);
    __syncthreads();
    if (!s.flag) return;

    // ---- the row ----
    const Chunk* sums = p.sums + (size_t)row * p.chunks;
    uint64_t first = 0;
    uint32_t words = 0;
    for (int c = tid; c < p.chunks; c += kThreads) {
        const uint64_t at = get64(&sums[c].max_at);
        first = at > first ? at : first;
        words += (uint32_t)get64(&sums[c].count);
    }
    first = block_max(first, s.waves_u);
    uint32_t n_words;
    block_before(words, s.waves_i, &n_words);
    Row* r = p.rows + row;
    if (first == 0 || greedy) {
        if (tid == 0) {
            r->state = first ? kDone : kEmpty;
            r->greedy = 1;
            r->key = (uint32_t)(first >> 32);
            r->at = (int)~(uint32_t)first;
            r->total = 1.0;
            r->top = r->inv8 = 0.0;
            if (p.token) p.token[row] = first ? (int)~(uint32_t)first : -1;
        }
        return;
    }
    const float best_logit = of_key((uint32_t)(first >> 32));
    const double row_top = floor(scaled(best_logit, inv8));
    for (int c = tid; c < p.chunks; c += kThreads) {
        const double below = infinite(row_top) ? (infinite(get(&sums[c].top)) ? 0.0 : (double)kRest) : row_top - get(&sums[c].top);
        const int off = below < (double)kRest ? (int)below : kRest;
        s.row.below[c] = off;
        s.chunk[c] = off == kRest ? 0.0 : get(&sums[c].weight) * (s.scale[off] * 0x1p30);
    }
    if (tid == 0) {
        r->state = kDone;
        r->greedy = 0;
        r->best = best_logit;
        r->top = row_top;
        r->inv8 = inv8;
        r->key = kNothing;
        r->at = -1;
    }
    __syncthreads();
    if (!cuts) {
        const double total = draw<E>(p, row, row_top, inv8, kNothing, -1, s);
        if (tid == 0) r->total = total;
        return;
    }

    // counts and weights of the row's bins, and their running sums
    const uint64_t* hist = p.hist + (size_t)row * p.chunks * kBins;
    constexpr int PER = kBins / kThreads;
    uint32_t cnt[PER], cnt_sum = 0;
    double wgt[PER], wgt_sum = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = tid * PER + i;
        cnt[i] = 0;
        uint64_t w = 0;
        for (int c = 0; c < p.chunks && b < kRest; ++c) {
            const int lb = b - s.row.below[c];
            if (lb < 0) continue;
            const uint64_t h = get64(hist + (size_t)c * kBins + lb);
            cnt[i] += (uint32_t)(h >> kCountShift);
            w += h & kWeightMask;
        }
        wgt[i] = (double)w * s.scale[b];
        cnt_sum += cnt[i];
        wgt_sum += wgt[i];
    }
    uint32_t known;
    uint32_t cnt_before = block_before(cnt_sum, s.waves_i, &known);
    if (tid == kThreads - 1) cnt[PER - 1] = n_words - known;
    double total;
    double wgt_before = block_before(wgt_sum, s.waves_d, &total);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = tid * PER + i;
        s.row.count[b] = cnt_before += cnt[i];
        s.row.weight[b] = wgt_before += wgt[i];
    }
    __syncthreads();
    if (tid == 0) {
        // (in order, by one thread: a binary search each)
        auto bin_of = [&](auto past) {
            int lo = 0, hi = kRest;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (past(mid)) hi = mid;
                else lo = mid + 1;
            }
            return lo;
        };
        auto count_to = [&](int b) { return b < 0 ? 0u : s.row.count[b]; };
        auto weight_to = [&](int b) { return b < 0 ? 0.0 : s.row.weight[b]; };
        bool by_k = k > 0 && (uint32_t)k < n_words, by_part = part < 1.f;
        int lo = kBins, hi = -1, bin_k = kRest;
        if (by_k) lo = hi = bin_k = bin_of([&](int b) { return count_to(b) >= (uint32_t)k; });
        if (by_part) {
            const double share = part > 0.f ? (double)part : 0.0;
            const double from = share * (by_k ? weight_to(bin_k - 1) : total), to = share * (by_k ? weight_to(bin_k) : total);
            lo = min(bin_k, bin_of([&](int b) { return weight_to(b) >= from && count_to(b) > 0; }));
            hi = by_k ? bin_k : min(bin_k, bin_of([&](int b) { return weight_to(b) >= to && count_to(b) > 0; }));
        }
        uint32_t min_key = 0;
        if (least > 0.f) {
            const double c = least < 1.f ? (double)best_logit + (double)T * log((double)least) : (double)best_logit;
            float at = (float)c;
            if ((double)at < c) at = of_key(key_of(at) + 1);
            if (at > -INFINITY) {
                min_key = key_of(at);
                const double below = infinite(row_top) ? (at == INFINITY ? 0.0 : (double)kRest) : row_top - floor(scaled(at, inv8));
                const int b = below < (double)kRest ? (int)below : kRest;
                if (b < lo) {
                    lo = hi = b;
                    by_k = by_part = false;
                }
            }
        }
        if (lo > hi) {                        // nothing cuts this row after all
            s.flag = 0;
        } else {
            s.flag = 1;
            r->state = kCut;
            r->part = part > 0.f ? (double)part : 0.0;
            r->lo = lo;
            r->hi = hi;
            r->k = by_k ? k : 0;
            r->by_part = by_part;
            r->min_key = min_key;
            r->listed = (int)(count_to(hi) - count_to(lo - 1));
            r->total = total;
            r->n = 0;
            r->least = 0xffffffffu;
            r->most = 0;
        }
    }
    __syncthreads();
    if (!s.flag) {
        total = draw<E>(p, row, row_top, inv8, kNothing, -1, s);
        if (tid == 0) r->total = total;
    }
}

// ---- the cut: grid (chunks, rows) -------------------------------------------------------------------------------
// f(x, number) of every word that lies in the row's bins lo .. hi, by the threads of a workgroup
template <typename E, typename F>
__device__ __forceinline__ void each_word(const SampleParams& p, const Row& r, int row, bool listed, int n, F f) {
    if (listed) {
        const uint64_t* list = p.list + (size_t)row * kList;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const uint64_t e = get64(list + i);
            f(of_key((uint32_t)(e >> 32)), (int)(uint32_t)e);
        }
    } else {
        constexpr int FLIGHT = 8;
        const char* logits = p.logits + row * p.stride;
        for (int x0 = threadIdx.x; x0 < p.n_vocab; x0 += FLIGHT * kThreads) {
            float v[FLIGHT];
#pragma unroll
            for (int i = 0; i < FLIGHT; ++i) v[i] = entry_at<E>(logits, min(x0 + i * kThreads, p.n_vocab - 1));
#pragma unroll
            for (int i = 0; i < FLIGHT; ++i) {
                const int x = x0 + i * kThreads;
                if (x >= p.n_vocab || !(v[i] > -INFINITY)) continue;
                const int b = place_of(v[i], r.inv8, r.top).bin;
                if (b >= r.lo && b <= r.hi) f(v[i], x);
            }
        }
    }
}

// A listed word's weight as an integer, in units of exp((top - lo + 1) / 8) 2^-38: 2^24 of them fit 64 bits.
__device__ __forceinline__ uint64_t fixed_weight(const Row& r, const Shared& s, float x) {
    const Place pl = place_of(x, r.inv8, r.top);
    return pl.bin == kRest ? 0 : (uint64_t)((double)pl.weight * (s.scale[max(pl.bin - r.lo, 0)] * 0x1p38) + 0.5);
}

// The logit at which the listed words, in order, first come to `need` words or to `need` in weight: in s.got_key, the
// words and the weight in front of it in got_count and got_weight, how many have it in got_here, what one of them
// weighs in got_each.
template <typename E, bool WEIGHT>
__device__ void narrow(const SampleParams& p, const Row& r, int row, bool listed, int n, uint32_t least, uint32_t most, double need, Shared& s) {
    const int tid = threadIdx.x;
    constexpr int PER = kRanges / kThreads;
    uint32_t count = 0;
    double weight = 0.0;
    for (;;) {
        const uint32_t span = most - least;
        const int bits = span ? 32 - __clz((int)span) : 1, shift = max(0, bits - 10);
        __syncthreads();
        for (int i = tid; i < kRanges; i += kThreads) {
            s.range.count[i] = 0;
            s.range.weight[i] = 0;
        }
        if (tid == 0) s.at = kRanges, s.last = 0;
        __syncthreads();
        each_word<E>(p, r, row, listed, n, [&](float x, int) {
            const uint32_t k = key_of(x);
            if (k < least || k > most) return;
            const uint32_t at = (most - k) >> shift;
            atomicAdd(&s.range.count[at], 1u);
            atomicAdd(&s.range.weight[at], (unsigned long long)fixed_weight(r, s, x));
        });
        __syncthreads();
        uint32_t c_mine = 0, c_all;
        uint64_t w_mine = 0, w_all;
        for (int i = 0; i < PER; ++i) {
            c_mine += s.range.count[tid * PER + i];
            w_mine += s.range.weight[tid * PER + i];
        }
        uint32_t c_run = block_before(c_mine, s.waves_i, &c_all);
        uint64_t w_run = block_before(w_mine, s.waves_u, &w_all);
        const uint32_t c_before = c_run;
        const uint64_t w_before = w_run;
        int found = kRanges, some = 0;
        for (int i = 0; i < PER; ++i) {
            const int at = tid * PER + i;
            c_run += s.range.count[at];
            w_run += s.range.weight[at];
            if (!s.range.count[at]) continue;
            some = at;
            const double have = WEIGHT ? weight + (double)w_run : (double)(count + c_run);
            if (have >= need) found = min(found, at);
        }
        if (found < kRanges) atomicMin(&s.at, found);
        if (some) atomicMax(&s.last, some);
        __syncthreads();
        // (rounding may leave the last one short of the need)
        const int at = s.at < kRanges ? s.at : s.last;
        if (tid == at / PER) {
            uint32_t c = c_before;
            uint64_t w = w_before;
            for (int i = tid * PER; i < at; ++i) {
                c += s.range.count[i];
                w += s.range.weight[i];
            }
            s.got_count = count + c;
            s.got_weight = weight + (double)w;
            s.got_here = s.range.count[at];
            s.got_each = s.range.count[at] ? (double)s.range.weight[at] / (double)s.range.count[at] : 0.0;
        }
        __syncthreads();
        count = s.got_count;
        weight = s.got_weight;
        const uint32_t top = most - ((uint32_t)at << shift);
        if (shift == 0) {
            if (tid == 0) s.got_key = top;
            __syncthreads();
            return;
        }
        const uint32_t width = (1u << shift) - 1;
        least = top - least > width ? top - width : least;
        most = top;
    }
}

// The number of the m-th word (from 1) among the listed ones with a key, in order of their numbers.
template <typename E>
__device__ int nth(const SampleParams& p, const Row& r, int row, bool listed, int n, uint32_t key, uint32_t m, Shared& s) {
    const int tid = threadIdx.x;
    constexpr int PER = kRanges / kThreads;
    uint32_t lo = 0, skipped = 0;
    for (int shift = 14; shift >= 0; shift -= shift > 10 ? 10 : 4) {  // numbers of 24 bits: by 10, 10 and 4 of them
        __syncthreads();
        for (int i = tid; i < kRanges; i += kThreads) s.range.count[i] = 0;
        if (tid == 0) s.at = kRanges - 1;
        __syncthreads();
        each_word<E>(p, r, row, listed, n, [&](float x, int number) {
            const uint32_t at = ((uint32_t)number - lo) >> shift;
            if (key_of(x) == key && (uint32_t)number >= lo && at < kRanges) atomicAdd(&s.range.count[at], 1u);
        });
        __syncthreads();
        uint32_t mine = 0, all;
        for (int i = 0; i < PER; ++i) mine += s.range.count[tid * PER + i];
        const uint32_t before = block_before(mine, s.waves_i, &all);
        uint32_t run = skipped + before;
        int found = kRanges;
        for (int i = 0; i < PER; ++i) {
            run += s.range.count[tid * PER + i];
            if (run >= m) found = min(found, tid * PER + i);
        }
        if (found < kRanges) atomicMin(&s.at, found);
        __syncthreads();
        const int at = s.at;
        if (tid == at / PER) {
            uint32_t c = skipped + before;
            for (int i = tid * PER; i < at; ++i) c += s.range.count[i];
            s.got_count = c;
        }
        __syncthreads();
        skipped = s.got_count;
        lo += (uint32_t)at << shift;
        if (shift == 0) break;
    }
    return (int)lo;
}

template <typename E>
__global__ void __launch_bounds__(kThreads) sample_cut_kernel(const SampleParams p) {
    __shared__ Shared s;
    const int row = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x;
    Row* rp = p.rows + row;
    if (rp->state != kCut) return;
    const Row r = *rp;
    uint64_t* ticket = p.tickets + (size_t)(gridDim.y + row) * kTicketStride;
    if (tid == 0) ticket_open(ticket, p.epoch);
    const bool listed = r.listed <= kList;
    float f[kTiles][kPer];
    uint32_t hits = 0, mine = 0, least = 0xffffffffu, most = 0;      // (a bit of hits per word)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int x = chunk * kChunk + t * kTile + tid * kPer;
        load_logits<E>(p.logits + row * p.stride, x, min(p.n_vocab, (chunk + 1) * kChunk), f[t]);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (!(f[t][i] > -INFINITY)) continue;
            const int b = place_of(f[t][i], r.inv8, r.top).bin;
            if (b < r.lo || b > r.hi) continue;
            hits |= 1u << (t * kPer + i);
            ++mine;
            const uint32_t k = key_of(f[t][i]);
            least = min(least, k);
            most = max(most, k);
        }
    }
    static_assert(kTiles * kPer <= 32, "a bit per word");
    uint32_t all;
    const uint32_t before = block_before(mine, s.waves_i, &all);
    const uint32_t top_key = (uint32_t)block_max(most, s.waves_u), low_key = ~(uint32_t)block_max((uint32_t)~least, s.waves_u);
    if (tid == 0 && all) {
        s.got_count = atomicAdd(&rp->n, all);
        atomicMin(&rp->least, low_key);
        atomicMax(&rp->most, top_key);
    }
    __syncthreads();
    if (all && listed) {
        uint32_t at = s.got_count + before;
        uint64_t* list = p.list + (size_t)row * kList;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (hits >> (t * kPer + i) & 1) {
                    if (at < (uint32_t)kList) put64(list + at, ((uint64_t)key_of(f[t][i]) << 32) | (uint32_t)(chunk * kChunk + t * kTile + tid * kPer + i));
                    ++at;
                }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) s.flag = ticket_last(ticket, p.epoch, p.chunks);
    __syncthreads();
    if (!s.flag) return;

    // ---- the row ----
    const int n = (int)min(get32(&rp->n), (uint32_t)kList);
    const uint32_t all_least = get32(&rp->least), all_most = get32(&rp->most);
    bin_scales(s.scale);
    __syncthreads();
    // the chunks' words above the bins that the cut lies in
    const Chunk* sums = p.sums + (size_t)row * p.chunks;
    const uint64_t* hist = p.hist + (size_t)row * p.chunks * kBins;
    for (int c = tid; c < p.chunks; c += kThreads) s.chunk[c] = 0.0;
    __syncthreads();
    double above = 0.0;
    uint32_t above_n = 0;
    for (int c = tid >> 6; c < p.chunks; c += kThreads / 64) {        // a wavefront per chunk
        const double below = infinite(r.top) ? (infinite(sums[c].top) ? 0.0 : (double)kRest) : r.top - sums[c].top;
        double w = 0.0;
        if (below < (double)kRest)
            for (int b = (int)below + (tid & 63); b < r.lo; b += 64) {
                const uint64_t h = hist[(size_t)c * kBins + b - (int)below];
                w += (double)(h & kWeightMask) * s.scale[b];
                above_n += (uint32_t)(h >> kCountShift);
            }
        w = wave_sum(w);
        if ((tid & 63) == 0) {
            s.chunk[c] = w;
            above += w;
        }
    }
    double above_all;
    block_before(above, s.waves_d, &above_all);
    uint32_t above_count;
    block_before(above_n, s.waves_i, &above_count);
    // weights of listed words are counted in `unit`s
    const double unit = s.scale[min(r.lo, kRest - 1)] * 0x1p-8;       // (exp(-lo / 8) 2^-38)
    double total = r.total;
    uint32_t key = kNothing;
    int at = -1;
    if (r.k) {
        const uint32_t need = (uint32_t)r.k - above_count;
        narrow<E, false>(p, r, row, listed, n, all_least, all_most, (double)need, s);
        key = s.got_key;
        const uint32_t ties = need - s.got_count, here = s.got_here;
        total = above_all + (s.got_weight + (double)ties * s.got_each) * unit;
        at = ties < here && !r.by_part ? nth<E>(p, r, row, listed, n, key, ties, s) : 0x7fffffff;
        if (r.by_part) at = (int)ties;        // (so far a count: the other cut lies in front of this one)
    }
    if (r.by_part) {
        const double need = (r.part * total - above_all) / unit;
        const uint32_t key_k = key;
        const int ties_k = at;
        narrow<E, true>(p, r, row, listed, n, r.k ? key_k : all_least, all_most, need, s);
        key = s.got_key;
        const uint32_t here = r.k && key == key_k ? (uint32_t)ties_k : s.got_here;
        double more = s.got_each > 0.0 ? ceil((need - s.got_weight) / s.got_each) : 1.0;
        more = more < 1.0 ? 1.0 : more;
        const uint32_t ties = more < (double)here ? (uint32_t)more : here;
        at = ties < s.got_here ? nth<E>(p, r, row, listed, n, key, ties, s) : 0x7fffffff;
    }
    if (r.min_key > key) {
        key = r.min_key;
        at = 0x7fffffff;
    }
    // the kept ones among the listed
    __syncthreads();
    for (int c = tid; c < p.chunks; c += kThreads) s.fixed[c] = 0;
    __syncthreads();
    each_word<E>(p, r, row, listed, n, [&](float x, int number) {
        const uint32_t k = key_of(x);
        if (k > key || (k == key && number <= at)) atomicAdd(&s.fixed[number / kChunk], (unsigned long long)fixed_weight(r, s, x));
    });
    __syncthreads();
    for (int c = tid; c < p.chunks; c += kThreads) s.chunk[c] += (double)s.fixed[c] * unit;
    total = draw<E>(p, row, r.top, r.inv8, key, at, s);
    if (tid == 0) {
        rp->total = total;
        rp->key = key;
        rp->at = at;
        rp->state = kDone;
    }
}

// ---- probabilities: grid (chunks, rows) ----------------------------------------------------------------------------
template <typename E, typename O>
__global__ void __launch_bounds__(kThreads) sample_probs_kernel(const SampleParams p) {
    const int row = blockIdx.y;
    const Row* rp = p.rows + row;
    const int state = rp->state, at = rp->at;
    const bool greedy = rp->greedy;
    const uint32_t key = rp->key;
    // weights relative to the largest logit's: differences of logits are exact, of 8 l / T they are not where T is next to nothing
    const double top = rp->top, inv8 = rp->inv8, best = (double)rp->best, step = inv8 * (0.125 * 1.44269504088896340736);
    const float each = (float)(greedy || state == kEmpty ? 1.0 : (double)place_of(rp->best, inv8, top).weight * 0x1p-30 / rp->total);
    const int end = min(p.n_vocab, (int)(blockIdx.x + 1) * kChunk);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const int x = blockIdx.x * kChunk + t * kTile + threadIdx.x * kPer;
        if (x >= end) break;
        float f[kPer];
        load_logits<E>(p.logits + row * p.stride, x, end, f);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t k = key_of(f[i]);
            const bool kept = state != kEmpty && f[i] > -INFINITY && (k > key || (k == key && x + i <= at));
            float y = 0.f;
            if (kept) {
                if (greedy) y = 1.f;
                else if (infinite(top)) y = f[i] == INFINITY ? each : 0.f;
                else {                        // 2^(whole + part)
                    const double z = ((double)f[i] - best) * step, whole = floor(z);
                    y = whole < -400.0 ? 0.f : ldexpf(__builtin_amdgcn_exp2f((float)(z - whole)) * each, (int)whole);
                }
            }
            f[i] = y;
        }
        struct __attribute__((packed, aligned(sizeof(O)))) Any { O w[16 / sizeof(O)]; };
        O* out = (O*)(p.probs + row * p.probs_stride) + x;
        constexpr int N = 16 / sizeof(O);
        if (x + kPer <= end) {
#pragma unroll
            for (int y = 0; y < kPer / N; ++y) {
                Any a;
#pragma unroll
                for (int i = 0; i < N; ++i) a.w[i] = (O)f[y * N + i];
                *(Any*)(out + y * N) = a;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (x + i < end) out[i] = (O)f[i];
        }
    }
}

struct SamplePlan {
    int chunks;
    size_t off_hist, off_rows, off_list, off_tickets, total;
};
SamplePlan plan_sample(int n_rows, int n_vocab) {
    SamplePlan pl;
    pl.chunks = (n_vocab + kChunk - 1) / kChunk;
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    const size_t parts = (size_t)n_rows * pl.chunks;
    take(sizeof(Chunk) * parts);
    pl.off_hist = take(sizeof(uint64_t) * kBins * parts);
    pl.off_rows = take(sizeof(Row) * n_rows);
    pl.off_list = take(sizeof(uint64_t) * kList * n_rows);
    pl.off_tickets = take(sizeof(uint64_t) * kTicketStride * 2 * n_rows);
    pl.total = o;
    return pl;
}
int32_t check_sample(int n_rows, int n_vocab) {
    if (n_rows < 1 || n_vocab < 1) return fail(DIP_ERR_INVALID_ARG, "sample: sizes must be >= 1");
    if (n_rows > 65535) return fail(DIP_ERR_UNSUPPORTED, "sample: more than 65535 rows");
    if (n_vocab > 1 << 24) return fail(DIP_ERR_UNSUPPORTED, "sample: n_vocab must be at most 2^24");
    return DIP_OK;
}

template <typename E>
int32_t launch_sample(SampleParams& p, int n_rows, bool cuts, int probs_dtype, hipStream_t stream) {
    const dim3 grid(p.chunks, n_rows), block(kThreads);
    p.epoch = next_epoch();
    int32_t st = check_hip(launch_timed(sample_scan_kernel<E>, grid, block, stream, DIP_KERNEL_SAMPLE, p), "sample_scan launch");
    if (!st && cuts) st = check_hip(launch_timed(sample_cut_kernel<E>, grid, block, stream, DIP_KERNEL_SAMPLE, p), "sample_cut launch");
    if (st || !p.probs) return st;
    return check_hip(probs_dtype == DIP_F32 ? launch_timed(sample_probs_kernel<E, float>, grid, block, stream, DIP_KERNEL_SAMPLE, p)
                                            : launch_timed(sample_probs_kernel<E, __bf16>, grid, block, stream, DIP_KERNEL_SAMPLE, p),
                     "sample_probs launch");
}

}  // namespace
}  // namespace dip

using namespace dip;

extern "C" {

size_t dip_sample_workspace_bytes(int32_t n_rows, int32_t n_vocab) {
    if (check_sample(n_rows, n_vocab)) return 0;
    return plan_sample(n_rows, n_vocab).total;
}

int32_t dip_sample(const void* logits, int64_t stride, int32_t dtype, int32_t n_rows, int32_t n_vocab, const dip_sampling* how,
                   const float* u, int32_t* token, void* probs, int64_t probs_stride, int32_t probs_dtype, void* ws, size_t ws_bytes,
                   void* stream) {
    int32_t st = check_sample(n_rows, n_vocab);
    if (st) return st;
    if (!logits) return fail(DIP_ERR_INVALID_ARG, "sample: null pointer");
    if (!token && !probs) return fail(DIP_ERR_INVALID_ARG, "sample: neither token nor probs");
    if (token && !u) return fail(DIP_ERR_INVALID_ARG, "sample: a token is drawn by a number, and u is null");
    if (dtype != DIP_F32 && dtype != DIP_BF16) return fail(DIP_ERR_UNSUPPORTED, "sample: dtype %d", dtype);
    if (probs && probs_dtype != DIP_F32 && probs_dtype != DIP_BF16) return fail(DIP_ERR_UNSUPPORTED, "sample: probs_dtype %d", probs_dtype);
    const int es = elem_bytes(dtype), os = probs ? elem_bytes(probs_dtype) : 1;
    if (stride < n_vocab || (probs && probs_stride < n_vocab)) return fail(DIP_ERR_INVALID_ARG, "sample: strides smaller than a row");
    if (reinterpret_cast<uintptr_t>(logits) % es || reinterpret_cast<uintptr_t>(probs) % os)
        return fail(DIP_ERR_UNSUPPORTED, "sample: rows must be aligned to their elements");
    if (probs && !(probs == logits && probs_dtype == dtype && (probs_stride == stride || n_rows == 1)) &&
        rows_overlap(logits, stride * es, (int64_t)n_vocab * es, probs, probs_stride * os, (int64_t)n_vocab * os, n_rows))
        return fail(DIP_ERR_INVALID_ARG, "sample: probs overlaps logits without being it");
    const SamplePlan pl = plan_sample(n_rows, n_vocab);
    st = validate_ws(ws, ws_bytes, pl.total);
    if (st) return st;
    char* base = (char*)ws;
    SampleParams p;
    p.logits = (const char*)logits;
    p.stride = stride * es;
    p.n_vocab = n_vocab;
    p.chunks = pl.chunks;
    p.temperature = how ? how->temperature : nullptr;
    p.top_k = how ? how->top_k : nullptr;
    p.top_p = how ? how->top_p : nullptr;
    p.min_p = how ? how->min_p : nullptr;
    p.u = u;
    p.token = token;
    p.probs = (char*)probs;
    p.probs_stride = probs_stride * os;
    p.sums = (Chunk*)base;
    p.hist = (uint64_t*)(base + pl.off_hist);
    p.rows = (Row*)(base + pl.off_rows);
    p.list = (uint64_t*)(base + pl.off_list);
    p.tickets = (uint64_t*)(base + pl.off_tickets);
    const bool cuts = p.top_k || p.top_p || p.min_p;
    return dtype == DIP_F32 ? launch_sample<float>(p, n_rows, cuts, probs_dtype, (hipStream_t)stream)
                            : launch_sample<uint16_t>(p, n_rows, cuts, probs_dtype, (hipStream_t)stream);
}

}  // extern "C"
