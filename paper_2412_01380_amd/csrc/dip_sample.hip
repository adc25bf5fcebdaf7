// From logits to tokens and probabilities (dip_sample).
//
// The kept words are the first ones in order of (logit, number), so every rule is a cut in one order: behind the top_k-th word,
// behind the word at which the weights pass top_p of their sum, in front of the first word below min_p.  A cut is a logit and
// a number among the words that have it.  It is found without sorting:
//   sample_scan_kernel     a workgroup per chunk of a row: its maximum, and a histogram of count and weight over bins an eighth
//                          of a nat wide, aligned to a grid that all chunks share
//   sample_row_kernel      a workgroup per row adds the histograms up and says which bins, and so which logits, the cut lies
//                          in -- or, where no rule applies, draws
//   sample_collect_kernel  the words with these logits (a few in a hundred) go into a list
//   sample_cut_kernel      a workgroup per row narrows the cut down over the list, to a word, and draws; one rule after the other, each
//                          within the one bin that the running sums of the bins say
//   sample_probs_kernel    the probabilities
// A word's place is an integer: D = top - rint(8 2^23 l / T), in fp64, is how far below a grid line above the maximum it
// lies, in units of 2^-23 of a bin.  Its bin is D >> 23, and its weight exp(-bin / 8) times a factor in (0.88, 1] that follows
// from the other bits and is held in units of 2^-30.  So sums over a bin are integer sums, the same in any order, and 2^-26
// accurate relative to the weight itself however small it is (but for the last bin's, 63.75 nats and more down, which counts for
// nothing), and two chunks agree on every word's bin.  (Of an fp32 l / T 2^-24 is lost, which at 30 nats is a weight off by 2 in
// 10^6.)

#include <cfloat>
#include <cmath>
#include <type_traits>

#include "dip_vocab_device.h"

namespace dip {
namespace {

// Where the time goes: 512 rows of 128256, fp32, with probabilities, 228 us; under the profiler, logits that change from call to call:
// chunks 65 (263 MB; the integer places and the histogram take longer than the read, 41), rows 16, list 52, cut 31, probabilities 77
// (525 MB).  64 rows in bf16 without probabilities 49 us, four launches in a chain, a row of 32064 with them 34 us, five: the cut is the
// longest of them (14 to 23 us of loads, barriers and sums that wait for one another).  Without a rule 19 us for the 64 rows and 154
// for the 512, greedy 10 and 113.  Words that meet in one bin queue for its LDS word: where 95 % of them are -1e4 64 rows without a rule take
// 40 us and 512 303, and 18 and 138 where these are -inf, which no bin counts.
//
constexpr int kThreads = 256;             // of the kernels over chunks
constexpr int kRowThreads = 512;          // of the kernels that have a workgroup per row
constexpr int kTile = kThreads * kPer;
constexpr int kMaxTiles = 2;              // of a chunk, in registers (four: chunks 76 instead of 70 us, cut 35 instead of 29 of 512 rows of 128256)
constexpr int kMaxChunks = (1 << 24) / (kMaxTiles * kTile);
constexpr int kBins = 512;                // the last one: all that lies 64 nats and more below the maximum
constexpr int kRest = kBins - 1;
constexpr int kPlaceBits = 23;            // of a place within a bin
// Most words of a row's list.  Where more qualify, a workgroup goes through the row itself again: top_p 0.9 of 64 rows takes 49 us where
// logits deviate by 2.5, 60 by 1, 246 by 0.5, 408 where all are equal, and behind a top_k of 20000 307.
constexpr int kList = 8192;
constexpr int kRanges = 1024;             // key ranges of a step of narrowing down
constexpr int kFew = 64;                  // words that a wavefront puts in order
constexpr float kOne = 0x1p30f;           // weight 1 within a bin
constexpr int kCountShift = 45;           // a histogram word: count, weight
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

// rate = 8 2^23 / T, 0 for an infinite temperature; top: the grid line above a maximum (+inf where the maximum is).  A maximum
// on a grid line has bin 1.
__device__ __forceinline__ double place(float x, double rate) { return rint((double)x * rate); }
__device__ __forceinline__ double top_of(float best, double rate) {
    if (best == INFINITY) return (double)INFINITY;
    return (floor(place(best, rate) * 0x1p-23) + 1.0) * 0x1p23;
}
// how far a finite word lies below a finite top, at most 2^32 - 1
__device__ __forceinline__ uint32_t below(float x, double rate, double top) { return (uint32_t)fmin(top - place(x, rate), 4294967295.0); }
// its weight within its bin, in units of 2^-30: 1 + (exp(t) - 1) by the series of the latter, of which the first term left
// out is 1e-10
__device__ __forceinline__ uint32_t weight_at(uint32_t d) {
    const float t = (float)(d & ((1u << kPlaceBits) - 1)) * -0x1p-26f;
    float q = fmaf(t, kOne / 720.f, kOne / 120.f);
    q = fmaf(t, q, kOne / 24.f);
    q = fmaf(t, q, kOne / 6.f);
    q = fmaf(t, q, kOne / 2.f);
    q = fmaf(t, q, kOne);
    return (1u << 30) + (uint32_t)(int32_t)(q * t);
}
struct Place {
    int bin;
    uint32_t weight;
};
// of a word above -inf
__device__ __forceinline__ Place place_of(float x, double rate, double top) {
    if (top == (double)INFINITY) return x == INFINITY ? Place{0, 1u << 30} : Place{kRest, 0};
    const uint32_t d = below(x, rate, top);
    return {(int)(d >> kPlaceBits), weight_at(d)};
}
// what bins weigh: exp(-bin / 8) for weights in units of 2^-30, nothing behind the last
__device__ __forceinline__ void bin_scales(double* out) {
    for (int b = threadIdx.x; b < kBins; b += kRowThreads) out[b] = b == kRest ? 0.0 : exp(-0.125 * b) * 0x1p-30;
}
// bins that a chunk's top lies below the row's
__device__ __forceinline__ int bins_below(double chunk_top, double row_top) {
    if (row_top == (double)INFINITY) return chunk_top == (double)INFINITY ? 0 : kRest;
    return (int)fmin((row_top - chunk_top) * 0x1p-23, (double)kRest);
}

// ---- workspace -----------------------------------------------------------------------------------------
struct alignas(32) Chunk {
    double top;               // of its maximum, -inf: no words
    double weight;            // of its words, in units of exp(top / 8)
    float best;
    int32_t first;            // of a greedy row: the first word that has it
};
struct alignas(128) Row {
    double top;
    double rate;
    double total;             // of the kept words, in units of exp(top / 8)
    double part;              // top_p's share
    uint32_t key;             // kept: a larger key, or this one and a number up to
    int32_t at;
    int32_t state;
    int32_t greedy;
    int32_t lo;               // the first bin that the cut may lie in, and the keys of the bins that it may
    uint32_t least, most;
    int32_t k;                // words up to top_k's cut, 0: no such rule; its bin, and words and weight in front of that
    int32_t k_bin;
    uint32_t k_count;
    int32_t by_part;          // top_p cuts
    double k_weight;
    uint32_t min_key;         // min_p's cut, 0: no such rule
    int32_t listed;           // words with these keys: in the list, or too many for it
    uint32_t n;               // words in the list so far
    float best;               // the largest logit
};

struct SampleParams {
    const char* logits;
    int64_t stride;           // bytes
    int n_rows, n_vocab, chunks, chunk;
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
    double* bins;             // [row][kBins], of rows that top_p cuts: running weights of the bins
    uint64_t* list;           // [row][most_listed]: key, number
    int most_listed;          // kList, or a whole row
};

// a row's settings
struct How {
    float T;
    int k;                    // 0: all
    float part, least;        // 1 and more: all; 0: all
    bool greedy, cuts;
    double rate;
};
__device__ __forceinline__ How how_of(const SampleParams& p, int row) {
    How h;
    h.T = p.temperature ? p.temperature[row] : 1.f;
    h.greedy = !(h.T > 0.f);
    h.rate = h.greedy ? 0.0 : 0x1p26 / (double)h.T;
    const int k = p.top_k ? p.top_k[row] : 0;
    h.k = k > 0 && k < p.n_vocab ? k : 0;
    const float part = p.top_p ? p.top_p[row] : 1.f, least = p.min_p ? p.min_p[row] : 0.f;
    h.part = part < 1.f ? fmaxf(part, 0.f) : 1.f;
    h.least = isinf(h.T) || !(least > 0.f) ? 0.f : fminf(least, 1.f);
    h.cuts = !h.greedy && (h.k || h.part < 1.f || h.least > 0.f);
    return h;
}

__device__ __forceinline__ float widened(float x) { return x; }
__device__ __forceinline__ float widened(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
// kPer words from x on, -inf from `end` on and in place of NaN
template <typename E>
__device__ __forceinline__ void load_logits(const char* row, int x, int end, float (&f)[kPer]) {
    load_entries<E>(row, x, end, f);
#pragma unroll
    for (int i = 0; i < kPer; ++i) f[i] = fmaxf(f[i], -INFINITY);
    if (x + kPer > end)
#pragma unroll
        for (int i = 0; i < kPer; ++i) f[i] = x + i < end ? f[i] : -INFINITY;
}

// exclusive sum over a workgroup, in order of the threads; *total: of all
template <int THREADS, typename T>
__device__ __forceinline__ T block_before(T x, T* waves, T* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T upto = x;
    if constexpr (std::is_same<T, uint64_t>::value) {
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const T y = __shfl_up(upto, off);
            if (lane >= off) upto += y;
        }
    } else {
        upto = running(x);
    }
    __syncthreads();
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    T before = upto - x, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += waves[w];
        all += waves[w];
    }
    *total = all;
    return before;
}
template <int THREADS>
__device__ __forceinline__ float block_max(float x, float* waves) {
#pragma unroll
    for (int off = 32; off; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) x = fmaxf(x, waves[w]);
    return x;
}

// ---- chunks: grid (chunks, rows) ------------------------------------------------------------------------
template <typename E, int TILES>
__global__ void __launch_bounds__(kThreads) sample_scan_kernel(const SampleParams p) {
    __shared__ unsigned long long s_hist[kBins];
    __shared__ float s_max[kThreads / 64];
    __shared__ double s_sum[kThreads / 64];
    __shared__ int s_first;
    const int row = blockIdx.y, chunk = blockIdx.x, tid = threadIdx.x;
    const int begin = chunk * (TILES * kTile), end = min(p.n_vocab, begin + TILES * kTile);
    float f[TILES][kPer];
    float best = -INFINITY;
#pragma unroll
    for (int t = 0; t < TILES; ++t) load_logits<E>(p.logits + row * p.stride, begin + t * kTile + tid * kPer, end, f[t]);
    const How how = how_of(p, row);
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < kPer; ++i) best = fmaxf(best, f[t][i]);
    for (int b = tid; b < kBins; b += kThreads) s_hist[b] = 0;
    if (tid == 0) s_first = 0x7fffffff;
    best = block_max<kThreads>(best, s_max);
    const double top = best > -INFINITY ? top_of(best, how.rate) : -(double)INFINITY;
    Chunk* sum = p.sums + (size_t)row * p.chunks + chunk;
    if (tid == 0) {
        sum->top = top;
        sum->best = best;
    }
    if (how.greedy) {
        int first = 0x7fffffff;
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (f[t][i] == best) first = min(first, begin + t * kTile + tid * kPer + i);
        if (first != 0x7fffffff) atomicMin(&s_first, first);
        __syncthreads();
        if (tid == 0) sum->first = s_first;
        return;
    }
    if (best == INFINITY) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (f[t][i] > -INFINITY) {
                    const Place pl = place_of(f[t][i], how.rate, top);
                    atomicAdd(&s_hist[pl.bin], (1ull << kCountShift) | pl.weight);
                }
    } else if (best > -INFINITY) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (f[t][i] > -INFINITY) {
                    const uint32_t d = below(f[t][i], how.rate, top);
                    atomicAdd(&s_hist[d >> kPlaceBits], (1ull << kCountShift) | weight_at(d));
                }
    }
    __syncthreads();
    if (how.cuts) {
        uint64_t* out = p.hist + ((size_t)row * p.chunks + chunk) * kBins;
        for (int b = tid; b < kBins; b += kThreads) out[b] = s_hist[b];
    } else {
        double weight = 0.0, all;
        for (int b = tid; b < kRest; b += kThreads)
            if (const uint64_t h = s_hist[b]) weight += (double)(h & kWeightMask) * (exp(-0.125 * b) * 0x1p-30);
        block_before<kThreads>(weight, s_sum, &all);
        if (tid == 0) sum->weight = all;
    }
}

// The least of what the threads found, ascending with them (in LDS), by the first one of a wavefront that found anything;
// likewise the most, by the last one.  (512 atomics on one word take 3 us.)
__device__ __forceinline__ void to_least(int* least, bool found, int x) {
    const uint64_t mask = __ballot(found);
    if (mask && (int)(threadIdx.x & 63) == __ffsll((unsigned long long)mask) - 1) atomicMin(least, x);
}
__device__ __forceinline__ void to_most(int* most, bool found, int x) {
    const uint64_t mask = __ballot(found);
    if (mask && (int)(threadIdx.x & 63) == 63 - __clzll((long long)mask)) atomicMax(most, x);
}

// ---- the draw -----------------------------------------------------------------------------------------------
struct Draw {
    double scale[kBins];
    double chunk[kMaxChunks];             // weights of the chunks' kept words
    double waves[kRowThreads / 64];
    double target;
    int at, last;
};
// The place of the first of the threads' weights, in order, at which their running sum exceeds the target; where rounding leaves
// none, of the last weight above 0; -1: there is none.  weight(i), i < n: the thread's own, at place first + i, `before` in front of them.
template <typename F>
__device__ __forceinline__ int first_past(F weight, int n, int first, double before, double target, Draw& s) {
    if (threadIdx.x == 0) s.at = 0x7fffffff, s.last = -1;
    __syncthreads();
    int past = 0x7fffffff, some = -1;
    for (int i = 0; i < n; ++i) {
        const double w = weight(i);
        before += w;
        if (!(w > 0.0)) continue;
        some = first + i;
        if (before > target) past = min(past, first + i);
    }
    to_least(&s.at, past != 0x7fffffff, past);
    to_most(&s.last, some >= 0, some);
    __syncthreads();
    return s.at != 0x7fffffff ? s.at : s.last;
}
// kept: a key above `key`, or `key` and a number up to `at`.  Returns the sum of all; the token is thread 0's to write.
template <typename E>
__device__ __forceinline__ double draw(const SampleParams& p, int row, double top, double rate, uint32_t key, int at, Draw& s) {
    const int tid = threadIdx.x, lane = tid & 63;
    __syncthreads();
    // the chunk, contiguous ones to a thread
    const int per = (p.chunks + kRowThreads - 1) / kRowThreads, c0 = min(tid * per, p.chunks), n = min(p.chunks, c0 + per) - c0;
    double mine = 0.0;
    for (int i = 0; i < n; ++i) mine += s.chunk[c0 + i];
    double total;
    const double before = block_before<kRowThreads>(mine, s.waves, &total);
    if (!p.token) return total;
    const double target = (double)p.u[row] * total;
    const int c = first_past([&](int i) { return s.chunk[c0 + i]; }, n, c0, before, target, s);
    if (c < 0) {
        if (tid == 0) p.token[row] = -1;
        return total;
    }
    if (c >= c0 && c < c0 + n) {
        double sum = before;
        for (int i = c0; i < c; ++i) sum += s.chunk[i];
        s.target = target - sum;
    }
    // in it the thread's words, contiguous ones
    const char* logits = p.logits + row * p.stride;
    const int begin = c * p.chunk, end = min(begin + p.chunk, p.n_vocab), words = p.chunk / kRowThreads;     // 8, 16 or 32
    const float cut = of_key(key);                        // (of_key(kNothing) is -inf)
    auto weight_of = [&](float x, int number) {
        if (!(x > cut || (x == cut && number <= at)) || x == -INFINITY) return 0.0;
        const Place pl = place_of(x, rate, top);
        return (double)pl.weight * s.scale[pl.bin];
    };
    const int x = begin + tid * words;
    float f[kMaxTiles * kTile / kRowThreads / kPer][kPer];
    double sum = 0.0;
#pragma unroll
    for (int t = 0; t < kMaxTiles * kTile / kRowThreads / kPer; ++t)
        if (t * kPer < words) load_logits<E>(logits, x + t * kPer, min(end, x + words), f[t]);
#pragma unroll
    for (int t = 0; t < kMaxTiles * kTile / kRowThreads / kPer; ++t)
        if (t * kPer < words)
#pragma unroll
            for (int i = 0; i < kPer; ++i) sum += weight_of(f[t][i], x + t * kPer + i);
    double all;
    const double ahead = block_before<kRowThreads>(sum, s.waves, &all);
    const int thread = max(0, first_past([&](int) { return sum; }, 1, tid, ahead, s.target, s));
    __syncthreads();
    if (tid == thread) s.target -= ahead;
    __syncthreads();
    // and the word, a lane each
    if (tid < 64) {
        const int number = begin + thread * words + lane;
        double w = 0.0;
        if (lane < words && number < end) w = weight_of(fmaxf(entry_at<E>(logits, number), -INFINITY), number);
        const double upto = running(w);
        const uint64_t past = __ballot(w > 0.0 && upto > s.target), some = __ballot(w > 0.0);
        const int first = past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : -1;
        if (lane == 0) p.token[row] = first >= 0 ? number + first : -1;
    }
    return total;
}

// ---- what a row is to be cut at: grid (rows) --------------------------------------------------------------------
// The smallest key whose word lies in one of the first `bins` bins below a finite top, by one wavefront: 64 candidates at a
// time (a word's place falls as its key rises).
__device__ __forceinline__ uint32_t least_key(double rate, double top, int bins) {
    uint32_t from = kNothing + 1;         // the answer is `from` or more ...
    const int lane = threadIdx.x & 63;
    for (int shift = 26;; shift -= 6) {   // ... and less than from + 64 << shift
        shift = max(shift, 0);
        const uint64_t key = (uint64_t)from + ((uint64_t)lane << shift);
        const bool in = key > 0xff7fffffull || top - place(of_key((uint32_t)key), rate) < bins * 0x1p23;
        const uint64_t mask = __ballot(in);
        const int first = mask ? __ffsll((unsigned long long)mask) - 1 : 64;
        if (shift == 0) return first ? from + first : from;
        from += first ? (uint32_t)(first - 1) << shift : 0;
        if (!first) return from;
    }
}

template <typename E>
__global__ void __launch_bounds__(kRowThreads) sample_row_kernel(const SampleParams p) {
    __shared__ Draw s;
    __shared__ double s_weight[kBins];
    __shared__ uint32_t s_count[kBins];
    __shared__ int s_below[kMaxChunks];
    __shared__ float s_max[kRowThreads / 64];
    __shared__ uint32_t s_waves[kRowThreads / 64];
    __shared__ int s_range[2];
    const int row = blockIdx.x, tid = threadIdx.x;
    const How how = how_of(p, row);
    const Chunk* sums = p.sums + (size_t)row * p.chunks;
    Row* r = p.rows + row;
    float best = -INFINITY;
    for (int c = tid; c < p.chunks; c += kRowThreads) best = fmaxf(best, sums[c].best);
    best = block_max<kRowThreads>(best, s_max);
    if (best == -INFINITY || how.greedy) {
        if (tid == 0) s_range[0] = 0x7fffffff;
        __syncthreads();
        if (best > -INFINITY)
            for (int c = tid; c < p.chunks; c += kRowThreads)
                if (sums[c].best == best) atomicMin(&s_range[0], sums[c].first);
        __syncthreads();
        if (tid == 0) {
            r->state = best > -INFINITY ? kDone : kEmpty;
            r->greedy = 1;
            r->key = key_of(best);
            r->at = s_range[0];
            r->total = 1.0;
            r->top = r->rate = 0.0;
            if (p.token) p.token[row] = best > -INFINITY ? s_range[0] : -1;
        }
        return;
    }
    const double top = top_of(best, how.rate);
    bin_scales(s.scale);
    if (tid == 0) {
        r->state = kDone;
        r->greedy = 0;
        r->best = best;
        r->top = top;
        r->rate = how.rate;
        r->key = kNothing;
        r->at = -1;
    }
    __syncthreads();
    for (int c = tid; c < p.chunks; c += kRowThreads) {
        const int off = bins_below(sums[c].top, top);
        s_below[c] = off;
        // (a chunk whose largest word is in the last bin of the row has nothing to draw, whatever it weighs beside that word)
        const bool some = off < kRest && place_of(sums[c].best, how.rate, top).bin < kRest;
        s.chunk[c] = !some || how.cuts ? 0.0 : sums[c].weight * (s.scale[off] * 0x1p30);
    }
    __syncthreads();
    if (!how.cuts) {
        const double total = draw<E>(p, row, top, how.rate, kNothing, -1, s);
        if (tid == 0) r->total = total;
        return;
    }

    // counts and weights of the row's bins, and their running sums
    const uint64_t* hist = p.hist + (size_t)row * p.chunks * kBins;
    constexpr int PER = kBins / kRowThreads;
    uint32_t cnt[PER], cnt_sum = 0, rest = 0;
    double wgt[PER], wgt_sum = 0.0;
    uint64_t w[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) cnt[i] = 0, w[i] = 0;
    constexpr int FLIGHT = 16;            // chunks on their way at a time
    for (int c0 = 0; c0 < p.chunks; c0 += FLIGHT) {
        uint64_t h[FLIGHT][PER];
#pragma unroll
        for (int c = 0; c < FLIGHT; ++c) {
            const int off = c0 + c < p.chunks ? s_below[c0 + c] : kBins;
#pragma unroll
            for (int i = 0; i < PER; ++i) {               // (a chunk whose maximum lies lower: its bins are shifted)
                const int b = tid * PER + i;
                h[c][i] = b >= off && (off == 0 || b < kRest) ? hist[(size_t)(c0 + c) * kBins + b - off] : 0;
            }
        }
#pragma unroll
        for (int c = 0; c < FLIGHT; ++c)
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                cnt[i] += (uint32_t)(h[c][i] >> kCountShift);
                w[i] += h[c][i] & kWeightMask;
            }
    }
    // what is shifted out of them
    for (int c = tid / 64; c < p.chunks; c += kRowThreads / 64)
        for (int b = kBins - 1 - (tid & 63); s_below[c] && b >= max(0, kRest - s_below[c]); b -= 64) rest += (uint32_t)(hist[(size_t)c * kBins + b] >> kCountShift);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        wgt[i] = (double)w[i] * s.scale[tid * PER + i];
        cnt_sum += cnt[i];
        wgt_sum += wgt[i];
    }
    uint32_t known, more;
    uint32_t cnt_before = block_before<kRowThreads>(cnt_sum, s_waves, &known);
    block_before<kRowThreads>(rest, s_waves, &more);
    const uint32_t n_words = known + more;
    if (tid == kRowThreads - 1) cnt[PER - 1] += more;
    double total;
    double wgt_before = block_before<kRowThreads>(wgt_sum, s.waves, &total);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = tid * PER + i;
        s_count[b] = cnt_before += cnt[i];
        s_weight[b] = wgt_before += wgt[i];
    }
    __syncthreads();
    if (tid < 64) {
        // the first bin at which the running sums satisfy a rule: every lane looks at eight neighbouring ones
        auto bin_of = [&](auto past) {
            int first = kRest;
            for (int i = kBins / 64 - 1; i >= 0; --i)
                if (past(tid * (kBins / 64) + i)) first = tid * (kBins / 64) + i;
            const uint64_t mask = __ballot(past(tid * (kBins / 64) + kBins / 64 - 1));
            const int lane = mask ? __ffsll((unsigned long long)mask) - 1 : 63;
            return __shfl(first, lane);
        };
        auto count_to = [&](int b) { return b < 0 ? 0u : s_count[b]; };
        auto weight_to = [&](int b) { return b < 0 ? 0.0 : s_weight[b]; };
        bool by_k = how.k && (uint32_t)how.k < n_words, by_part = how.part < 1.f;
        int lo = kBins, hi = -1, bin_k = kRest;
        if (by_k) lo = hi = bin_k = bin_of([&](int b) { return s_count[b] >= (uint32_t)how.k; });
        if (by_part) {
            const double from = (double)how.part * (by_k ? weight_to(bin_k - 1) : total), to = (double)how.part * (by_k ? weight_to(bin_k) : total);
            lo = min(bin_k, bin_of([&](int b) { return s_weight[b] >= from && s_count[b] > 0; }));
            hi = by_k ? bin_k : min(bin_k, bin_of([&](int b) { return s_weight[b] >= to && s_count[b] > 0; }));
        }
        uint32_t min_key = 0;
        if (how.least > 0.f) {
            const double c = how.least < 1.f ? (double)best + (double)how.T * log((double)how.least) : (double)best;
            float at = (float)c;
            if ((double)at < c) at = of_key(key_of(at) + 1);
            if (at > -INFINITY) {
                min_key = key_of(at);
                const int b = place_of(at, how.rate, top).bin;
                if (b < lo) {
                    lo = hi = b;
                    by_k = by_part = false;
                }
            }
        }
        if (lo <= hi) {
            // the keys that these bins hold
            uint32_t least = kNothing + 1, most = 0xff800000u;
            if (top != (double)INFINITY) {
                if (hi < kRest) least = least_key(how.rate, top, hi + 1);
                most = lo > 0 ? least_key(how.rate, top, lo) - 1 : 0xff7fffffu;
            } else if (hi == 0) {
                least = most;
            } else if (lo == kRest) {
                most = 0xff7fffffu;
            }
            if (by_part)
                for (int b = tid; b < kBins; b += 64) p.bins[(size_t)row * kBins + b] = s_weight[b];
            if (tid == 0) {
                r->state = kCut;
                r->part = (double)how.part;
                r->lo = lo;
                r->least = least;
                r->most = most;
                r->k = by_k ? how.k : 0;
                r->k_bin = bin_k;
                r->k_count = count_to(bin_k - 1);
                r->k_weight = weight_to(bin_k - 1);
                r->by_part = by_part;
                r->min_key = min_key;
                r->listed = (int)(count_to(hi) - count_to(lo - 1));
                r->total = total;
                r->n = 0;
            }
        }
        if (tid == 0) s_range[0] = lo <= hi;
    }
    __syncthreads();
    if (s_range[0]) return;
    // nothing cuts this row after all
    for (int c = tid >> 6; c < p.chunks; c += kRowThreads / 64) {
        double sum = 0.0;
        for (int b = tid & 63; b < kRest - s_below[c]; b += 64) sum += (double)(hist[(size_t)c * kBins + b] & kWeightMask) * s.scale[b + s_below[c]];
        sum = wave_sum(sum);
        if ((tid & 63) == 0) s.chunk[c] = sum;
    }
    __syncthreads();
    total = draw<E>(p, row, top, how.rate, kNothing, -1, s);
    if (tid == 0) r->total = total;
}

// ---- words that the cut lies among: grid (chunks, rows) -----------------------------------------------------------
template <typename E, int TILES>
__global__ void __launch_bounds__(kThreads) sample_collect_kernel(const SampleParams p) {
    __shared__ uint32_t s_waves[kThreads / 64];
    __shared__ uint32_t s_at;
    const int row = blockIdx.y, tid = threadIdx.x;
    Row* r = p.rows + row;
    if (r->state != kCut || r->listed > p.most_listed) return;
    const float least = of_key(r->least), most = of_key(r->most);
    const int begin = blockIdx.x * (TILES * kTile), end = min(p.n_vocab, begin + TILES * kTile);
    const float best = p.sums[(size_t)row * p.chunks + blockIdx.x].best;
    if (best < least) return;
    float f[TILES][kPer];
    uint64_t hits = 0;                    // a bit per word
    static_assert(kMaxTiles * kPer <= 64, "a bit per word");
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
        load_logits<E>(p.logits + row * p.stride, begin + t * kTile + tid * kPer, end, f[t]);
        uint32_t mask = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) mask |= f[t][i] >= least && f[t][i] <= most ? 1u << i : 0u;
        hits |= (uint64_t)mask << (t * kPer);
    }
    uint32_t all;
    const uint32_t before = block_before<kThreads>((uint32_t)__popcll(hits), s_waves, &all);
    if (!all) return;
    if (tid == 0) s_at = atomicAdd(&r->n, all);
    __syncthreads();
    uint32_t at = s_at + before;
    uint64_t* list = p.list + (size_t)row * p.most_listed;
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (hits >> (t * kPer + i) & 1) {
                if (at < (uint32_t)p.most_listed) list[at] = ((uint64_t)key_of(f[t][i]) << 32) | (uint32_t)(begin + t * kTile + tid * kPer + i);
                ++at;
            }
}

// ---- the cut: grid (rows) --------------------------------------------------------------------------------------------
struct Cut {
    Draw d;
    union {
        struct {
            uint32_t count[kRanges];
            unsigned long long weight[kRanges];
        } range;
        unsigned long long fixed[kMaxChunks];     // chunk weights of the listed words
    };
    uint64_t few[kFew];
    uint64_t waves_u[kRowThreads / 64];
    uint32_t waves_i[kRowThreads / 64];
    int at, last;
    uint32_t n_few, key;
    uint32_t count, here;
    double weight, each;
};
struct Listed {
    int row, n;
    bool listed;
    double rate, top;
    uint32_t least, most;     // keys of the list
    int bin;                  // the one that is looked at, and keys that it lies between
    uint32_t bin_least, bin_most;
    __device__ __forceinline__ void look_at(int b) {
        bin = b;
        bin_least = least;
        bin_most = most;
        if (top == (double)INFINITY || rate == 0.0) return;
        // its words' places, a unit and two keys to either side for what rounding may do
        const double high = (top - (double)b * 0x1p23 + 1.0) / rate, low = (top - (double)(b + 1) * 0x1p23 - 1.0) / rate;
        bin_most = max(least, min(most, key_of((float)high) + 2));
        if (b < kRest) bin_least = min(most, max(least, key_of((float)low) - 2));
    }
};
// f(key, number) of every word whose key lies among those that the cut may have, by the threads of a workgroup
template <typename E, typename F>
__device__ __forceinline__ void each_word(const SampleParams& p, const Listed& l, F f) {
    constexpr int FLIGHT = 8;
    if (l.listed) {
        const uint64_t* list = p.list + (size_t)l.row * p.most_listed;
        for (int i0 = threadIdx.x; i0 < l.n; i0 += FLIGHT * kRowThreads) {
            uint64_t e[FLIGHT];
#pragma unroll
            for (int i = 0; i < FLIGHT; ++i) e[i] = list[min(i0 + i * kRowThreads, l.n - 1)];
#pragma unroll
            for (int i = 0; i < FLIGHT; ++i)
                if (i0 + i * kRowThreads < l.n) f((uint32_t)(e[i] >> 32), (int)(uint32_t)e[i]);
        }
    } else {
        const char* logits = p.logits + l.row * p.stride;
        for (int x0 = threadIdx.x; x0 < p.n_vocab; x0 += FLIGHT * kRowThreads) {
            float v[FLIGHT];
#pragma unroll
            for (int i = 0; i < FLIGHT; ++i) v[i] = entry_at<E>(logits, min(x0 + i * kRowThreads, p.n_vocab - 1));
#pragma unroll
            for (int i = 0; i < FLIGHT; ++i) {
                const uint32_t k = key_of(fmaxf(v[i], -INFINITY));
                if (x0 + i * kRowThreads < p.n_vocab && k >= l.least && k <= l.most) f(k, x0 + i * kRowThreads);
            }
        }
    }
}
// add(n) by the active lanes: those that agree with the first of them in `at` and `key` leave it to that one, n of them together.
// (A wavefront's atomics on one LDS word take their turns: rows of 128256 equal logits 935 us one by one, 494 so, all rules; 408 since
// each rule looks at one bin.)
template <typename F>
__device__ __forceinline__ void add_alike(uint32_t at, uint32_t key, F add) {
    const bool alike = at == (uint32_t)__builtin_amdgcn_readfirstlane((int)at) && key == (uint32_t)__builtin_amdgcn_readfirstlane((int)key);
    const uint64_t mask = __ballot(alike);
    if (!alike) add(1u);
    else if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)mask) - 1) add((uint32_t)__popcll(mask));
}
// Whether a listed word lies in the bin that is looked at; its weight there, in units of the bin's: 2^24 of them fit 64 bits, and nothing is
// lost.  (Weights of several bins in units of the first one's are a few units each where the others lie 20 nats below it.)
__device__ __forceinline__ bool in_bin(const Listed& l, uint32_t key, uint32_t& weight) {
    const Place pl = place_of(of_key(key), l.rate, l.top);
    weight = pl.bin == kRest ? 0 : pl.weight;
    return pl.bin == l.bin;
}

// The number of the m-th word (from 1) of those with a key in [least, most], in order of their numbers; their key in s.key.
template <typename E>
__device__ __forceinline__ int nth(const SampleParams& p, const Listed& l, uint32_t least, uint32_t most, uint32_t m, Cut& s) {
    const int tid = threadIdx.x;
    constexpr int PER = kRanges / kRowThreads;
    uint32_t lo = 0, skipped = 0;
    for (int shift = max(0, 32 - __clz(p.n_vocab) - 10);; shift = max(0, shift - 10)) {
        __syncthreads();
        for (int i = tid; i < kRanges; i += kRowThreads) s.range.count[i] = 0;
        if (tid == 0) s.at = kRanges - 1;
        __syncthreads();
        each_word<E>(p, l, [&](uint32_t k, int number) {
            const uint32_t at = ((uint32_t)number - lo) >> shift;
            if (k < least || k > most || (uint32_t)number < lo || at >= kRanges) return;
            add_alike(at, 0, [&](uint32_t n) { atomicAdd(&s.range.count[at], n); });
            s.key = k;
        });
        __syncthreads();
        uint32_t mine = 0, all;
        for (int i = 0; i < PER; ++i) mine += s.range.count[tid * PER + i];
        const uint32_t before = block_before<kRowThreads>(mine, s.waves_i, &all);
        uint32_t run = skipped + before;
        int found = kRanges;
        for (int i = 0; i < PER; ++i) {
            run += s.range.count[tid * PER + i];
            if (run >= m) found = min(found, tid * PER + i);
        }
        to_least(&s.at, found < kRanges, found);
        __syncthreads();
        const int at = s.at;
        if (tid == at / PER) {
            uint32_t c = skipped + before;
            for (int i = tid * PER; i < at; ++i) c += s.range.count[i];
            s.count = c;
        }
        __syncthreads();
        skipped = s.count;
        lo += (uint32_t)at << shift;
        if (shift == 0) return (int)lo;
    }
}

// The word at which the listed ones of the bin, in order, first come to `need` words or to `need` in weight: its key in s.key, its
// number in s.at, and what all up to it weigh in s.weight.  Words behind (end_key, end_at) are not looked at.
template <typename E, bool WEIGHT>
__device__ __forceinline__ void find(const SampleParams& p, const Listed& l, uint32_t end_key, int end_at, double need, Cut& s) {
    const int tid = threadIdx.x, lane = tid & 63;
    constexpr int PER = kRanges / kRowThreads;
    uint32_t least = max(end_key, l.bin_least), most = max(least, l.bin_most), count = 0;
    double weight = 0.0;
    auto ends = [&](uint32_t k, int number) { return k == end_key && number > end_at; };
    for (;;) {
        const uint32_t span = most - least;
        const int bits = span ? 32 - __clz((int)span) : 1, shift = max(0, bits - 10);
        __syncthreads();
        for (int i = tid; i < kRanges; i += kRowThreads) {
            s.range.count[i] = 0;
            s.range.weight[i] = 0;
        }
        if (tid == 0) s.at = kRanges, s.last = 0, s.n_few = 0;
        __syncthreads();
        each_word<E>(p, l, [&](uint32_t k, int number) {
            if (k < least || k > most || ends(k, number)) return;
            const uint32_t at = (most - k) >> shift;
            uint32_t w;
            if (!in_bin(l, k, w)) return;
            add_alike(at, k, [&](uint32_t n) {
                atomicAdd(&s.range.count[at], n);
                atomicAdd(&s.range.weight[at], (unsigned long long)w * n);
            });
        });
        __syncthreads();
        uint32_t c_mine = 0, c_all;
        uint64_t w_mine = 0, w_all;
        for (int i = 0; i < PER; ++i) {
            c_mine += s.range.count[tid * PER + i];
            w_mine += s.range.weight[tid * PER + i];
        }
        const uint32_t c_before = block_before<kRowThreads>(c_mine, s.waves_i, &c_all);
        const uint64_t w_before = block_before<kRowThreads>(w_mine, s.waves_u, &w_all);
        uint32_t c_run = c_before;
        uint64_t w_run = w_before;
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
        to_least(&s.at, found < kRanges, found);
        to_most(&s.last, some > 0, some);
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
            s.count = count + c;
            s.weight = weight + (double)w;
            s.here = s.range.count[at];
            s.each = s.range.count[at] ? (double)s.range.weight[at] / (double)s.range.count[at] : 0.0;
        }
        __syncthreads();
        count = s.count;
        weight = s.weight;
        const uint32_t here = s.here, high = most - ((uint32_t)at << shift), width = (1u << shift) - 1;
        least = high - least > width ? high - width : least;
        most = high;
        if (here == 0) {                                  // (no listed word: nothing is cut)
            if (tid == 0) s.key = kNothing, s.at = 0x7fffffff;
            __syncthreads();
            return;
        }
        if (here <= (uint32_t)kFew) {
            each_word<E>(p, l, [&](uint32_t k, int number) {
                uint32_t w;
                if (k < least || k > most || ends(k, number) || !in_bin(l, k, w)) return;
                s.few[atomicAdd(&s.n_few, 1u)] = ((uint64_t)k << 32) | (uint32_t)~number;
            });
            __syncthreads();
            if (tid < 64) {                               // every lane a word: what lies in front of it
                const uint64_t mine = lane < (int)here ? s.few[lane] : 0;
                uint32_t w = 0, c = 1;
                if (lane < (int)here) in_bin(l, (uint32_t)(mine >> 32), w);
                uint64_t upto = w;
                for (int j = 0; j < (int)here; ++j) {
                    const uint64_t other = s.few[j];
                    const uint32_t ow = __shfl(w, j);
                    if (other > mine) {
                        ++c;
                        upto += ow;
                    }
                }
                const double have = WEIGHT ? weight + (double)upto : (double)(count + c);
                // the first that comes to the need, or the last
                const uint64_t past = __ballot(lane < (int)here && have >= need);
                uint32_t rank = lane < (int)here && (past == 0 || (past >> lane & 1)) ? c : past ? 65u : 0u;
                for (int off = 32; off; off >>= 1) {
                    const uint32_t y = __shfl_xor(rank, off);
                    rank = past ? min(rank, y) : max(rank, y);
                }
                if (lane < (int)here && c == rank) {
                    s.key = (uint32_t)(mine >> 32);
                    s.at = (int)~(uint32_t)mine;
                    s.weight = weight + (double)upto;
                }
            }
            __syncthreads();
            return;
        }
        // one logit that many words have: a range is no wider than the distance of two
        if (shift <= (sizeof(E) == 2 ? 15 : 0)) {
            double more = WEIGHT ? (s.each > 0.0 ? ceil((need - weight) / s.each) : 1.0) : need - (double)count;
            more = fmin(fmax(more, 1.0), (double)here);
            const double all = weight + more * s.each;
            const int number = nth<E>(p, l, least, most, (uint32_t)more, s);
            __syncthreads();
            if (tid == 0) {
                s.at = number;
                s.weight = all;
            }
            __syncthreads();
            return;
        }
    }
}

template <typename E>
__global__ void __launch_bounds__(kRowThreads) sample_cut_kernel(const SampleParams p) {
    __shared__ Cut s;
    const int row = blockIdx.x, tid = threadIdx.x;
    Row* rp = p.rows + row;
    if (rp->state != kCut) return;
    const Row r = *rp;
    Listed l = {row, min((int)r.n, p.most_listed), r.listed <= p.most_listed, r.rate, r.top, r.least, r.most};
    bin_scales(s.d.scale);
    const double upto = r.by_part ? p.bins[(size_t)row * kBins + tid] : 0.0, before = r.by_part && tid > 0 ? p.bins[(size_t)row * kBins + tid - 1] : 0.0;
    static_assert(kRowThreads == kBins, "a bin of each thread");
    __syncthreads();
    // the weight that a bin's are units of (behind the last but one nothing weighs anything)
    const auto unit = [&](int bin) { return s.d.scale[min(bin, kRest - 1)]; };
    double total = r.total;
    uint32_t key = kNothing;
    int at = 0x7fffffff;
    if (r.k) {
        l.look_at(r.k_bin);
        find<E, false>(p, l, key, at, (double)((uint32_t)r.k - r.k_count), s);
        key = s.key;
        at = s.at;
        total = r.k_weight + s.weight * unit(l.bin);
    }
    if (r.by_part) {
        // the first bin that the running weights pass the need in, up to top_k's
        const double need = r.part * total;
        __syncthreads();
        if (tid == 0) s.at = r.k ? r.k_bin : kRest;
        __syncthreads();
        to_least(&s.at, tid >= r.lo && upto >= need, tid);
        __syncthreads();
        l.look_at(s.at);
        if (tid == l.bin) s.d.target = need - before;
        __syncthreads();
        find<E, true>(p, l, key, at, s.d.target / unit(l.bin), s);
        key = s.key;
        at = s.at;
    }
    if (r.min_key > key) {
        key = r.min_key;
        at = 0x7fffffff;
    }
    // the chunks' words above the bin that the cut lies in, a wavefront per chunk
    l.look_at(place_of(of_key(key), r.rate, r.top).bin);
    const Chunk* sums = p.sums + (size_t)row * p.chunks;
    const uint64_t* hist = p.hist + (size_t)row * p.chunks * kBins;
    for (int c = tid >> 6; c < p.chunks; c += kRowThreads / 64) {
        const int off = bins_below(sums[c].top, r.top);
        double w = 0.0;
        for (int b = tid & 63; b < l.bin - off; b += 64) w += (double)(hist[(size_t)c * kBins + b] & kWeightMask) * s.d.scale[b + off];
        w = wave_sum(w);
        if ((tid & 63) == 0) s.d.chunk[c] = w;
    }
    // the kept ones of the bin itself
    __syncthreads();
    for (int c = tid; c < p.chunks; c += kRowThreads) s.fixed[c] = 0;
    __syncthreads();
    each_word<E>(p, l, [&](uint32_t k, int number) {
        uint32_t w;
        if (k < key || (k == key && number > at) || !in_bin(l, k, w)) return;
        const uint32_t c = (uint32_t)number / (uint32_t)p.chunk;
        add_alike(c, k, [&](uint32_t n) { atomicAdd(&s.fixed[c], (unsigned long long)w * n); });
    });
    __syncthreads();
    for (int c = tid; c < p.chunks; c += kRowThreads) s.d.chunk[c] += (double)s.fixed[c] * unit(l.bin);
    total = draw<E>(p, row, r.top, r.rate, key, at, s.d);
    if (tid == 0) {
        rp->total = total;
        rp->key = key;
        rp->at = at;
        rp->state = kDone;
    }
}

// ---- probabilities: grid (tiles, rows) ----------------------------------------------------------------------------
// Four neighbouring words of a thread at a time, so that a wavefront writes one run of whole lines, past the caches: what they hold of
// the logits is worth more.  (Sixteen of a thread, through the caches: 120 instead of 81 us for 512 rows of 128256 in fp32, and the next
// call's chunks and list 70 and 50 instead of 57 and 43.  Read four at a time, these two take 62 and 47.)
template <typename E, typename O>
__global__ void __launch_bounds__(kThreads) sample_probs_kernel(const SampleParams p) {
    constexpr int N = 4, GROUPS = kTile / (N * kThreads);
    typedef E In __attribute__((ext_vector_type(N), aligned(sizeof(E))));
    typedef O Out __attribute__((ext_vector_type(N), aligned(sizeof(O))));
    const int row = blockIdx.y, x0 = blockIdx.x * kTile + threadIdx.x * N;
    const char* logits = p.logits + row * p.stride;
    float f[GROUPS][N];
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
        const int x = x0 + j * (N * kThreads);
        if (x + N <= p.n_vocab) {
            const In v = *(const In*)(logits + (size_t)x * sizeof(E));
#pragma unroll
            for (int i = 0; i < N; ++i) f[j][i] = widened(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) f[j][i] = x + i < p.n_vocab ? entry_at<E>(logits, x + i) : -INFINITY;
        }
    }
    const Row* rp = p.rows + row;
    const int state = rp->state, at = rp->at;
    const bool greedy = rp->greedy;
    const float cut = of_key(rp->key);
    // weights relative to the largest logit's: differences of logits are exact, of 8 l / T they are not where T is next to nothing
    const double top = rp->top, rate = rp->rate, best = (double)rp->best, step = rate * (0x1p-26 * 1.44269504088896340736);
    float each = 0.f;
    if (state != kEmpty && !greedy) {
        const Place first = place_of(rp->best, rate, top);
        each = (float)((double)first.weight * (first.bin ? 0.88249690258459540286 : 1.0) * 0x1p-30 / rp->total);
    }
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
        const int x = x0 + j * (N * kThreads);
        if (x >= p.n_vocab) break;
        bool kept[N], any = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {                     // (a NaN is neither above the cut nor at it)
            kept[i] = state != kEmpty && f[j][i] > -INFINITY && (f[j][i] > cut || (f[j][i] == cut && x + i <= at));
            any |= kept[i];
        }
        float y[N] = {0.f, 0.f, 0.f, 0.f};
        if (__any(any)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float w;
                if (greedy) w = 1.f;
                else if (top == (double)INFINITY) w = f[j][i] == INFINITY ? each : 0.f;
                else {                                    // 2^(whole + part)
                    const double z = ((double)f[j][i] - best) * step, whole = floor(fmax(z, -400.0));
                    w = ldexpf(__builtin_amdgcn_exp2f((float)(z - whole)) * each, (int)whole);
                }
                y[i] = kept[i] ? w : 0.f;
            }
        }
        O* out = (O*)(p.probs + row * p.probs_stride) + x;
        if (x + N <= p.n_vocab) {
            Out a;
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] = (O)y[i];
            __builtin_nontemporal_store(a, (Out*)out);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (x + i < p.n_vocab) out[i] = (O)y[i];
        }
    }
}

struct SamplePlan {
    int tiles, chunks, most_listed;
    size_t off_hist, off_rows, off_bins, off_list, total;
};
SamplePlan plan_sample(int n_rows, int n_vocab) {
    SamplePlan pl;
    const int64_t tiles = (n_vocab + kTile - 1) / kTile;
    pl.tiles = kMaxTiles;
    while (pl.tiles > 1 && n_rows * ((tiles + pl.tiles - 1) / pl.tiles) < 1024 && tiles / (pl.tiles / 2) < kMaxChunks) pl.tiles /= 2;
    pl.chunks = (int)((tiles + pl.tiles - 1) / pl.tiles);
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    const size_t parts = (size_t)n_rows * pl.chunks;
    take(sizeof(Chunk) * parts);
    pl.off_hist = take(sizeof(uint64_t) * kBins * parts);
    pl.off_rows = take(sizeof(Row) * n_rows);
    pl.off_bins = take(sizeof(double) * kBins * n_rows);
    pl.most_listed = n_vocab < kList ? n_vocab : kList;
    pl.off_list = take(sizeof(uint64_t) * pl.most_listed * n_rows);
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
int32_t launch_sample(const SampleParams& p, const SamplePlan& pl, bool cuts, int probs_dtype, hipStream_t stream) {
    const dim3 chunks(p.chunks, p.n_rows), rows(p.n_rows), tiles((p.n_vocab + kTile - 1) / kTile, p.n_rows), wide(kThreads), tall(kRowThreads);
    const auto go = [&](auto kernel, dim3 grid, dim3 block, const char* what) { return check_hip(launch_timed(kernel, grid, block, stream, DIP_KERNEL_SAMPLE, p), what); };
    int32_t st = go(pl.tiles == 2 ? sample_scan_kernel<E, 2> : sample_scan_kernel<E, 1>, chunks, wide, "sample_scan launch");
    if (!st) st = go(sample_row_kernel<E>, rows, tall, "sample_row launch");
    if (!st && cuts)
        st = go(pl.tiles == 2 ? sample_collect_kernel<E, 2> : sample_collect_kernel<E, 1>, chunks, wide,
                "sample_collect launch");
    if (!st && cuts) st = go(sample_cut_kernel<E>, rows, tall, "sample_cut launch");
    if (!st && p.probs) st = go(probs_dtype == DIP_F32 ? sample_probs_kernel<E, float> : sample_probs_kernel<E, __bf16>, tiles, wide, "sample_probs launch");
    return st;
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
    p.n_rows = n_rows;
    p.n_vocab = n_vocab;
    p.chunks = pl.chunks;
    p.chunk = pl.tiles * kTile;
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
    p.bins = (double*)(base + pl.off_bins);
    p.list = (uint64_t*)(base + pl.off_list);
    p.most_listed = pl.most_listed;
    const bool cuts = p.top_k || p.top_p || p.min_p;
    return dtype == DIP_F32 ? launch_sample<float>(p, pl, cuts, probs_dtype, (hipStream_t)stream)
                            : launch_sample<uint16_t>(p, pl, cuts, probs_dtype, (hipStream_t)stream);
}

}  // extern "C"
