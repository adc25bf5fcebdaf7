// Verification of drafted trees against the target's probabilities (dip_verify_tree).
//
// The usual rule tries the children of a node in turn and replaces the target r by norm((r - q)+)
// after each refusal.  Written without the norms, the j-th r is (p - lam_j q)+ / G_j with
// lam_0 = 0, G_0 = 1, lam_{j+1} = lam_j + G_j and G_j the sum of (p - lam_j q)+: for a node that
// was refused j children everything about its rows is in the numbers lam_j and G_j, and a child's test
// needs two probabilities and these.  So the walk itself is a few loads, done by every workgroup for
// itself, and the passes over whole rows are plain sums that split over any number of workgroups:
// G_1 .. G_{m-1} of the nodes with several children (one launch each: lam_{j+1} needs G_j), then the sum
// over the row at which the walk ends, then the draw.
// Sums and comparisons are in fp64: the outputs are decisions, and with sums that are 1e-16 off in
// whatever order they are taken, all orders decide alike (an fp32 sum of 128000 terms leaves 1 in 10^5
// draws open).  fp64 adds at half the fp32 rate cost nothing here: the kernels wait for memory.

#include "dip_decode_internal.h"

namespace dip {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxChunks = 64;            // of a row; a lane of one wavefront sums each
constexpr int kMinChunk = 4096;           // entries: 16 a thread

struct VerifyParams {
    BatchView b;
    const int32_t* tokens;
    const int32_t* parents;
    const char* p;
    const char* q;
    int64_t p_stride;         // bytes
    int64_t q_stride;
    int n_vocab;
    int chunk;                // entries of a chunk, a multiple of 8
    int chunks;
    const float* u;
    const float* u_sample;
    int max_kids;
    int round;                // G_j that a sums launch computes
    double* g_part;           // [max_kids - 1][n_rows][chunks]: G_1 ..
    double* w_part;           // [n_batch][chunks] sums of (p - lam q)+ at the last node
    double* p_part;           // [n_batch][chunks] sums of p there
    int32_t* last_row;        // n_batch (-1: no walk)
    double* last_lam;         // n_batch
    int32_t* keep;
    int32_t* path;
    int32_t* token;
};

template <typename E>
__device__ __forceinline__ float prob_at(const char* row, int x);
template <>
__device__ __forceinline__ float prob_at<float>(const char* row, int x) { return ((const float*)row)[x]; }
template <>
__device__ __forceinline__ float prob_at<uint16_t>(const char* row, int x) {
    return __uint_as_float((uint32_t)((const uint16_t*)row)[x] << 16);
}
// 16 bytes of a row, widened (exactly)
template <typename E>
struct Piece {
    static constexpr int N = 16 / sizeof(E);
    float f[N];
    __device__ __forceinline__ void load(const char* row, int x) {
        // (rows of an odd vocabulary start anywhere: a 16-byte load that asks for no more than E's alignment)
        struct __attribute__((packed, aligned(sizeof(E)))) Any { uint32_t w[4]; };
        const Any r = *(const Any*)(row + (size_t)x * sizeof(E));
        const uint32_t* w = r.w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(E) == 4) {
                f[i] = __uint_as_float(w[i]);
            } else {
                f[2 * i] = __uint_as_float(w[i] << 16);
                f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
};

__device__ __forceinline__ double weight(float p, float q, double lam) {
    const double w = (double)p - lam * (double)q;
    return w > 0.0 ? w : 0.0;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int off = 32; off; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
// sum over the workgroup, in thread 0
__device__ __forceinline__ double block_sum(double x, double* waves) {
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) s += waves[w];
    return s;
}

// sums over a chunk of a row: *w of (p - lam q)+, *all of p
template <typename E, bool BOTH>
__device__ __forceinline__ void chunk_sums(const VerifyParams& a, const char* p, const char* q, double lam, int chunk, double* w, double* all) {
    constexpr int N = Piece<E>::N;
    const int end = min((chunk + 1) * a.chunk, a.n_vocab);
    double sw = 0.0, sp = 0.0;
    for (int x = chunk * a.chunk + threadIdx.x * N; x < end; x += kThreads * N) {
        if (x + N <= end) {
            Piece<E> pp, qq;
            pp.load(p, x);
            qq.load(q, x);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sw += weight(pp.f[i], qq.f[i], lam);
                if (BOTH) sp += (double)pp.f[i];
            }
        } else {
            for (int y = x; y < end; ++y) {
                const float pv = prob_at<E>(p, y);
                sw += weight(pv, prob_at<E>(q, y), lam);
                if (BOTH) sp += (double)pv;
            }
        }
    }
    *w = sw;
    *all = sp;
}

// G_j (j >= 1) of a row: its chunks' sums, added by one thread in order
__device__ __forceinline__ double g_of(const VerifyParams& a, int j, int row) {
    const double* part = a.g_part + ((size_t)(j - 1) * a.b.n_rows + row) * a.chunks;
    double s = 0.0;
    for (int c = 0; c < a.chunks; ++c) s += part[c];
    return s;
}

// ---- G_round of every node with more than `round` children: grid (chunks, nodes, entries) ----------
template <typename E>
__global__ void __launch_bounds__(kThreads) verify_sums_kernel(const VerifyParams a) {
    __shared__ double s_waves[kThreads / 64];
    __shared__ double s_lam;
    const EntryRows er = entry_rows(a.b, blockIdx.z);
    const int t = blockIdx.y;
    if (t >= er.rows) return;
    const int lane = threadIdx.x & 63;
    // (every wavefront counts for itself)
    const int parent = lane < er.rows && lane > t ? a.parents[er.first + lane] : -1;
    if (__popcll(__ballot(parent == t)) <= a.round) return;
    const int row = er.first + t;
    if (threadIdx.x == 0) {
        double lam = 1.0;
        for (int j = 1; j < a.round; ++j) lam += g_of(a, j, row);
        s_lam = lam;
    }
    __syncthreads();
    double w, all;
    chunk_sums<E, false>(a, a.p + row * a.p_stride, a.q + row * a.q_stride, s_lam, blockIdx.x, &w, &all);
    w = block_sum(w, s_waves);
    if (threadIdx.x == 0) a.g_part[((size_t)(a.round - 1) * a.b.n_rows + row) * a.chunks + blockIdx.x] = w;
}

// ---- the walk, and the sums over the row where it ends: grid (chunks, entries) ------------------------
template <typename E>
__global__ void __launch_bounds__(kThreads) verify_walk_kernel(const VerifyParams a) {
    __shared__ double s_waves[kThreads / 64];
    __shared__ int s_row;
    __shared__ double s_lam;
    const int e = blockIdx.y;
    const EntryRows er = entry_rows(a.b, e);
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {
        const bool is = lane < er.rows;
        const int row = er.first + lane;
        const int parent = is ? a.parents[row] : -2;
        const bool child = parent >= 0 && parent < lane;
        int order = 0;                                // earlier children of the same node
        const int of = child ? parent : -3;
        for (int s = 0; s < er.rows; ++s) {
            const int other = __shfl(of, s);          // (every lane takes part)
            order += s < lane && other == of;
        }
        bool taken = false;
        if (child && order < a.max_kids) {
            const int x = a.tokens[row], up = er.first + parent;
            if ((unsigned)x < (unsigned)a.n_vocab) {
                const float pv = prob_at<E>(a.p + up * a.p_stride, x), qv = prob_at<E>(a.q + up * a.q_stride, x);
                double lam = 0.0, G = 1.0;
                for (int j = 0; j < order; ++j) {
                    lam += G;
                    G = g_of(a, j + 1, up);
                }
                taken = (double)a.u[row] * (double)qv * G < weight(pv, qv, lam);
            }
        }
        const uint64_t take = __ballot(taken);
        int node = -1, kept = 0, at_path = -1;        // lane i keeps the walk's i-th node
        if (er.rows > 0 && __shfl(parent, 0) == -1) {
            node = 0;
            for (;;) {
                if (lane == kept) at_path = node;
                ++kept;
                const uint64_t next = __ballot(child && parent == node) & take;
                if (!next) break;
                node = __ffsll((unsigned long long)next) - 1;   // (children lie behind their parent: this ends)
            }
        }
        if (blockIdx.x == 0) {
            if (is) a.path[row] = at_path;
            if (lane == 0) a.keep[e] = kept;
        }
        const int kids = min(__popcll(__ballot(child && parent == node)), a.max_kids);
        if (lane == 0) {
            double lam = 0.0;
            if (node >= 0)
                for (int j = 0; j < kids; ++j) lam += j ? g_of(a, j, er.first + node) : 1.0;
            s_row = node < 0 ? -1 : er.first + node;
            s_lam = lam;
            if (blockIdx.x == 0) {
                a.last_row[e] = s_row;
                a.last_lam[e] = lam;
            }
        }
    }
    __syncthreads();
    const int row = s_row;
    if (row < 0) return;
    double w, all;
    chunk_sums<E, true>(a, a.p + row * a.p_stride, a.q + row * a.q_stride, s_lam, blockIdx.x, &w, &all);
    w = block_sum(w, s_waves);
    all = block_sum(all, s_waves);
    if (threadIdx.x == 0) {
        a.w_part[(size_t)e * a.chunks + blockIdx.x] = w;
        a.p_part[(size_t)e * a.chunks + blockIdx.x] = all;
    }
}

// ---- the draw: one workgroup per entry -------------------------------------------------------------
// The chunk in which the running sum passes u * sum, then the entry within it.
template <typename E>
__global__ void __launch_bounds__(kThreads) verify_draw_kernel(const VerifyParams a) {
    __shared__ double s_waves[kThreads / 64];
    __shared__ double s_target, s_lam;
    __shared__ int s_chunk, s_found, s_lastpos;
    const int e = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = a.last_row[e];
    if (row < 0) {
        if (tid == 0) a.token[e] = -1;
        return;
    }
    if (tid < 64) {
        // running sums over the chunks, lane c up to chunk c
        auto running = [&](const double* part) {
            double x = lane < a.chunks ? part[(size_t)e * a.chunks + lane] : 0.0;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const double y = __shfl_up(x, off);
                if (lane >= off) x += y;
            }
            return x;
        };
        double lam = a.last_lam[e];
        double upto = running(a.w_part);
        double total = __shfl(upto, 63);
        if (!(total > 0.0)) {                         // p == q everywhere: the target itself
            lam = 0.0;
            upto = running(a.p_part);
            total = __shfl(upto, 63);
        }
        const double target = (double)a.u_sample[e] * total;
        const double left = __shfl_up(upto, 1);
        const double before = lane ? left : 0.0;
        const uint64_t past = __ballot(upto > target);
        const uint64_t some = __ballot(upto > before);
        // (rounding may leave no chunk past the target: then the last one that holds anything)
        const int at = past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : -1;
        const double skip = __shfl(before, at < 0 ? 0 : at);
        if (lane == 0) {
            s_chunk = total > 0.0 ? at : -1;
            s_target = target - skip;
            s_lam = lam;
            s_found = 0x7fffffff;
            s_lastpos = -1;
        }
    }
    __syncthreads();
    const int c = s_chunk;
    if (c < 0) {
        if (tid == 0) a.token[e] = -1;
        return;
    }
    const char* p = a.p + row * a.p_stride;
    const char* q = a.q + row * a.q_stride;
    const double lam = s_lam, target = s_target;
    constexpr int N = Piece<E>::N;
    const int end = min((c + 1) * a.chunk, a.n_vocab);
    double before = 0.0;                              // sum of the chunk's earlier tiles
    for (int x0 = c * a.chunk; x0 < end; x0 += kThreads * N) {
        const int x = x0 + tid * N;
        double w[N], mine = 0.0;
        float pf[N], qf[N];
        if (x + N <= end) {
            Piece<E> pp, qq;
            pp.load(p, x);
            qq.load(q, x);
#pragma unroll
            for (int i = 0; i < N; ++i) { pf[i] = pp.f[i]; qf[i] = qq.f[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                pf[i] = x + i < end ? prob_at<E>(p, x + i) : 0.f;
                qf[i] = x + i < end ? prob_at<E>(q, x + i) : 0.f;
            }
        }
        int lastpos = -1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w[i] = weight(pf[i], qf[i], lam);
            mine += w[i];
            if (w[i] > 0.0) lastpos = x + i;
        }
        double upto = mine;                           // inclusive running sum over the threads
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const double y = __shfl_up(upto, off);
            if (lane >= off) upto += y;
        }
        __syncthreads();
        if (lane == 63) s_waves[wave] = upto;
        __syncthreads();
        double ahead = before, tile = 0.0;
        for (int v = 0; v < kThreads / 64; ++v) {
            if (v < wave) ahead += s_waves[v];
            tile += s_waves[v];
        }
        double run = ahead + (upto - mine);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            run += w[i];
            if (w[i] > 0.0 && run > target) {
                atomicMin(&s_found, x + i);
                break;
            }
        }
        if (lastpos >= 0) atomicMax(&s_lastpos, lastpos);
        before += tile;
        __syncthreads();
        if (s_found != 0x7fffffff) break;
    }
    if (tid == 0) a.token[e] = s_found != 0x7fffffff ? s_found : s_lastpos;
}

struct VerifyPlan {
    int chunk, chunks, rounds;
    size_t off_g, off_w, off_p, off_lam, off_row, total;
};
VerifyPlan plan_verify(const dip_batch* b, int n_vocab, int max_kids) {
    VerifyPlan pl;
    int chunk = (n_vocab + kMaxChunks - 1) / kMaxChunks;
    if (chunk < kMinChunk) chunk = kMinChunk;
    pl.chunk = (chunk + 7) / 8 * 8;
    pl.chunks = (n_vocab + pl.chunk - 1) / pl.chunk;
    const int widest = rows_bound(b) - 1;             // children that one node can have
    pl.rounds = (max_kids < widest ? max_kids : widest) - 1;
    if (pl.rounds < 0) pl.rounds = 0;
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    pl.off_g = take(sizeof(double) * pl.rounds * b->n_rows * pl.chunks);
    pl.off_w = take(sizeof(double) * b->n_batch * pl.chunks);
    pl.off_p = take(sizeof(double) * b->n_batch * pl.chunks);
    pl.off_lam = take(sizeof(double) * b->n_batch);
    pl.off_row = take(sizeof(int32_t) * b->n_batch);
    pl.total = o;
    return pl;
}
int32_t check_verify(const dip_batch* b, int n_vocab, int max_kids) {
    int32_t st = validate_batch(b, false);
    if (st) return st;
    if (rows_bound(b) > DIP_MAX_TREE) return fail(DIP_ERR_UNSUPPORTED, "a tree has at most %d nodes", DIP_MAX_TREE);
    if (n_vocab < 1) return fail(DIP_ERR_INVALID_ARG, "n_vocab must be >= 1");
    if (n_vocab > 1 << 24) return fail(DIP_ERR_UNSUPPORTED, "n_vocab must be at most 2^24");
    if (max_kids < 1 || max_kids >= DIP_MAX_TREE) return fail(DIP_ERR_INVALID_ARG, "max_kids must be in [1, %d]", DIP_MAX_TREE - 1);
    return DIP_OK;
}

template <typename E>
int32_t launch_verify(VerifyParams& a, const VerifyPlan& pl, hipStream_t stream) {
    for (int j = 1; j <= pl.rounds; ++j) {
        a.round = j;
        const int32_t st = check_hip(launch_timed(verify_sums_kernel<E>, dim3(pl.chunks, a.b.max_rows, a.b.n_batch), dim3(kThreads), stream,
                                                  DIP_KERNEL_VERIFY, a), "verify_sums launch");
        if (st) return st;
    }
    const int32_t st = check_hip(launch_timed(verify_walk_kernel<E>, dim3(pl.chunks, a.b.n_batch), dim3(kThreads), stream,
                                              DIP_KERNEL_VERIFY, a), "verify_walk launch");
    if (st) return st;
    return check_hip(launch_timed(verify_draw_kernel<E>, dim3(a.b.n_batch), dim3(kThreads), stream, DIP_KERNEL_VERIFY, a),
                     "verify_draw launch");
}

}  // namespace
}  // namespace dip

using namespace dip;

extern "C" {

size_t dip_verify_tree_workspace_bytes(const dip_batch* batch, int32_t n_vocab, int32_t max_kids) {
    if (check_verify(batch, n_vocab, max_kids)) return 0;
    return plan_verify(batch, n_vocab, max_kids).total;
}

int32_t dip_verify_tree(const dip_batch* batch, const int32_t* tokens, const int32_t* parents, const void* p, int64_t p_stride,
                        const void* q, int64_t q_stride, int32_t dtype, int32_t n_vocab, const float* u, const float* u_sample,
                        int32_t max_kids, int32_t* keep, int32_t* path, int32_t* token, void* ws, size_t ws_bytes, void* stream) {
    int32_t st = check_verify(batch, n_vocab, max_kids);
    if (st) return st;
    if (!tokens || !parents || !p || !q || !u || !u_sample || !keep || !path || !token)
        return fail(DIP_ERR_INVALID_ARG, "verify_tree: null pointer");
    if (dtype != DIP_F32 && dtype != DIP_BF16) return fail(DIP_ERR_UNSUPPORTED, "verify_tree: dtype %d", dtype);
    const int es = elem_bytes(dtype);
    if (p_stride < n_vocab || q_stride < n_vocab) return fail(DIP_ERR_INVALID_ARG, "verify_tree: strides smaller than a row");
    if (reinterpret_cast<uintptr_t>(p) % es || reinterpret_cast<uintptr_t>(q) % es)
        return fail(DIP_ERR_UNSUPPORTED, "verify_tree: p and q must be aligned to their elements");
    const VerifyPlan pl = plan_verify(batch, n_vocab, max_kids);
    st = validate_ws(ws, ws_bytes, pl.total);
    if (st) return st;
    char* base = (char*)ws;
    VerifyParams a;
    a.b = view_of(batch);
    a.tokens = tokens;
    a.parents = parents;
    a.p = (const char*)p;
    a.q = (const char*)q;
    a.p_stride = p_stride * es;
    a.q_stride = q_stride * es;
    a.n_vocab = n_vocab;
    a.chunk = pl.chunk;
    a.chunks = pl.chunks;
    a.u = u;
    a.u_sample = u_sample;
    a.max_kids = max_kids;
    a.round = 0;
    a.g_part = (double*)(base + pl.off_g);
    a.w_part = (double*)(base + pl.off_w);
    a.p_part = (double*)(base + pl.off_p);
    a.last_row = (int32_t*)(base + pl.off_row);
    a.last_lam = (double*)(base + pl.off_lam);
    a.keep = keep;
    a.path = path;
    a.token = token;
    return dtype == DIP_F32 ? launch_verify<float>(a, pl, (hipStream_t)stream) : launch_verify<uint16_t>(a, pl, (hipStream_t)stream);
}

}  // extern "C"
