// Verification of drafted trees against the target's probabilities (dip_verify_tree).
//
// The usual rule tries the children of a node in turn and replaces the target r by norm((r - q)+)
// after each refusal.  Written without the norms, the j-th r is (p - lam_j q)+ / G_j with
// lam_0 = 0, G_0 = 1, lam_{j+1} = lam_j + G_j and G_j the sum of (p - lam_j q)+: for a node that
// was refused j children everything about its rows is in the numbers lam_j and G_j, and a child's test
// needs two probabilities and these.  So the walk itself is a few loads, done by every workgroup for itself,
// and the passes over whole rows are plain sums that split over any number of workgroups: G_1 .. G_{m-1} of the
// nodes with several children (one launch each: lam_{j+1} needs G_j; only nodes that the walk can still
// reach and whose first j children are refused), then the sum over the row at which the walk ends, whose last
// workgroup to finish draws the token.
// Sums and comparisons are in fp64: the outputs are decisions, and with sums that are 1e-16 off in
// whatever order they are taken, all orders decide alike (an fp32 sum of 128000 terms leaves 1 in 10^5
// draws open).  fp64 adds at half the fp32 rate cost nothing here: the kernels wait for memory.
//
// What bounds it: the walk is four dependent loads (rows, tree, probabilities, sums) and so is the draw, about
// 12 us with the launch before any row is read; 64 trees of 16 nodes at 128256 words read 66 MB for the
// last row and about as much for the refused children.  Measured: one chain of 5 at 32064 words 12 us, 16 trees
// of 8 nodes (bf16, 128256 words) 23 us, 64 of 16 (fp32) 39 us.

#include "dip_vocab_device.h"

namespace dip {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxChunks = 64;            // of a row; a lane of one wavefront sums each
constexpr int kMinChunk = kThreads * kPer;

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
    uint64_t* tickets;        // a word per entry
    uint64_t epoch;
    int32_t* keep;
    int32_t* path;
    int32_t* token;
};

__device__ __forceinline__ double weight(float p, float q, double lam) {
    const double w = (double)p - lam * (double)q;
    return w > 0.0 ? w : 0.0;
}

// a thread's part of the sums over a chunk of a row: *w of (p - lam q)+, *all of p
template <typename E>
__device__ __forceinline__ void chunk_sums(const VerifyParams& a, int row, double lam, int chunk, double* w, double* all) {
    const char* p = a.p + row * a.p_stride;
    const char* q = a.q + row * a.q_stride;
    const int end = min((chunk + 1) * a.chunk, a.n_vocab);
    double sw = 0.0, sp = 0.0;
    for (int x = chunk * a.chunk + threadIdx.x * kPer; x < end; x += kThreads * kPer) {
        float pf[kPer], qf[kPer];
        load_entries<E>(p, x, end, pf);
        load_entries<E>(q, x, end, qf);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            sw += weight(pf[i], qf[i], lam);
            sp += (double)pf[i];
        }
    }
    *w = sw;
    *all = sp;
}

// One wavefront, lane t for node t: which children are taken, as far as G_1 .. G_{known} say.
struct Walk {
    uint64_t kids;            // this node's children
    uint64_t refused;         // nodes tried and refused ...
    uint64_t taken;           // ... and taken, where every earlier sibling was refused
    double next;              // lam_{j+1} of its parent, this node being child j <= known
    bool reached;             // this node stands, or may do so once more is known
};
template <typename E>
__device__ __forceinline__ Walk walk(const VerifyParams& a, const EntryRows& er, int known) {
    const int lane = threadIdx.x & 63, row = er.first + lane;
    const bool is = lane < er.rows;
    const int parent = is ? a.parents[row] : -2;
    const int x = is ? a.tokens[row] : -1;
    const double u = is ? (double)a.u[row] : 0.0;
    const bool child = parent >= 0 && parent < lane;
    const int of = child ? parent : -3, up = er.first + (child ? parent : 0);
    const bool fits = child && (unsigned)x < (unsigned)a.n_vocab;
    float pv = 0.f, qv = 0.f;
    if (fits) {
        pv = entry_at<E>(a.p + up * a.p_stride, x);
        qv = entry_at<E>(a.q + up * a.q_stride, x);
    }
    Walk w;
    uint64_t earlier = 0;                             // siblings before this node
    w.kids = 0;
    for (int s = 0; s < er.rows; ++s) {
        const int other = __builtin_amdgcn_readlane(of, s);
        if (other == of && s < lane) earlier |= 1ull << s;
        if (other == lane) w.kids |= 1ull << s;
    }
    const int order = child ? __popcll(earlier) : -1;
    // G_j for every child j >= 1: a lane adds the chunks of its parent's row, 16 on their way at a time
    double G = 1.0, lam = 0.0;
    if (order >= 1 && order <= known && order < a.max_kids) {
        constexpr int FLIGHT = 16;
        const double* part = a.g_part + ((size_t)(order - 1) * a.b.n_rows + up) * a.chunks;
        G = 0.0;
        for (int c = 0; c < a.chunks; c += FLIGHT) {
            double x[FLIGHT];
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f) x[f] = part[min(c + f, a.chunks - 1)];
#pragma unroll
            for (int f = 0; f < FLIGHT; ++f) G += c + f < a.chunks ? x[f] : 0.0;
        }
    }
    w.next = 1.0;
    w.refused = w.taken = 0;
    const int elder = earlier ? 63 - __clzll((long long)earlier) : lane;
    uint64_t open = 0;                                // children whose test is not known yet
    for (int k = 0; k < a.max_kids; ++k) {
        const bool mine = order == k && (earlier & ~(w.refused | open)) == 0;
        if (!__any(mine)) break;
        if (k > known) {
            open |= __ballot(mine);
            continue;
        }
        const double upto = __shfl(w.next, elder);
        if (k > 0 && order == k) {
            lam = upto;
            w.next = upto + G;
        }
        const bool take = mine && fits && u * (double)qv * G < weight(pv, qv, lam);
        w.taken |= __ballot(mine && take);
        w.refused |= __ballot(mine && !take);
    }
    // a node is reached if it and all its ancestors up to node 0 are: pointers jump 1, 2, 4 .. steps up
    bool all = ((w.taken | open) >> lane) & 1;
    int at = child ? parent : -2;
    if (lane == 0 && parent == -1) {
        all = true;
        at = -1;
    }
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        const int from = at < 0 ? lane : at;
        const bool theirs = __shfl((int)all, from);
        const int next = __shfl(at, from);
        if (at >= 0) {
            all = all && theirs;
            at = next;
        }
    }
    w.reached = all && at == -1;
    return w;
}

// ---- G_round of the nodes that can be reached and have refused `round` children, with more to come: grid
// (chunks, entries) -------------------------------------------------------------------------------------
template <typename E>
__global__ void __launch_bounds__(kThreads) verify_sums_kernel(const VerifyParams a) {
    __shared__ double s_waves[kThreads / 64];
    __shared__ uint64_t s_nodes;
    __shared__ double s_lam[64];
    const EntryRows er = entry_rows(a.b, blockIdx.y);
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {
        const Walk w = walk<E>(a, er, a.round - 1);
        const bool need = w.reached && __popcll(w.kids) > a.round && __popcll(w.kids & w.refused) == a.round;
        const uint64_t nodes = __ballot(need), tried = w.kids & w.refused;
        s_lam[lane] = __shfl(w.next, tried ? 63 - __clzll((long long)tried) : lane);
        if (lane == 0) s_nodes = nodes;
    }
    __syncthreads();
    for (uint64_t left = s_nodes; left; left &= left - 1) {
        const int t = __ffsll((unsigned long long)left) - 1;
        double w, all;
        chunk_sums<E>(a, er.first + t, s_lam[t], blockIdx.x, &w, &all);
        w = block_sum(w, s_waves);
        if (threadIdx.x == 0) a.g_part[((size_t)(a.round - 1) * a.b.n_rows + er.first + t) * a.chunks + blockIdx.x] = w;
    }
}

// ---- the walk, the sums over the row where it ends, and the draw: grid (chunks, entries) ------------------
template <typename E>
__global__ void __launch_bounds__(kThreads) verify_walk_kernel(const VerifyParams a) {
    __shared__ double s_waves[kThreads / 64];
    __shared__ double s_lam, s_target;
    __shared__ int s_row, s_chunk, s_found, s_lastpos;
    const double u_sample = (double)a.u_sample[blockIdx.y];
    const int e = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const EntryRows er = entry_rows(a.b, e);
    uint64_t* ticket = a.tickets + (size_t)e * kTicketStride;
    if (tid < 64) {
        const Walk w = walk<E>(a, er, a.max_kids);
        if (lane == 0) ticket_open(ticket, a.epoch);  // (behind the walk's loads, which return in order)
        const uint64_t path = __ballot(w.reached);
        const int kept = __popcll(path), last = path ? 63 - __clzll((long long)path) : 0;
        if (blockIdx.x == 0) {
            if (w.reached) a.path[er.first + __popcll(path & ((1ull << lane) - 1))] = lane;
            if (lane >= kept && lane < er.rows) a.path[er.first + lane] = -1;
            if (lane == 0) a.keep[e] = kept;
        }
        // all children of the last node (up to max_kids) were tried and refused
        const uint64_t tried = w.kids & w.refused;
        const double upto = __shfl(w.next, tried ? 63 - __clzll((long long)tried) : lane);
        const double lam = of_lane(tried ? upto : 0.0, last);
        if (lane == 0) {
            s_row = kept ? er.first + last : -1;
            s_lam = lam;
            s_found = 0x7fffffff;
            s_lastpos = -1;
        }
    }
    __syncthreads();
    const int row = s_row;
    if (row < 0) {
        if (blockIdx.x == 0 && tid == 0) a.token[e] = -1;
        return;
    }
    double w, all;
    chunk_sums<E>(a, row, s_lam, blockIdx.x, &w, &all);
    w = block_sum(w, s_waves);
    all = block_sum(all, s_waves);
    double* w_part = a.w_part + (size_t)e * a.chunks;
    double* p_part = a.p_part + (size_t)e * a.chunks;
    if (tid == 0) {
        put(w_part + blockIdx.x, w);
        put(p_part + blockIdx.x, all);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        s_chunk = ticket_last(ticket, a.epoch, a.chunks);
    }
    __syncthreads();
    if (!s_chunk) return;

    // the draw: the chunk in which the running sum passes u * sum, then the entry within it
    __syncthreads();
    if (tid < 64) {
        // running sums over the chunks, lane c up to chunk c
        auto up_to = [&](const double* part) { return running(lane < a.chunks ? get(part + lane) : 0.0); };
        double lam = s_lam;
        double upto = up_to(w_part);
        double total = of_lane(upto, 63);
        if (!(total > 0.0)) {                         // p == q everywhere: the target itself
            lam = 0.0;
            upto = up_to(p_part);
            total = of_lane(upto, 63);
        }
        const double target = u_sample * total;
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
    const int end = min((c + 1) * a.chunk, a.n_vocab);
    double before = 0.0;                              // sum of the chunk's earlier tiles
    for (int x0 = c * a.chunk; x0 < end; x0 += kThreads * kPer) {
        const int x = x0 + tid * kPer;
        float pf[kPer], qf[kPer];
        load_entries<E>(p, x, end, pf);
        load_entries<E>(q, x, end, qf);
        double mine = 0.0;
        int lastpos = -1;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const double y = weight(pf[i], qf[i], lam);
            mine += y;
            if (y > 0.0) lastpos = x + i;
        }
        const double upto = running(mine);
        __syncthreads();
        if (lane == 63) s_waves[wave] = upto;
        __syncthreads();
        double ahead = before, tile = 0.0;
        for (int v = 0; v < kThreads / 64; ++v) {
            if (v < wave) ahead += s_waves[v];
            tile += s_waves[v];
        }
        double run = ahead + (upto - mine);
        int found = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const double y = weight(pf[i], qf[i], lam);
            run += y;
            if (y > 0.0 && run > target) found = min(found, x + i);
        }
        if (found != 0x7fffffff) atomicMin(&s_found, found);
        if (lastpos >= 0) atomicMax(&s_lastpos, lastpos);
        before += tile;
        __syncthreads();
        if (s_found != 0x7fffffff) break;
    }
    if (tid == 0) a.token[e] = s_found != 0x7fffffff ? s_found : s_lastpos;
}

struct VerifyPlan {
    int chunk, chunks, rounds;
    size_t off_g, off_w, off_p, off_tickets, total;
};
VerifyPlan plan_verify(const dip_batch* b, int n_vocab, int max_kids) {
    VerifyPlan pl;
    int chunk = (n_vocab + kMaxChunks - 1) / kMaxChunks;
    if (chunk < kMinChunk) chunk = kMinChunk;
    // twice as much to a workgroup where there are more than the chip holds at a time: every one walks the tree
    // (64 entries of 128256: 41 us; with 4096 to a workgroup 46, with 16384 and half the workgroups 50)
    if (chunk == kMinChunk && (int64_t)b->n_batch * ((n_vocab + chunk - 1) / chunk) > 1024) chunk *= 2;
    pl.chunk = (chunk + kPer - 1) / kPer * kPer;
    pl.chunks = (n_vocab + pl.chunk - 1) / pl.chunk;
    const int widest = rows_bound(b) - 1;             // children that one node can have
    pl.rounds = (max_kids < widest ? max_kids : widest) - 1;
    if (pl.rounds < 0) pl.rounds = 0;
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    pl.off_g = take(sizeof(double) * pl.rounds * b->n_rows * pl.chunks);
    pl.off_w = take(sizeof(double) * b->n_batch * pl.chunks);
    pl.off_p = take(sizeof(double) * b->n_batch * pl.chunks);
    pl.off_tickets = take(sizeof(uint64_t) * kTicketStride * b->n_batch);
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
        const int32_t st = check_hip(launch_timed(verify_sums_kernel<E>, dim3(pl.chunks, a.b.n_batch), dim3(kThreads), stream,
                                                  DIP_KERNEL_VERIFY, a), "verify_sums launch");
        if (st) return st;
    }
    a.epoch = next_epoch();
    return check_hip(launch_timed(verify_walk_kernel<E>, dim3(pl.chunks, a.b.n_batch), dim3(kThreads), stream, DIP_KERNEL_VERIFY, a),
                     "verify_walk launch");
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
    a.tickets = (uint64_t*)(base + pl.off_tickets);
    a.epoch = 0;
    a.keep = keep;
    a.path = path;
    a.token = token;
    return dtype == DIP_F32 ? launch_verify<float>(a, pl, (hipStream_t)stream) : launch_verify<uint16_t>(a, pl, (hipStream_t)stream);
}

}  // extern "C"
