// Pages of a key/value cache: init, free, fork, reserve with copy on write, append, compact.
// The pool's whole state is page_refs (how many table entries name a page): a free page is one
// that nobody names, and the lowest ones are given out first, so that which page goes where
// follows from the tables alone -- no list whose order would depend on the order of atomics.
// Counts are changed with integer atomics, whose order does not show in the result.
// Rows are written and committed only where all of an entry's rows have pages that no other sequence holds: that is
// what reserve leaves an entry with, or else it grants it nothing (lacks_room).
//
// A decode step is reserve (two launches), append, compact (two): all wait for memory.  A few drafts of a few
// branches are bound by the launches themselves (2 to 8 us each; six branches of 8 rows, 32 layers: 35 us with
// fork and free, 7 launches); 16 branches of up to 256 rows, 40 layers, 10 heads of 128, by bytes: append 225 us,
// move 125, copy on write 48 of 421 us, against 383 us for the bytes at the rate of a plain copy (4.83 TB/s).

#include "dip_decode_internal.h"

namespace dip {

// ---- argument checks ----------------------------------------------------------------------
int32_t validate_kv(const dip_kv_cache* c) {
    if (!c) return fail(DIP_ERR_INVALID_ARG, "cache: null descriptor");
    if (!c->k || !c->v || !c->page_table || !c->seq_len || !c->page_refs)
        return fail(DIP_ERR_INVALID_ARG, "cache: null pointer");
    if (c->dtype != DIP_F32 && c->dtype != DIP_BF16)
        return fail(DIP_ERR_UNSUPPORTED, "cache: dtype %d is neither DIP_F32 nor DIP_BF16", c->dtype);
    if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->n_seqs < 1 || c->max_pages < 1)
        return fail(DIP_ERR_INVALID_ARG, "cache: sizes must be >= 1");
    if (c->page_size < 1 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
        return fail(DIP_ERR_UNSUPPORTED, "cache: page_size must be a power of two in [1, 4096], got %d", c->page_size);
    // (a length and the rows on top of it, at most 2^24, then fit 32 bits)
    if ((int64_t)c->max_pages * c->page_size > ((int64_t)1 << 31) - (1 << 25))
        return fail(DIP_ERR_UNSUPPORTED, "cache: max_pages * page_size must be at most 2^31 - 2^25");
    const int per = 16 / elem_bytes(c->dtype);
    if (c->head_dim % per) return fail(DIP_ERR_UNSUPPORTED, "cache: head_dim must be a multiple of %d", per);
    if (c->head_dim > 65536 || c->n_kv_heads > 65535 || c->n_layers > 32767)
        return fail(DIP_ERR_UNSUPPORTED, "cache: more than 65536 dims, 65535 heads or 32767 layers");
    const int64_t strides[4] = {c->layer_stride, c->page_stride, c->head_stride, c->slot_stride};
    for (int64_t s : strides)
        if (s % per) return fail(DIP_ERR_UNSUPPORTED, "cache: strides must be multiples of 16 bytes");
    if (c->slot_stride < c->head_dim || c->head_stride < c->head_dim || c->page_stride < c->head_dim ||
        (c->n_layers > 1 && c->layer_stride < c->head_dim))
        return fail(DIP_ERR_INVALID_ARG, "cache: strides smaller than a head");
    if (!aligned16(c->k) || !aligned16(c->v)) return fail(DIP_ERR_UNSUPPORTED, "cache: k and v must be 16-byte aligned");
    return DIP_OK;
}

int32_t validate_batch(const dip_batch* b, bool need_seqs) {
    if (!b) return fail(DIP_ERR_INVALID_ARG, "batch: null descriptor");
    if (!b->row_start || (need_seqs && !b->seqs)) return fail(DIP_ERR_INVALID_ARG, "batch: null pointer");
    if (b->n_batch < 1 || b->n_batch > DIP_MAX_BATCH)
        return fail(DIP_ERR_UNSUPPORTED, "batch: n_batch must be in [1, %d], got %d", DIP_MAX_BATCH, b->n_batch);
    if (b->n_rows < 1 || b->max_rows < 1) return fail(DIP_ERR_INVALID_ARG, "batch: n_rows and max_rows must be >= 1");
    if (b->n_rows >= 1 << 24) return fail(DIP_ERR_UNSUPPORTED, "batch: n_rows must be below 2^24");
    if (b->max_len < 0) return fail(DIP_ERR_INVALID_ARG, "batch: max_len must be >= 0");
    return DIP_OK;
}

int32_t validate_ws(const void* ws, size_t have, size_t need) {
    if (!ws || have < need) return fail(DIP_ERR_WORKSPACE, "workspace: %zu bytes needed, %zu given", need, ws ? have : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(DIP_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    return DIP_OK;
}

KvView view_of(const dip_kv_cache* c) {
    const int per = 16 / elem_bytes(c->dtype);
    KvView v;
    v.k = (char*)c->k;
    v.v = (char*)c->v;
    v.table = c->page_table;
    v.seq_len = c->seq_len;
    v.refs = c->page_refs;
    v.n_pages = c->n_pages;
    v.n_seqs = c->n_seqs;
    v.max_pages = c->max_pages;
    v.n_layers = c->n_layers;
    v.n_heads = c->n_kv_heads;
    v.page_shift = log2_of(c->page_size);
    v.pieces = c->head_dim / per;
    v.layer_stride = c->layer_stride / per;
    v.page_stride = c->page_stride / per;
    v.head_stride = c->head_stride / per;
    v.slot_stride = c->slot_stride / per;
    return v;
}

namespace {

constexpr int kThreads = 256;
typedef unsigned int piece_t __attribute__((ext_vector_type(4)));   // 16 bytes

__device__ __forceinline__ bool is_page(const KvView& c, int p) { return (unsigned)p < (unsigned)c.n_pages; }

// ---- init, free, fork ---------------------------------------------------------------------
struct InitParams {
    KvView c;
};
__global__ void __launch_bounds__(kThreads) kv_init_kernel(const InitParams p) {
    const int64_t entries = (int64_t)p.c.n_seqs * p.c.max_pages;
    const int64_t step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < entries; i += step) p.c.table[i] = -1;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < p.c.n_pages; i += step) p.c.refs[i] = 0;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < p.c.n_seqs; i += step) p.c.seq_len[i] = 0;
}

struct SeqsParams {
    KvView c;
    const int32_t* a;         // sequences to free, or sources
    const int32_t* b;         // destinations
};
// (an entry is taken out by exchange, so that a sequence that is listed twice gives a page up once)
__device__ __forceinline__ void give_up(const KvView& c, int32_t* entry) {
    if (*entry == -1) return;
    const int old = atomicExch(entry, -1);
    if (is_page(c, old)) atomicSub(&c.refs[old], 1);
}
__global__ void __launch_bounds__(kThreads) kv_free_kernel(const SeqsParams p) {
    const int seq = p.a[blockIdx.x];
    if ((unsigned)seq >= (unsigned)p.c.n_seqs) return;
    int32_t* row = p.c.table + (size_t)seq * p.c.max_pages;
    for (int j = threadIdx.x; j < p.c.max_pages; j += kThreads) give_up(p.c, row + j);
    if (threadIdx.x == 0) p.c.seq_len[seq] = 0;
}
__global__ void __launch_bounds__(kThreads) kv_fork_kernel(const SeqsParams p) {
    const int src = p.a[blockIdx.x], dst = p.b[blockIdx.x];
    if ((unsigned)src >= (unsigned)p.c.n_seqs || (unsigned)dst >= (unsigned)p.c.n_seqs || src == dst) return;
    const int len = entry_len(p.c, src);
    const int held = (len + (1 << p.c.page_shift) - 1) >> p.c.page_shift;
    const int32_t* from = p.c.table + (size_t)src * p.c.max_pages;
    int32_t* to = p.c.table + (size_t)dst * p.c.max_pages;
    for (int j = threadIdx.x; j < p.c.max_pages; j += kThreads) {
        const int page = j < held ? from[j] : -1;
        to[j] = page;
        if (is_page(p.c, page)) atomicAdd(&p.c.refs[page], 1);
    }
    if (threadIdx.x == 0) p.c.seq_len[dst] = len;
}

// ---- reserve ------------------------------------------------------------------------------
// One workgroup: the lowest free pages go to the wanted table entries in order, which is a prefix
// sum over both.  Bound by latency (a handful of round trips to memory: 7 us), not by its bytes.  One, because
// several would have to agree on the order through memory; 1024 threads look at 4096 counts at a time and stop
// once there are as many free pages as are wanted (about 75 us where the last of 200000 pages are the only
// free ones).
// An "item" is a table entry that some row of the step falls into, entries in order.
constexpr int kReserveThreads = 1024;
struct CopyItem {
    int32_t from, to, slots, pad;  // from < 0: nothing to copy
};
struct ReserveParams {
    KvView c;
    BatchView b;
    int32_t* granted;         // nullable
    uint64_t* wanted;         // one bit per item, 64 to a word
    int32_t* free_pages;      // n_pages
    CopyItem* copies;         // n_batch
};

// inclusive sum over the workgroup; *total the sum of all
__device__ __forceinline__ int scan_add(int x, int* wave_sums, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(x, off);
        if (lane >= off) x += y;
    }
    __syncthreads();          // (the sums of an earlier scan are read)
    if (lane == 63) wave_sums[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kReserveThreads / 64; ++w) {
        const int s = wave_sums[w];
        if (w < wave) before += s;
        all += s;
    }
    *total = all;
    return x + before;
}

__global__ void __launch_bounds__(kReserveThreads) kv_reserve_kernel(const ReserveParams p) {
    __shared__ int s_first[DIP_MAX_BATCH + 1];   // first item of each entry
    __shared__ int s_seq[DIP_MAX_BATCH];
    __shared__ int s_len[DIP_MAX_BATCH];
    __shared__ int s_need[DIP_MAX_BATCH];        // items without a page of their own; later: granted
    __shared__ int s_waves[kReserveThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int page = 1 << p.c.page_shift;

    int items = 0, fits = 0;
    if (tid < p.b.n_batch) {
        const int rows = entry_rows(p.b, tid).rows;
        const int seq = entry_seq(p.b, p.c, tid);
        const int len = seq >= 0 ? entry_len(p.c, seq) : 0;
        // (64 bits: a length at the end of the table and the rows on top of it)
        const int64_t last = ((int64_t)len + rows + page - 1) >> p.c.page_shift;
        fits = seq >= 0 && last <= p.c.max_pages;
        if (fits && rows > 0) items = (int)last - (len >> p.c.page_shift);
        s_seq[tid] = seq;
        s_len[tid] = len;
        s_need[tid] = 0;
        p.copies[tid].from = -1;
    }
    int n_items;
    const int upto = scan_add(items, s_waves, &n_items);
    if (tid < p.b.n_batch) s_first[tid + 1] = upto;
    if (tid == 0) s_first[0] = 0;
    __syncthreads();

    auto entry_of = [&](int item) {              // the entry with s_first[e] <= item < s_first[e + 1]
        int lo = 0, hi = p.b.n_batch;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_first[mid] <= item) lo = mid; else hi = mid;
        }
        return lo;
    };
    auto table_at = [&](int item, int e) {
        return p.c.table + (size_t)s_seq[e] * p.c.max_pages + (s_len[e] >> p.c.page_shift) + (item - s_first[e]);
    };

    // which items want a page; all of them are looked at before any count changes
    for (int base = 0; base < n_items; base += kReserveThreads) {
        const int item = base + tid;
        bool want = false;
        if (item < n_items) {
            const int e = entry_of(item);
            const int held = *table_at(item, e);
            want = !is_page(p.c, held) || p.c.refs[held] > 1;
            if (want) atomicAdd(&s_need[e], 1);
        }
        const uint64_t mask = __ballot(want);
        if (lane == 0 && item < n_items) p.wanted[item >> 6] = mask;
    }
    __syncthreads();
    int n_wanted;
    const int need = tid < p.b.n_batch ? s_need[tid] : 0;
    const int need_upto = scan_add(need, s_waves, &n_wanted);

    // the lowest free pages, as many as are wanted
    int n_free = 0;
    for (int base = 0; base < p.c.n_pages && n_free < n_wanted; base += 4 * kReserveThreads) {
        const int at = base + 4 * tid;
        int is_free[4], mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            is_free[i] = at + i < p.c.n_pages && p.c.refs[at + i] == 0;
            mine += is_free[i];
        }
        int found;
        int rank = n_free + scan_add(mine, s_waves, &found) - mine;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (is_free[i]) p.free_pages[rank++] = at + i;
        n_free += found;
    }

    bool ok = false;
    if (tid < p.b.n_batch) {
        ok = fits && (need == 0 || need_upto <= n_free);
        if (p.granted) p.granted[tid] = ok;
    }
    __syncthreads();
    if (tid < p.b.n_batch) s_need[tid] = ok;
    __syncthreads();

    // hand them out
    const bool refused = n_wanted > n_free;
    int given = 0;
    for (int base = 0; base < n_items; base += kReserveThreads) {
        const int item = base + tid;
        const bool want = item < n_items && ((p.wanted[item >> 6] >> (item & 63)) & 1);
        int found;
        const int rank = given + scan_add(want, s_waves, &found) - 1;
        given += found;
        if (!want) continue;
        const int e = entry_of(item);
        if (!s_need[e]) continue;
        int32_t* entry = table_at(item, e);
        const int old = *entry, fresh = p.free_pages[rank];
        *entry = fresh;
        p.c.refs[fresh] = 1;
        if (is_page(p.c, old)) {
            atomicSub(&p.c.refs[old], 1);
            const int slots = s_len[e] & (page - 1);
            if (item == s_first[e] && slots) p.copies[e] = {old, fresh, slots, 0};
        }
    }

    // Entries that were refused, by wavefront: whoever is left alone with all its pages, the others that held them having
    // taken new ones, has its room too.  (Counts past this compute unit's cache, which may hold them as they were.)
    if (!refused || !p.granted) return;
    __syncthreads();
    for (int e = tid >> 6; e < p.b.n_batch; e += kReserveThreads / 64) {
        const int first = s_first[e], end = s_first[e + 1];
        if (s_need[e] || first == end) continue;
        bool lacks = false;
        for (int item = first + lane; item < end; item += 64) {
            const int held = *table_at(item, e);
            lacks |= !is_page(p.c, held) || __hip_atomic_load(&p.c.refs[held], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) > 1;
        }
        if (!__any(lacks) && lane == 0) p.granted[e] = 1;
    }
}

// What an entry has of a page that it had to exchange, or whole pages: one workgroup per (copy,
// layer, k or v), 16 bytes a thread, four in flight.  In order of address, so that a row of slots or of heads is
// one run whichever of the two strides is the small one.  16 tails of a 64-slot page, 40 layers: 47 us.
struct CopyParams {
    KvView c;
    const CopyItem* copies;   // or, when null, whole pages src -> dst
    const int32_t* src;
    const int32_t* dst;
};
__global__ void __launch_bounds__(kThreads) kv_copy_kernel(const CopyParams p) {
    int from, to, slots;
    if (p.copies) {
        const CopyItem it = p.copies[blockIdx.x];
        from = it.from; to = it.to; slots = it.slots;
        if (from < 0) return;
    } else {
        from = p.src[blockIdx.x]; to = p.dst[blockIdx.x]; slots = 1 << p.c.page_shift;
        if (!is_page(p.c, from) || !is_page(p.c, to) || from == to) return;
    }
    piece_t* base = (piece_t*)(blockIdx.z ? p.c.v : p.c.k) + (int64_t)blockIdx.y * p.c.layer_stride;
    const piece_t* a = base + (int64_t)from * p.c.page_stride;
    piece_t* b = base + (int64_t)to * p.c.page_stride;
    // pieces in the order in which they lie in memory: the inner one of slots and heads first
    const bool head_inner = p.c.head_stride < p.c.slot_stride;
    const int inner = head_inner ? p.c.n_heads : slots;
    const int64_t s_in = head_inner ? p.c.head_stride : p.c.slot_stride;
    const int64_t s_out = head_inner ? p.c.slot_stride : p.c.head_stride;
    const int n = slots * p.c.n_heads * p.c.pieces;      // < 2^31: checked on the host
    constexpr int FLIGHT = 4;
    for (int i0 = threadIdx.x; i0 < n; i0 += FLIGHT * kThreads) {
        piece_t x[FLIGHT];
        int64_t off[FLIGHT];
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f) {
            const int i = i0 + f * kThreads;
            if (i < n) {
                const int row = i / p.c.pieces, c = i - row * p.c.pieces;
                const int o = row / inner, in = row - o * inner;
                off[f] = o * s_out + in * s_in + c;
                x[f] = a[off[f]];
            }
        }
#pragma unroll
        for (int f = 0; f < FLIGHT; ++f)
            if (i0 + f * kThreads < n) b[off[f]] = x[f];
    }
}

// Whether some row of an entry (of one or more) falls into no page or into one that another sequence holds: this
// thread's part of the pages, true for any thread of a workgroup says that the entry has no room.
// This may be asked while other entries give pages up: a page that two tables name came to be so by a fork, so that it
// lies within the committed length of both, and only pages beyond that are given up meanwhile.
__device__ __forceinline__ bool lacks_room(const KvView& c, const int32_t* table, int len, int rows) {
    const int last = (len + rows - 1) >> c.page_shift;
    bool lacks = last >= c.max_pages;
    for (int j = (len >> c.page_shift) + threadIdx.x; j <= min(last, c.max_pages - 1); j += kThreads) {
        const int page = table[j];
        lacks |= !is_page(c, page) || c.refs[page] > 1;
    }
    return lacks;
}

// ---- append -------------------------------------------------------------------------------
// A thread moves 16 bytes of k and the same of v.  Bound by bytes (1.1 GB read and written in 225 us at 16
// entries of up to 256 rows, 40 layers), small ones by latency: hence fewer rows to a workgroup then.
struct AppendParams {
    KvView c;
    BatchView b;
    const char* k_new;
    const char* v_new;
    int64_t row_stride;       // 16-byte pieces
    int64_t new_layer_stride;
    int layer;
    int rows_per_wg;
};
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const AppendParams p) {
    const EntryRows er = entry_rows(p.b, blockIdx.x);
    const int t0 = blockIdx.y * p.rows_per_wg;
    if (t0 >= er.rows) return;
    const int seq = entry_seq(p.b, p.c, blockIdx.x);
    if (seq < 0) return;
    const int len = entry_len(p.c, seq);
    const int32_t* table = p.c.table + (size_t)seq * p.c.max_pages;
    const int per_row = p.c.n_heads * p.c.pieces;
    const int n = min(p.rows_per_wg, er.rows - t0) * per_row;
    const int slot_mask = (1 << p.c.page_shift) - 1;
    const int64_t src_base = (int64_t)blockIdx.z * p.new_layer_stride + (int64_t)(er.first + t0) * p.row_stride;
    const int64_t dst_base = (int64_t)(p.layer + (int)blockIdx.z) * p.c.layer_stride;
    // (read once: pass by the caches, 425 -> 416 us of 16 branches of up to 256 rows; with stores that do so too 420.  The
    // first pieces are on their way while the pages are looked at.)
    piece_t a, b;
    auto load = [&](int i) {
        const int r = i / per_row;
        const int64_t src = src_base + (int64_t)r * p.row_stride + (i - r * per_row);
        a = __builtin_nontemporal_load((const piece_t*)p.k_new + src);
        b = __builtin_nontemporal_load((const piece_t*)p.v_new + src);
    };
    if ((int)threadIdx.x < n) load(threadIdx.x);
    if (__syncthreads_or(lacks_room(p.c, table, len, er.rows))) return;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int r = i / per_row, c = i - r * per_row;
        const int pos = len + t0 + r, page = table[pos >> p.c.page_shift];
        const int h = c / p.c.pieces, x = c - h * p.c.pieces;
        const int64_t dst = dst_base + page * p.c.page_stride + h * p.c.head_stride + (pos & slot_mask) * p.c.slot_stride + x;
        ((piece_t*)p.c.k)[dst] = a;
        ((piece_t*)p.c.v)[dst] = b;
        if (i + kThreads < n) load(i + kThreads);
    }
}

// ---- compact ------------------------------------------------------------------------------
// Row path[j] moves to row j <= path[j].  A workgroup takes some heads' rows of a layer, all of k or of v, and
// reads a batch of rows into registers before it writes any: what is written over is behind, or was read.
// Row by row, each move waiting for the one before it, 16 entries of up to 256 rows took 214 us; in batches 110, and 125
// with the look at the pages' counts.
// (Batches go in ascending order: a later one reads rows that no earlier one wrote, since path[j] >= j.)
struct CompactParams {
    KvView c;
    BatchView b;
    const int32_t* path;      // nullable
    const int32_t* keep;      // nullable
    int heads;                // of a workgroup
};
__device__ __forceinline__ int kept_rows(const CompactParams& p, const EntryRows& er) {
    return p.keep ? min(max(p.keep[blockIdx.x], 0), er.rows) : er.rows;
}
constexpr int kMoves = 16;                // 16-byte pieces of a thread in flight
__global__ void __launch_bounds__(kThreads) kv_move_kernel(const CompactParams p) {
    const EntryRows er = entry_rows(p.b, blockIdx.x);
    const int kept = kept_rows(p, er);
    const int seq = entry_seq(p.b, p.c, blockIdx.x);
    if (seq < 0 || kept == 0) return;
    const int groups = (p.c.n_heads + p.heads - 1) / p.heads;
    const int h0 = (blockIdx.z % groups) * p.heads, heads = min(p.heads, p.c.n_heads - h0);
    piece_t* base = (piece_t*)(blockIdx.z / groups ? p.c.v : p.c.k) + (int64_t)blockIdx.y * p.c.layer_stride + h0 * p.c.head_stride;
    const int len = entry_len(p.c, seq);
    const int32_t* table = p.c.table + (size_t)seq * p.c.max_pages;
    const bool lacks = lacks_room(p.c, table, len, er.rows);
    const int32_t* path = p.path + er.first;
    const int slot_mask = (1 << p.c.page_shift) - 1;
    auto place = [&](int row) {                       // (of an entry that has room)
        const int pos = len + row;
        return table[min(pos >> p.c.page_shift, p.c.max_pages - 1)] * p.c.page_stride + (pos & slot_mask) * p.c.slot_stride;
    };
    const int per = heads * p.c.pieces;               // pieces of a row
    // rows of a batch; a row of more pieces than a workgroup holds goes in parts, each through all rows
    const int wide_most = min(per, kMoves * kThreads), rows = min(kMoves * kThreads / wide_most, kThreads);
    __shared__ int64_t s_from[kThreads], s_to[kThreads];   // of the batch's rows; s_from < 0: stays
    for (int c0 = 0; c0 < per; c0 += wide_most) {
        const int wide = min(wide_most, per - c0);
        for (int j0 = 0; j0 < kept; j0 += rows) {
            const int n_rows = min(rows, kept - j0), n = n_rows * wide;
            if ((int)threadIdx.x < n_rows) {
                const int j = j0 + threadIdx.x, src = path[j];
                s_from[threadIdx.x] = src > j && src < er.rows ? place(src) : -1;
                s_to[threadIdx.x] = place(j);
            }
            if (__syncthreads_or(lacks)) return;
            piece_t val[kMoves];
#pragma unroll
            for (int m = 0; m < kMoves; ++m) {
                if (m * kThreads >= n) break;
                const int i = m * kThreads + threadIdx.x;
                const int j = i / wide, c = c0 + i - j * wide, h = c / p.c.pieces;
                if (i < n && s_from[j] >= 0) val[m] = base[s_from[j] + h * p.c.head_stride + (c - h * p.c.pieces)];
            }
            __syncthreads();                          // (the batch is read)
#pragma unroll
            for (int m = 0; m < kMoves; ++m) {
                if (m * kThreads >= n) break;
                const int i = m * kThreads + threadIdx.x;
                const int j = i / wide, c = c0 + i - j * wide, h = c / p.c.pieces;
                if (i < n && s_from[j] >= 0) base[s_to[j] + h * p.c.head_stride + (c - h * p.c.pieces)] = val[m];
            }
            __syncthreads();                          // (and written, before the next one is read)
        }
    }
}
__global__ void __launch_bounds__(kThreads) kv_commit_kernel(const CompactParams p) {
    const EntryRows er = entry_rows(p.b, blockIdx.x);
    const int kept = kept_rows(p, er);
    const int seq = entry_seq(p.b, p.c, blockIdx.x);
    if (seq < 0) return;
    const int before = entry_len(p.c, seq), page = 1 << p.c.page_shift;
    int32_t* row = p.c.table + (size_t)seq * p.c.max_pages;
    const int len = kept && !__syncthreads_or(lacks_room(p.c, row, before, er.rows)) ? before + kept : before;
    const int held = (len + page - 1) >> p.c.page_shift;
    for (int j = held + threadIdx.x; j < p.c.max_pages; j += kThreads) give_up(p.c, row + j);
    if (threadIdx.x == 0) p.c.seq_len[seq] = len;
}

size_t reserve_items(const dip_kv_cache* c, const dip_batch* b) {
    const int64_t per = (int64_t)rows_bound(b) / c->page_size + 2;
    return (size_t)b->n_batch * (size_t)(per < c->max_pages ? per : c->max_pages);
}
size_t reserve_bytes(const dip_kv_cache* c, const dip_batch* b) {
    return align_up(sizeof(CopyItem) * DIP_MAX_BATCH, 256) + align_up(sizeof(int32_t) * c->n_pages, 256) +
           align_up(reserve_items(c, b) / 8 + 8, 256);
}
constexpr int kMaxList = (1 << 24) - 1;  // sequences or pages of one call: a launch has fewer than 2^32 threads

int32_t check_list(const void* a, const void* b, int32_t n) {
    if (!a || !b) return fail(DIP_ERR_INVALID_ARG, "null list");
    if (n < 1 || n > kMaxList) return fail(DIP_ERR_INVALID_ARG, "a list has 1 .. %d entries, got %d", kMaxList, n);
    return DIP_OK;
}
int32_t check_page_bytes(const dip_kv_cache* c) {
    if ((int64_t)c->page_size * c->n_kv_heads * c->head_dim >= (int64_t)1 << 30)
        return fail(DIP_ERR_UNSUPPORTED, "cache: a page has 2^30 elements or more");
    return DIP_OK;
}

}  // namespace
}  // namespace dip

using namespace dip;

extern "C" {

int32_t dip_kv_init(const dip_kv_cache* cache, void* stream) {
    int32_t st = validate_kv(cache);
    if (st) return st;
    const InitParams p = {view_of(cache)};
    const int64_t most = (int64_t)cache->n_seqs * cache->max_pages > cache->n_pages ? (int64_t)cache->n_seqs * cache->max_pages : cache->n_pages;
    const int64_t wgs = (most + kThreads - 1) / kThreads;
    return check_hip(launch_timed(kv_init_kernel, dim3((unsigned)(wgs < 2048 ? wgs : 2048)), dim3(kThreads), (hipStream_t)stream,
                                  DIP_KERNEL_KV, p), "kv_init launch");
}

int32_t dip_kv_free(const dip_kv_cache* cache, const int32_t* seqs, int32_t n, void* stream) {
    int32_t st = validate_kv(cache);
    if (!st) st = check_list(seqs, seqs, n);
    if (st) return st;
    const SeqsParams p = {view_of(cache), seqs, nullptr};
    return check_hip(launch_timed(kv_free_kernel, dim3(n), dim3(kThreads), (hipStream_t)stream, DIP_KERNEL_KV, p), "kv_free launch");
}

int32_t dip_kv_fork(const dip_kv_cache* cache, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
    int32_t st = validate_kv(cache);
    if (!st) st = check_list(src, dst, n);
    if (st) return st;
    const SeqsParams p = {view_of(cache), src, dst};
    return check_hip(launch_timed(kv_fork_kernel, dim3(n), dim3(kThreads), (hipStream_t)stream, DIP_KERNEL_KV, p), "kv_fork launch");
}

int32_t dip_kv_copy_pages(const dip_kv_cache* cache, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
    int32_t st = validate_kv(cache);
    if (!st) st = check_list(src, dst, n);
    if (!st) st = check_page_bytes(cache);
    if (st) return st;
    const CopyParams p = {view_of(cache), nullptr, src, dst};
    return check_hip(launch_timed(kv_copy_kernel, dim3(n, cache->n_layers, 2), dim3(kThreads), (hipStream_t)stream, DIP_KERNEL_KV, p),
                     "kv_copy launch");
}

size_t dip_kv_reserve_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch) {
    if (validate_kv(cache) || validate_batch(batch, true)) return 0;
    return reserve_bytes(cache, batch);
}

int32_t dip_kv_reserve(const dip_kv_cache* cache, const dip_batch* batch, int32_t* granted, void* ws, size_t ws_bytes, void* stream) {
    int32_t st = validate_kv(cache);
    if (!st) st = validate_batch(batch, true);
    if (!st) st = check_page_bytes(cache);
    if (!st) st = validate_ws(ws, ws_bytes, reserve_bytes(cache, batch));
    if (st) return st;
    char* at = (char*)ws;
    ReserveParams p;
    p.c = view_of(cache);
    p.b = view_of(batch);
    p.granted = granted;
    p.copies = (CopyItem*)at;
    at += align_up(sizeof(CopyItem) * DIP_MAX_BATCH, 256);
    p.free_pages = (int32_t*)at;
    at += align_up(sizeof(int32_t) * cache->n_pages, 256);
    p.wanted = (uint64_t*)at;
    st = check_hip(launch_timed(kv_reserve_kernel, dim3(1), dim3(kReserveThreads), (hipStream_t)stream, DIP_KERNEL_KV, p), "kv_reserve launch");
    if (st) return st;
    const CopyParams cp = {p.c, p.copies, nullptr, nullptr};
    return check_hip(launch_timed(kv_copy_kernel, dim3(batch->n_batch, cache->n_layers, 2), dim3(kThreads), (hipStream_t)stream,
                                  DIP_KERNEL_KV, cp), "kv_copy launch");
}

int32_t dip_kv_append(const dip_kv_cache* cache, int32_t layer, int32_t n_layers, const dip_batch* batch, const void* k_new,
                      const void* v_new, int64_t row_stride, int64_t new_layer_stride, void* stream) {
    int32_t st = validate_kv(cache);
    if (!st) st = validate_batch(batch, true);
    if (!st) st = check_page_bytes(cache);
    if (st) return st;
    if (layer < 0 || n_layers < 1 || n_layers > cache->n_layers || layer > cache->n_layers - n_layers)
        return fail(DIP_ERR_INVALID_ARG, "layers %d .. %d outside the cache's %d", layer, layer + n_layers - 1, cache->n_layers);
    if (!k_new || !v_new) return fail(DIP_ERR_INVALID_ARG, "null rows");
    const int per = 16 / elem_bytes(cache->dtype);
    if (row_stride < (int64_t)cache->n_kv_heads * cache->head_dim || (n_layers > 1 && new_layer_stride < 1))
        return fail(DIP_ERR_INVALID_ARG, "row_stride smaller than a row, or no layer stride");
    if (row_stride % per || new_layer_stride % per || !aligned16(k_new) || !aligned16(v_new))
        return fail(DIP_ERR_UNSUPPORTED, "new rows must start on 16-byte boundaries");
    AppendParams p;
    p.c = view_of(cache);
    p.b = view_of(batch);
    p.k_new = (const char*)k_new;
    p.v_new = (const char*)v_new;
    p.row_stride = row_stride / per;
    p.new_layer_stride = new_layer_stride / per;
    p.layer = layer;
    // rows of a workgroup: 16 where that leaves enough workgroups for the chip, else fewer (and their pieces fit 32 bits)
    int rows = 16;
    while (rows > 1 && ((int64_t)batch->n_rows * n_layers / rows < 1024 || (int64_t)rows * p.c.n_heads * p.c.pieces > 1 << 28)) rows >>= 1;
    p.rows_per_wg = rows;
    const unsigned blocks = (unsigned)((p.b.max_rows + rows - 1) / rows);
    if (blocks > 65535) return fail(DIP_ERR_UNSUPPORTED, "max_rows is too large for one call");
    return check_hip(launch_timed(kv_append_kernel, dim3(batch->n_batch, blocks, n_layers), dim3(kThreads), (hipStream_t)stream,
                                  DIP_KERNEL_KV, p), "kv_append launch");
}

int32_t dip_kv_compact(const dip_kv_cache* cache, const dip_batch* batch, const int32_t* path, const int32_t* keep, void* stream) {
    int32_t st = validate_kv(cache);
    if (!st) st = validate_batch(batch, true);
    if (!st) st = check_page_bytes(cache);
    if (st) return st;
    CompactParams p = {view_of(cache), view_of(batch), path, keep, 1};
    if (path) {
        // as many heads to a workgroup as its registers take rows of
        const int64_t most = (int64_t)p.b.max_rows * p.c.pieces;
        int64_t heads = kMoves * kThreads / (most > 0 ? most : 1);
        heads = heads < 1 ? 1 : heads > cache->n_kv_heads ? cache->n_kv_heads : heads;
        p.heads = (int)heads;
        const int64_t groups = 2 * ((cache->n_kv_heads + heads - 1) / heads);
        if (groups > 65535) return fail(DIP_ERR_UNSUPPORTED, "cache: too many heads");
        st = check_hip(launch_timed(kv_move_kernel, dim3(batch->n_batch, cache->n_layers, (unsigned)groups), dim3(kThreads),
                                    (hipStream_t)stream, DIP_KERNEL_KV, p), "kv_move launch");
        if (st) return st;
    }
    return check_hip(launch_timed(kv_commit_kernel, dim3(batch->n_batch), dim3(kThreads), (hipStream_t)stream, DIP_KERNEL_KV, p),
                     "kv_commit launch");
}

}  // extern "C"
