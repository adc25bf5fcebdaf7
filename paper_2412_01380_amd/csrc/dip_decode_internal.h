// Shared by the translation units of the calls around the MLP (cache pages, attention,
// verification): argument checks, and what a workgroup looks up about an entry of the batch.
#ifndef DIP_DECODE_INTERNAL_H_
#define DIP_DECODE_INTERNAL_H_

#include "dip_internal.h"

namespace dip {

// ---- argument checks (host) ---------------------------------------------------------------
int32_t validate_kv(const dip_kv_cache* c);
int32_t validate_batch(const dip_batch* b, bool need_seqs);
int32_t validate_ws(const void* ws, size_t have, size_t need);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline int elem_bytes(int dtype) { return dtype == DIP_F32 ? 4 : 2; }
inline int rows_bound(const dip_batch* b) { return b->max_rows < b->n_rows ? b->max_rows : b->n_rows; }
inline int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

// Whether one of `rows` rows at x, x_width bytes each, meets one at y.
inline bool rows_overlap(const void* x, int64_t x_stride, int64_t x_width, const void* y, int64_t y_stride, int64_t y_width, int64_t rows) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
    const uintptr_t a_end = a + (uintptr_t)((rows - 1) * x_stride + x_width), b_end = b + (uintptr_t)((rows - 1) * y_stride + y_width);
    if (a_end <= b || b_end <= a) return false;
    if (x_stride != y_stride) return true;
    // (columns of one array side by side: no row of one meets a row of the other)
    const uintptr_t stride = (uintptr_t)x_stride, off = b >= a ? (b - a) % stride : (stride - (a - b) % stride) % stride;
    return off < (uintptr_t)x_width || off + (uintptr_t)y_width > stride;
}

// ---- the cache as the kernels take it ------------------------------------------------------
// Strides in 16-byte pieces; the page size is a power of two.
struct KvView {
    char* k;
    char* v;
    int32_t* table;
    int32_t* seq_len;
    int32_t* refs;
    int n_pages, n_seqs, max_pages, n_layers, n_heads;
    int page_shift;
    int pieces;               // 16-byte pieces of one head of one position
    int64_t layer_stride, page_stride, head_stride, slot_stride;
};
KvView view_of(const dip_kv_cache* c);

struct BatchView {
    const int32_t* seqs;
    const int32_t* row_start;
    int n_batch, n_rows, max_rows;
};
inline BatchView view_of(const dip_batch* b) { return {b->seqs, b->row_start, b->n_batch, b->n_rows, rows_bound(b)}; }

// An entry's rows, whatever row_start holds: [first, first + rows) lies inside [0, n_rows).
struct EntryRows {
    int first, rows;
};
__device__ __forceinline__ EntryRows entry_rows(const BatchView& b, int e) {
    int lo = b.row_start[e], hi = b.row_start[e + 1];
    lo = min(max(lo, 0), b.n_rows);
    hi = min(max(hi, lo), b.n_rows);
    return {lo, min(hi - lo, b.max_rows)};
}
// The sequence of an entry (-1: out of range) and its committed tokens, as far as the table goes.
__device__ __forceinline__ int entry_seq(const BatchView& b, const KvView& c, int e) {
    const int s = b.seqs[e];
    return (unsigned)s < (unsigned)c.n_seqs ? s : -1;
}
__device__ __forceinline__ int entry_len(const KvView& c, int seq) {
    return min(max(c.seq_len[seq], 0), c.max_pages << c.page_shift);
}

__device__ __forceinline__ bool is_page(const KvView& c, int p) { return (unsigned)p < (unsigned)c.n_pages; }
// Whether some row of an entry (of one or more) falls into no page or into one that another sequence holds: this
// thread's part of the pages, true for any thread of a workgroup says that the entry has no room.
// This may be asked while other entries give pages up: a page that two tables name came to be so by a fork, so that it
// lies within the committed length of both, and only pages beyond that are given up meanwhile.
template <int THREADS>
__device__ __forceinline__ bool lacks_room(const KvView& c, const int32_t* table, int len, int rows) {
    const int last = (len + rows - 1) >> c.page_shift;
    bool lacks = last >= c.max_pages;
    for (int j = (len >> c.page_shift) + threadIdx.x; j <= min(last, c.max_pages - 1); j += THREADS) {
        const int page = table[j];
        lacks |= !is_page(c, page) || c.refs[page] > 1;
    }
    return lacks;
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

// ---- the last workgroup of several -------------------------------------------------------------
// A ticket word is the tag of a launch (upper 48 bits) and the tickets drawn in it; a word with another tag
// counts as none, so nothing has to clear it.  Whoever draws the last ticket of a word goes on with what the
// others stored, through agent-scope accesses, which the L2s of all dies agree on, and had acknowledged
// (vmcnt 0) before their tickets.
constexpr int kTicketStride = 16;         // words: 128 bytes, so that atomics on different words do not queue
__device__ __forceinline__ void ticket_open(uint64_t* word, uint64_t epoch) {
    uint64_t seen = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if ((seen ^ epoch) >> 16)
        __hip_atomic_compare_exchange_strong(word, &seen, epoch, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// one thread, behind the barrier behind everybody's stores: whether this was the last of `n`
__device__ __forceinline__ bool ticket_last(uint64_t* word, uint64_t epoch, int n) {
    const bool last = __hip_atomic_fetch_add(word, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == epoch + (uint64_t)(n - 1);
    if (last) __hip_atomic_store(word, epoch, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // (for a replay)
    return last;
}

}  // namespace dip

#endif  // DIP_DECODE_INTERNAL_H_
