/*
 * libdip -- Dynamic Input Pruning (DIP) and cache-aware masking (DIP-CA) for the
 * batch-1 SwiGLU MLP forward, native on AMD MI355X (gfx950).
 *
 * Paper notation used throughout (Sec. 3-5):
 *   x        input activations of a linear layer (fp32 here)
 *   W^u,W^g  up / gate matrices in R^{d_ff x d_model}; W^d down matrix in R^{d_model x d_ff}
 *   GLU(x)   = W^u x (.) SiLU(W^g x)                                   (Sec. 3, Eq. 2)
 *   m        binary column mask with exactly k ones, m = topK(s, k)    (Alg. 1)
 *   c        binary residency mask: which columns are in the cache     (Sec. 5.2)
 *   s        = |x| (c + gamma (1 - c)) / ||x||_inf                     (Sec. 5.2, Eq. 10)
 *
 * Conventions
 *   - Plain C ABI.  Every pointer is a DEVICE pointer unless its comment says "host".
 *     Descriptor structs (dip_weight, dip_cache, dip_mlp, dip_debug) are host structs
 *     holding device pointers; the library reads them during the call only.
 *   - The library allocates nothing on the device: outputs, cache state and workspace
 *     belong to the caller, and it never frees caller memory.  The calls declared in this
 *     header keep no state between calls, with one exception that says so
 *     (dip_swiglu_mlp_forward_noalloc and its built-in scratch).  The process-wide
 *     switches for tuning and per-kernel timing live in dip_devtools.h.
 *   - All work is enqueued on the caller's stream (a hipStream_t passed as void*, NULL =
 *     the default stream).  No call synchronises with the host or reads device memory
 *     back.  Calls on one stream are ordered; calls that share a workspace or a cache on
 *     different streams race.  The scoring, selection, cache-update, product and forward
 *     calls enqueue kernel launches only (no allocation, no memset, no copy), so they may
 *     be captured into a HIP graph and replayed; dip_profile_enable must be off then.
 *   - Arguments are validated on the host before any HIP call.  On an error nothing is
 *     enqueued and no state changes.  Every function returns a dip_status; the message
 *     of the last failure on the calling thread is available from dip_last_error().
 *   - Bit masks: uint32_t[ceil(n/32)], feature i is bit (i & 31) of word (i >> 5); the
 *     padding bits of the last word are written as zero.  Index lists: int32_t, strictly
 *     ascending.
 *   - Weight layout is FEATURE-MAJOR: a matrix the paper writes as W in R^{n_out x n_in}
 *     is stored as n_in rows of n_out elements; stored row i is the paper's column
 *     W[:, i], everything that input feature i multiplies, so one selected column is one
 *     contiguous burst.  Row starts and row_stride_bytes must be multiples of 16.
 *   - Inputs must be finite.  Non-finite inputs never hang or fault; results are then
 *     unspecified.
 */
#ifndef DIP_H_
#define DIP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DIP_VERSION_MAJOR 0
#define DIP_VERSION_MINOR 1

typedef enum dip_status {
    DIP_OK = 0,
    DIP_ERR_INVALID_ARG = 1, /* null pointer, k outside [1, n], gamma outside [0, 1], ...   */
    DIP_ERR_UNSUPPORTED = 2, /* dtype / size / alignment the kernels do not handle          */
    DIP_ERR_WORKSPACE = 3,   /* workspace pointer null or smaller than *_workspace_bytes()  */
    DIP_ERR_HIP = 4          /* the HIP runtime reported an error at launch                 */
} dip_status;

typedef enum dip_dtype {
    DIP_F32 = 0,      /* fp32 weights                                                       */
    DIP_BF16 = 1,     /* bfloat16 weights, widened exactly to fp32 before the multiply      */
    DIP_INT4_G128 = 2 /* signed 4-bit codes, one fp16 scale per 128 consecutive elements of
                         a stored row (dip_weight.scales: n_out/128 per row, rows back to
                         back), w = scale * q; two codes per byte, low nibble = even
                         element; n_out must be a multiple of 128                           */
} dip_dtype;

typedef enum dip_policy {
    DIP_LRU = 0, /* evict the resident whose last use lies farthest back   (Sec. 5.1)       */
    DIP_LFU = 1  /* evict the resident with the smallest use counter       (Sec. 5.1)       */
} dip_policy;

/* Largest vector length the selection kernels handle (one workgroup keeps all keys in registers). */
#define DIP_MAX_N 32768

/* A feature-major weight matrix (see "Weight layout" above). */
typedef struct dip_weight {
    const void* data;         /* device; n_in rows                                          */
    const void* scales;       /* device; fp16 scales for DIP_INT4_G128, otherwise NULL      */
    int32_t dtype;            /* dip_dtype                                                   */
    int32_t n_in;             /* input features = stored rows                               */
    int32_t n_out;            /* outputs = elements per stored row                          */
    int32_t reserved;         /* must be 0                                                  */
    int64_t row_stride_bytes; /* distance between stored rows, >= n_out * element size      */
} dip_weight;

/* The three matrices of one SwiGLU MLP (Sec. 3, Eq. 1-2).  Up and gate are bundled per
 * input feature: stored row i of w_ug is [ W^u[:, i] ; W^g[:, i] ], 2*d_ff elements, so
 * w_ug.n_in = d_model, w_ug.n_out = 2*d_ff, and w_d.n_in = d_ff, w_d.n_out = d_model. */
typedef struct dip_mlp {
    dip_weight w_ug;
    dip_weight w_d;
} dip_mlp;

#define DIP_CACHE_META_WORDS 8
/* meta[] layout (device, uint32): */
#define DIP_META_STEP 0      /* 1-based step counter t; advanced by one per update          */
#define DIP_META_RESIDENT 1  /* number of resident columns after the last update            */
#define DIP_META_HITS 2      /* |m & c| of the last update                                  */
#define DIP_META_INSERTED 3  /* misses brought into the cache by the last update            */
#define DIP_META_EVICTED 4   /* residents evicted by the last update                        */
#define DIP_META_BYPASSED 5  /* misses that found no room and were not cached               */
#define DIP_META_CUM_HITS 6  /* running sum of hits   (wraps at 2^32)                       */
#define DIP_META_CUM_LOOKUPS 7 /* running sum of |m|  (wraps at 2^32)                       */

/* Residency state of one linear layer's columns (the paper's c, Sec. 5.2), owned by the caller. */
typedef struct dip_cache {
    uint32_t* bits;   /* device; ceil(n/32) words; bit set = column resident                */
    uint32_t* stamp;  /* device; n words; LRU: step of last use, LFU: use count             */
    uint32_t* meta;   /* device; DIP_CACHE_META_WORDS words                                 */
    int32_t n;        /* number of columns (input features of the layer)                   */
    int32_t capacity; /* at most this many columns resident, 0 <= capacity <= n             */
    int32_t policy;   /* dip_policy                                                         */
    int32_t reserved; /* must be 0                                                          */
} dip_cache;

/* Optional per-stage outputs of dip_swiglu_mlp_forward for stage-wise comparison; every
 * member may be NULL. */
typedef struct dip_debug {
    float* s_in;        /* d_model scores at pruning point 1                                */
    uint32_t* mask_in;  /* ceil(d_model/32) words                                           */
    int32_t* idx_in;    /* k_in ascending indices (16-byte aligned)                         */
    float* h;           /* d_ff: the sparse GLU output  GLU~(x)                             */
    float* s_mid;       /* d_ff scores at pruning point 2                                   */
    uint32_t* mask_mid; /* ceil(d_ff/32) words                                              */
    int32_t* idx_mid;   /* k_mid ascending indices (16-byte aligned)                        */
} dip_debug;

/* The sibling schemes of Sec. 3.2 that prune on a partial activation. */
typedef enum dip_scheme {
    DIP_GATE_PRUNING = 1, /* a = SiLU(W^g x) dense; topK(|a|) removes rows of W^u, columns of W^d */
    DIP_UP_PRUNING = 2    /* a = W^u x dense;       topK(|a|) removes rows of W^g, columns of W^d */
} dip_scheme;

/* The three matrices of one SwiGLU MLP stored for Gate / Up pruning.  The matrix that is
 * multiplied densely (W^g for gate pruning, W^u for up pruning) is feature-major like every
 * other matrix here.  The one whose ROWS the mask removes is NEURON-MAJOR: stored row j is
 * row j of the paper's matrix, the d_model weights of GLU unit j, so that a kept unit is one
 * contiguous burst; in its descriptor n_in = d_ff (stored rows) and n_out = d_model
 * (elements per stored row). */
typedef struct dip_mlp_split {
    dip_weight w_dense; /* feature-major, n_in = d_model, n_out = d_ff                      */
    dip_weight w_rows;  /* neuron-major,  n_in = d_ff,    n_out = d_model                   */
    dip_weight w_d;     /* feature-major, n_in = d_ff,    n_out = d_model                   */
} dip_mlp_split;

/* Optional stage outputs of dip_partial_pruning_forward; every member may be NULL. */
typedef struct dip_partial_debug {
    float* a;       /* d_ff: the partial activation the mask is taken from                  */
    uint32_t* mask; /* ceil(d_ff/32) words                                                  */
    int32_t* idx;   /* k ascending kept GLU units (16-byte aligned)                         */
    float* h_sel;   /* k values of GLU~(x) at those units (16-byte aligned)                 */
} dip_partial_debug;

/* A weight matrix kept in two tiers (Sec. 5: a small fast memory caching columns of a large
 * slow one).  `full` describes the whole feature-major matrix in PINNED HOST memory that the
 * GPU can read directly (full.data is that device-accessible host pointer); `slots` is the
 * fast tier: `capacity` rows of full.row_stride_bytes in HBM.  Column i is resident -- bit i
 * of the cache's residency mask -- exactly when slot_of[i] >= 0, and then slots row
 * slot_of[i] holds a copy of stored row i.  F32 and BF16 only. */
typedef struct dip_tiered_weight {
    dip_weight full;     /* data: host memory, device-accessible                            */
    void* slots;         /* device; capacity rows, 16-byte aligned                          */
    int32_t* slot_of;    /* device; full.n_in entries                                       */
    int32_t capacity;    /* slots; must equal the capacity of the cache used with it        */
    int32_t reserved;    /* must be 0                                                       */
} dip_tiered_weight;

typedef struct dip_tiered_mlp {
    dip_tiered_weight w_ug; /* bundled up/gate, as in dip_mlp                              */
    dip_tiered_weight w_d;
} dip_tiered_mlp;

/* (major << 16) | minor. */
int32_t dip_version(void);

/* Message of the last failing call on this thread (host string, never NULL, owned by the library). */
const char* dip_last_error(void);

/*
 * Cache-aware scores, Sec. 5.2 Eq. 10 / Alg. 1 step 1, in fp32 with this exact operation
 * order (round to nearest even, no fused operations, denormals kept):
 *     a = |x_i| ;  p = c_i ? a : fl(a * gamma) ;  s_i = fl(p / M),  M = max_i |x_i| ;
 *     M == 0  ->  s = 0.
 * cache_bits == NULL selects the plain DIP key of Sec. 4:  s_i = |x_i|  (gamma ignored).
 *   x          n floats          cache_bits  ceil(n/32) words or NULL
 *   s_out      n floats          1 <= n <= DIP_MAX_N,  0 <= gamma <= 1
 */
int32_t dip_ca_scores(const float* x, int32_t n, const uint32_t* cache_bits, float gamma,
                      float* s_out, void* stream);

/*
 * m = topK(s, k), Alg. 1 step 2 (per-token top-K thresholding, Sec. 3.1): exactly k
 * features with the largest keys; among equal keys the lowest index wins.  Keys must be
 * non-negative (scores are).
 *   s         n floats, 1 <= k <= n <= DIP_MAX_N
 *   mask_out  ceil(n/32) words, or NULL
 *   idx_out   k ascending indices, or NULL      (at least one of the two outputs is required)
 */
int32_t dip_prune_topk(const float* s, int32_t n, int32_t k, uint32_t* mask_out,
                       int32_t* idx_out, void* stream);

/*
 * Start a cache: step counter 1, all counters 0, stamps 0, residency = initial_bits
 * (ceil(n/32) words with at most `capacity` bits set -- not checked on the device; padding
 * bits must be zero) or empty when initial_bits is NULL.
 */
int32_t dip_cache_init(const dip_cache* cache, const uint32_t* initial_bits, void* stream);

/*
 * c' = cache_update(c, m), Alg. 1 step 3, for one token's mask m (ceil(n/32) words).
 * The mask is a set, so the update is set-valued and deterministic:
 *   hits   = m & c   keep their place; LRU stamps them with the current step
 *   misses = m & ~c  in ascending index order
 *   free   = capacity - |c| ;  victims V = c & ~m  (a column this token uses is never evicted)
 *   n_ins  = min(|misses|, free + |V|) ;  evict the max(0, n_ins - free) members of V with
 *            the smallest (stamp, index) ;  insert the first n_ins misses ;  the remaining
 *            misses bypass the cache (Sec. 6.4: when the active set does not fit, part of
 *            it is used without being cached).
 *   LFU: stamp counts every selection of a column, resident or not, and survives eviction.
 * Advances meta[DIP_META_STEP] and refreshes the other meta counters.
 */
int32_t dip_cache_update(const dip_cache* cache, const uint32_t* mask_bits, void* stream);

/*
 * Checkpoint helpers for a cache (the state survives between tokens, Alg. 1 returns c^(t)).
 * dip_cache_state_bytes: sizes of the three caller-owned arrays for n columns (host outputs,
 * each may be NULL).  dip_cache_export / dip_cache_import copy the whole state to / from one
 * contiguous blob of dip_cache_blob_bytes(n) bytes laid out [bits | stamp | meta], each part
 * starting on a 256-byte boundary; the blob may be device memory or host memory (pinned
 * host memory keeps the copy asynchronous).  Copies are enqueued on the stream.
 */
int32_t dip_cache_state_bytes(int32_t n, size_t* bits_bytes /* host */, size_t* stamp_bytes /* host */,
                              size_t* meta_bytes /* host */);
size_t dip_cache_blob_bytes(int32_t n);
int32_t dip_cache_export(const dip_cache* cache, void* blob, size_t blob_bytes, void* stream);
int32_t dip_cache_import(const dip_cache* cache, const void* blob, size_t blob_bytes, void* stream);

/*
 * Column-gathered matrix-vector product, Alg. 1 step 4 (W~ = W (.) m) applied to x:
 *     y[j] = sum_{t<k} W[j, idx[t]] * x[idx[t]]        fp32 accumulation.
 * The summation order is fixed by the launch configuration, so results are bit-repeatable.
 *   w        feature-major matrix (F32, BF16 or INT4_G128); a row is whole 16-byte loads
 *   x        w->n_in floats        idx   k ascending indices in [0, n_in), 1 <= k <= n_in
 *   y_out    w->n_out floats       ws    dip_gathered_gemv_workspace_bytes() bytes, 256-aligned
 */
size_t dip_gathered_gemv_workspace_bytes(const dip_weight* w, int32_t k);
int32_t dip_gathered_gemv(const dip_weight* w, const float* x, const int32_t* idx, int32_t k,
                          float* y_out, void* ws, size_t ws_bytes, void* stream);

/*
 * One token through one DIP / DIP-CA SwiGLU MLP (Sec. 4 composed with Alg. 1 at both
 * pruning points):
 *   1. s1 = score(x, c_in)          m1 = topK(s1, k_in)       c_in  <- cache_update(c_in,  m1)
 *   2. h~ = (sum_{i in m1} W^u[:,i] x_i) (.) SiLU(sum_{i in m1} W^g[:,i] x_i)
 *   3. s2 = score(h~, c_mid)        m2 = topK(s2, k_mid)      c_mid <- cache_update(c_mid, m2)
 *   4. y  = sum_{i in m2} W^d[:,i] h~_i
 * Scoring uses the cache state from before this token (the paper's c^(t-1)).  With a NULL
 * cache the key is |.| (DIP); a cache pointer switches that point to Eq. 10 (DIP-CA) and its
 * state is updated in place.
 *   x      d_model floats       y_out   d_model floats
 *   1 <= k_in <= d_model, 1 <= k_mid <= d_ff;  d_model, d_ff <= DIP_MAX_N
 *   dbg    NULL or stage outputs           ws   *_workspace_bytes() bytes, 256-aligned
 */
size_t dip_swiglu_mlp_forward_workspace_bytes(const dip_mlp* mlp, int32_t k_in, int32_t k_mid);
int32_t dip_swiglu_mlp_forward(const dip_mlp* mlp, const float* x, int32_t k_in, int32_t k_mid,
                               const dip_cache* cache_in, const dip_cache* cache_mid,
                               float gamma, float* y_out, const dip_debug* dbg, void* ws,
                               size_t ws_bytes, void* stream);

/*
 * dip_swiglu_mlp_forward for callers that cannot allocate device memory or hand over a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same arguments, results and ordering rules as dip_swiglu_mlp_forward, minus
 * the workspace: the scratch (index lists, h~, split-K partial sums, ticket counters) lives
 * in a device array built into the library, DIP_STATIC_SCRATCH_BYTES per GPU, held from
 * library load until the process ends.  The call allocates and frees nothing.  A layer
 * whose dip_swiglu_mlp_forward_workspace_bytes() exceeds DIP_STATIC_SCRATCH_BYTES is
 * rejected with DIP_ERR_WORKSPACE and nothing is enqueued.  All calls on one GPU share that
 * GPU's array, which may hold anything when a call starts (a launch knows its own ticket
 * counts by their tag; nothing is cleared): calls that overlap on one GPU -- different streams,
 * or replays of graphs that contain it running concurrently -- race.
 */
#define DIP_STATIC_SCRATCH_BYTES (4u << 20)
int32_t dip_swiglu_mlp_forward_noalloc(const dip_mlp* mlp, const float* x, int32_t k_in, int32_t k_mid,
                                       const dip_cache* cache_in, const dip_cache* cache_mid,
                                       float gamma, float* y_out, const dip_debug* dbg, void* stream);

/*
 * The same forward for n_layers independent layers in one call (a decode step over a
 * stack): layer l reads x + l * x_stride and writes y_out + l * y_stride (strides in
 * floats) and keeps k_in[l] of its inputs and k_mid[l] of its GLU units (host arrays of
 * n_layers entries: Sec. 4 allows different sparsity levels per matrix and layer).
 * The layers run phase by phase where their rows lie apart.  If the output of one overlaps the
 * input of a later one or the output of another, they run one after the other, in order.
 * mlps / caches_in / caches_mid are host arrays of n_layers descriptors; the cache arrays
 * may be NULL (DIP).  Every layer and pruning point needs a dip_cache of its own (the call
 * rejects shared state): every cache is scored with its state from before the call and all
 * are updated together in one launch at the end of it.
 * Results are those of one dip_swiglu_mlp_forward per layer up to the rounding of the fp32 sums:
 * the order of a sum follows from the shape, k and the number of consecutive layers of one
 * shape, so it is the same for every call like this one, and another for a call per layer, over
 * part of the stack, or with rows that overlap.  Where two scores of point 2 agree to within
 * that rounding the masks, and with them the caches, may differ by that pair of columns.
 * ws: dip_swiglu_mlp_forward_stack_workspace_bytes() bytes, 256-aligned.
 */
size_t dip_swiglu_mlp_forward_stack_workspace_bytes(const dip_mlp* mlps, int32_t n_layers,
                                                    const int32_t* k_in /* host */,
                                                    const int32_t* k_mid /* host */);
int32_t dip_swiglu_mlp_forward_stack(const dip_mlp* mlps, int32_t n_layers, const float* x,
                                     int64_t x_stride, const int32_t* k_in /* host */,
                                     const int32_t* k_mid /* host */, const dip_cache* caches_in,
                                     const dip_cache* caches_mid, float gamma, float* y_out,
                                     int64_t y_stride, void* ws, size_t ws_bytes, void* stream);

/*
 * A small decode batch through one layer: `batch` (1..8) rows X[b] (row stride d_model)
 * give `batch` independent batch-1 results Y[b] of dip_swiglu_mlp_forward -- every row has
 * its own two top-K masks -- while each stored column is read once if any row selected it
 * (the union of the row masks) and is accumulated only into the rows that selected it.
 * All rows are scored against the cache state from before the step; each cache is then
 * updated once with the union mask (Alg. 1 step 3).  The paper itself is batch 1 (Sec. 1).
 * Optional outputs for stage-wise comparison (each may be NULL):
 *   mask_in_out   [batch][ceil(d_model/32)] words     h_out  [batch][d_ff] floats
 *   mask_mid_out  [batch][ceil(d_ff/32)] words
 * Summation order is fixed by the launch configuration (bit-repeatable).
 * DIP_INT4_G128 weights with batch >= 3 are multiplied on the matrix cores (matrices of up to
 * 4 GiB; larger ones take the vector path): every row's activations are first scaled by a
 * power of two into [8, 16) -- exact, and undone exactly on the partial sums, so the result
 * does not depend on the magnitude of the activations -- and activation times group scale
 * enters as two fp16 terms (about 21 significant bits of the row's largest product); this
 * needs group scales of at most 4094 (|w| up to 28658; beyond that the sums overflow to
 * inf).  The sums are fp32 as everywhere else.
 */
size_t dip_swiglu_mlp_forward_batched_workspace_bytes(const dip_mlp* mlp, int32_t batch,
                                                      int32_t k_in, int32_t k_mid);
int32_t dip_swiglu_mlp_forward_batched(const dip_mlp* mlp, const float* X, int32_t batch,
                                       int32_t k_in, int32_t k_mid, const dip_cache* cache_in,
                                       const dip_cache* cache_mid, float gamma, float* Y,
                                       uint32_t* mask_in_out, float* h_out, uint32_t* mask_mid_out,
                                       void* ws, size_t ws_bytes, void* stream);

/*
 * The batched forward for n_layers independent layers in one call: layer l reads its `batch`
 * rows at X + l * x_stride ([batch][d_model], contiguous) and writes Y + l * y_stride (strides
 * in floats), with k_in[l] / k_mid[l] kept per row (host arrays).  Rules for overlapping rows,
 * for the order of the sums and for caches as in dip_swiglu_mlp_forward_stack: one dip_cache per
 * layer and point, all updated -- once each, with the union of the layer's row masks -- in one
 * launch at the end of the call.
 */
size_t dip_swiglu_mlp_forward_batched_stack_workspace_bytes(const dip_mlp* mlps, int32_t n_layers, int32_t batch,
                                                            const int32_t* k_in /* host */,
                                                            const int32_t* k_mid /* host */);
int32_t dip_swiglu_mlp_forward_batched_stack(const dip_mlp* mlps, int32_t n_layers, const float* X,
                                             int64_t x_stride, int32_t batch, const int32_t* k_in /* host */,
                                             const int32_t* k_mid /* host */, const dip_cache* caches_in,
                                             const dip_cache* caches_mid, float gamma, float* Y,
                                             int64_t y_stride, void* ws, size_t ws_bytes, void* stream);

/*
 * GLU pruning, Sec. 3.2: W^u x and W^g x are dense, m = topK(|GLU(x)|, k) removes columns
 * of W^d:  y = sum_{i in m} W^d[:, i] GLU(x)_i.  Same matrices, layout and workspace rules
 * as dip_swiglu_mlp_forward; x must be 16-byte aligned; the point-1 members of dbg must be NULL.
 */
size_t dip_glu_pruning_forward_workspace_bytes(const dip_mlp* mlp, int32_t k);
int32_t dip_glu_pruning_forward(const dip_mlp* mlp, const float* x, int32_t k, float* y_out,
                                const dip_debug* dbg, void* ws, size_t ws_bytes, void* stream);

/*
 * Row-gathered dot products: out[t] = W[idx[t], :] . x  for t < k, fp32 accumulation in a
 * fixed order -- what is left of W x when a mask removes rows of W (Sec. 3.2, the W^u of
 * gate pruning).
 *   w_rows   neuron-major matrix: n_in stored rows of n_out elements (n_out <= DIP_MAX_N)
 *   x        n_out floats, 16-byte aligned     idx   k ascending stored-row indices
 *   out      k floats
 */
int32_t dip_gathered_rowdot(const dip_weight* w_rows, const float* x, const int32_t* idx, int32_t k,
                            float* out, void* stream);

/*
 * Gate pruning and Up pruning, Sec. 3.2, one token through one MLP:
 *   1. a = SiLU(W^g x)  (gate)   or   a = W^u x  (up)        dense, all d_ff units, fp32
 *   2. m = topK(|a|, k)                                       lowest index wins ties
 *   3. h_j = (W^u x)_j a_j  (gate)   or   a_j SiLU((W^g x)_j)  (up)      for j in m only
 *   4. y = sum_{j in m} W^d[:, j] h_j
 * The fp32 array a is both the selection key and the factor in step 3.
 *   x     d_model floats, 16-byte aligned      y_out   d_model floats     1 <= k <= d_ff
 *   dbg   NULL or stage outputs                ws      *_workspace_bytes() bytes, 256-aligned
 */
size_t dip_partial_pruning_forward_workspace_bytes(const dip_mlp_split* mlp, int32_t k);
int32_t dip_partial_pruning_forward(const dip_mlp_split* mlp, int32_t scheme, const float* x,
                                    int32_t k, float* y_out, const dip_partial_debug* dbg,
                                    void* ws, size_t ws_bytes, void* stream);

/*
 * Two-tier residency made real (Sec. 5, Fig. 4; Alg. 1's c decides what the fast tier holds).
 * dip_tier_init: after dip_cache_init, give every resident column a slot (the r-th resident
 * column, ascending, gets slot r), copy those rows host -> HBM, mark the others slot_of = -1.
 * dip_tiered_mlp_forward: dip_swiglu_mlp_forward with both caches mandatory, where after each
 * cache update the inserted columns take over the slots of the evicted ones (i-th inserted,
 * ascending, <- slot of the i-th evicted; the rest get slots never used before), their rows
 * are copied host -> HBM, and the gathered product reads resident columns from their slots
 * and the misses that found no room (Sec. 6.4) straight from host memory.  y is bit-identical
 * to dip_swiglu_mlp_forward on the same inputs and cache states.
 */
size_t dip_tier_init_workspace_bytes(const dip_tiered_weight* tw);
int32_t dip_tier_init(const dip_tiered_weight* tw, const dip_cache* cache, void* ws, size_t ws_bytes,
                      void* stream);
size_t dip_tiered_mlp_forward_workspace_bytes(const dip_tiered_mlp* mlp, int32_t k_in, int32_t k_mid);
int32_t dip_tiered_mlp_forward(const dip_tiered_mlp* mlp, const float* x, int32_t k_in, int32_t k_mid,
                               const dip_cache* cache_in, const dip_cache* cache_mid, float gamma,
                               float* y_out, const dip_debug* dbg, void* ws, size_t ws_bytes,
                               void* stream);

/* ------------------------------------------------------------------------------------------
 * Around the MLP: one (speculative) decode step over a paged key/value cache
 *
 * A step takes `n_batch` sequences and, of each, a few new rows: the next token alone, a piece
 * of a prompt, or a tree of drafted tokens whose node 0 is the last token the sequence has
 * (at most DIP_MAX_TREE nodes).  dip_kv_reserve makes room for the rows, dip_kv_append writes
 * a layer's keys and values of them, dip_window_attention / dip_tree_attention attend,
 * dip_verify_tree says which drafts stand, dip_kv_compact keeps those and commits.
 * ------------------------------------------------------------------------------------------ */

/* A paged key/value cache, owned by the caller.  Element (layer l, page p, head h, slot s, dim d)
 * of k and of v lies l * layer_stride + p * page_stride + h * head_stride + s * slot_stride + d
 * elements from its start, so that heads may come before slots or behind them; all starts and
 * strides are multiples of 16 bytes.  Position i of sequence q is slot i % page_size of page
 * page_table[q * max_pages + i / page_size].
 * page_table, seq_len and page_refs are written by the calls below and read by whoever likes.
 * A table entry or sequence number outside its range is never followed out of bounds: rows that
 * would be written there are dropped, and what is read there is taken from page 0. */
typedef struct dip_kv_cache {
    void* k;              /* device                                                          */
    void* v;              /* device; the same type and strides                               */
    int32_t* page_table;  /* device; n_seqs * max_pages entries, -1: no page                 */
    int32_t* seq_len;     /* device; n_seqs: committed tokens of each sequence               */
    int32_t* page_refs;   /* device; n_pages: table entries that name the page, 0: free      */
    int32_t dtype;        /* DIP_F32 or DIP_BF16                                             */
    int32_t n_layers;
    int32_t n_pages;
    int32_t page_size;    /* slots of a page, a power of two in [1, 4096]                    */
    int32_t n_kv_heads;   /* page_size * n_kv_heads * head_dim < 2^30                        */
    int32_t head_dim;     /* a multiple of 16 bytes; the attention calls: 64, 96 or 128      */
    int32_t n_seqs;
    int32_t max_pages;    /* of one sequence; max_pages * page_size <= 2^31 - 2^25           */
    int64_t layer_stride; /* in elements                                                     */
    int64_t page_stride;
    int64_t head_stride;
    int64_t slot_stride;
} dip_kv_cache;

/* The rows of one step.  Entry b is sequence seqs[b] with rows row_start[b] .. row_start[b+1] - 1
 * of every row-indexed array; its row t stands at position seq_len + t (in a tree: node t).  The
 * host fields size the launches: rows of an entry beyond max_rows, and rows from n_rows on, are
 * not looked at, and of a sequence longer than max_len (its new rows included), or than its table,
 * positions from there on are seen by nobody. */
typedef struct dip_batch {
    const int32_t* seqs;      /* device; n_batch distinct sequences (dip_verify_tree: may be NULL)  */
    const int32_t* row_start; /* device; n_batch + 1 entries, ascending from 0 to n_rows            */
    int32_t n_batch;          /* 1 .. DIP_MAX_BATCH                                                 */
    int32_t n_rows;           /* rows of all entries, >= 1                                          */
    int32_t max_rows;         /* most rows of one entry, >= 1                                       */
    int32_t max_len;          /* most tokens of one sequence after this step (0: what fits the table) */
} dip_batch;

#define DIP_MAX_BATCH 1024
#define DIP_MAX_TREE 64

/* Every page free, every sequence empty (page_refs, page_table and seq_len are written; k and v are not). */
int32_t dip_kv_init(const dip_kv_cache* cache, void* stream);

/* Give up all pages of the n listed sequences (device array; a page is free when nobody holds it) and
 * make them empty.  Entries outside [0, n_seqs) are skipped, repeated ones count once. */
int32_t dip_kv_free(const dip_kv_cache* cache, const int32_t* seqs, int32_t n, void* stream);

/* Sequence dst[i] becomes a copy of sequence src[i] that shares its pages (up to seq_len tokens),
 * i < n (device arrays).  The destinations hold no pages (as after dip_kv_init or dip_kv_free) and are
 * distinct, and none is a source; several may have one source. */
int32_t dip_kv_fork(const dip_kv_cache* cache, const int32_t* src, const int32_t* dst, int32_t n, void* stream);

/* Copy whole pages, all layers, k and v: page src[i] to page dst[i], i < n (device arrays; the
 * destinations are distinct and none is a source; pairs out of range are skipped).  Tables and
 * counts stay as they are. */
int32_t dip_kv_copy_pages(const dip_kv_cache* cache, const int32_t* src, const int32_t* dst, int32_t n, void* stream);

/*
 * Make room for the rows of a step: every entry gets pages of its own for positions seq_len ..
 * seq_len + rows - 1.  A table entry without a page takes a free one; a page that other sequences
 * hold too when the call starts is exchanged for a free one, and what the entry has of it is copied
 * (copy on write; all layers).  The lowest free pages are given out, to the entries in order and to
 * each in order of position.  An entry whose pages, with all that earlier entries asked for, exceed the
 * free ones (or whose rows do not fit the table) gets none and its table stays.
 * granted[b] = 1 if, in the end, all rows of entry b have pages that no other sequence holds, be they new,
 * its own before, or left to it by the others that held them; otherwise granted[b] = 0, and until room is made for
 * it the entry's rows are passed over by dip_kv_append and dip_kv_compact, and what attention gives for
 * them is unspecified.  Calling it again for the same rows changes nothing if all entries were granted theirs.
 *   granted  n_batch words or NULL      ws  *_workspace_bytes() bytes, 256-aligned
 */
size_t dip_kv_reserve_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch);
int32_t dip_kv_reserve(const dip_kv_cache* cache, const dip_batch* batch, int32_t* granted, void* ws,
                       size_t ws_bytes, void* stream);

/*
 * Write keys and values of the step's rows into layers layer .. layer + n_layers - 1.  Row r of
 * layer l: n_kv_heads * head_dim elements at l * new_layer_stride + r * row_stride of k_new and
 * v_new (elements; multiples of 16 bytes; l counts from 0).  seq_len stays (dip_kv_compact commits).
 * An entry of which some row has no page, or one that another sequence holds too (dip_kv_reserve granted it
 * nothing, or it was forked since), is passed over whole.
 */
int32_t dip_kv_append(const dip_kv_cache* cache, int32_t layer, int32_t n_layers, const dip_batch* batch,
                      const void* k_new, const void* v_new, int64_t row_stride, int64_t new_layer_stride,
                      void* stream);

/* ---- rows turned to their positions ---- */

/* How a head is turned to position pos.  Pair i < dims / 2, (a, b), becomes
 *     scale * (a cos t - b sin t,  a sin t + b cos t),   t = pos * freq[i];
 * what lies behind the first `dims` dims passes through.  Angles are worked out in 64 bits and reduced to a
 * part of a turn before their sine and cosine are taken in fp32, so that far positions are as exact as near
 * ones; products and sums are fp32, rounded once. */
#define DIP_ROTARY_HALF 0        /* pair i: dims i and i + dims / 2                             */
#define DIP_ROTARY_INTERLEAVED 1 /* pair i: dims 2 i and 2 i + 1                                */
typedef struct dip_rotary {
    const double* freq; /* device; dims / 2 angles per position, radians                    */
    int32_t dims;       /* even, 2 .. the head's dims, at most DIP_MAX_ROTARY_DIMS          */
    int32_t layout;     /* DIP_ROTARY_HALF or DIP_ROTARY_INTERLEAVED                        */
    float scale;        /* of sines and cosines; 1 but for methods that ask for more        */
    int32_t reserved;   /* must be 0                                                        */
} dip_rotary;
#define DIP_MAX_ROTARY_DIMS 4096

/* Angles per position, f_i = base^(-2 i / dims), and as they are scaled for contexts longer than a model
 * was trained on. */
#define DIP_SCALING_NONE 0
#define DIP_SCALING_LINEAR 1 /* f_i / factor (position interpolation)                            */
#define DIP_SCALING_BASE 2   /* base * factor^(dims / (dims - 2)) in place of base               */
#define DIP_SCALING_PARTS 3  /* f_i (m + (1 - m) / factor), m = (turns - slow) / (fast - slow) within [0, 1],
                                turns = original_len f_i / 2 pi: quick pairs stay, slow ones are stretched */
#define DIP_SCALING_LIST 4   /* f_i / factors[i]                                                 */
typedef struct dip_rotary_scaling {
    int32_t kind;
    int32_t reserved;       /* must be 0                                                    */
    double factor;          /* > 0: LINEAR, BASE, PARTS                                     */
    double slow, fast;      /* 0 <= slow < fast: PARTS                                      */
    double original_len;    /* > 0: PARTS                                                   */
    const double* factors;  /* host; dims / 2 entries > 0: LIST                             */
} dip_rotary_scaling;

/* freq: host, dims / 2 entries.  scaling: host, NULL for none.  Angles (or a scaled base) beyond the finite numbers are refused.
 * Host only; nothing is enqueued. */
int32_t dip_rotary_frequencies(int32_t dims, double base, const dip_rotary_scaling* scaling /* host */,
                               double* freq /* host */);

/*
 * Rows turned to given positions: row r of out = row r of x at positions[r] (device; any int32, negative ones turn
 * back).  n_rows rows of n_heads * head_dim elements (DIP_F32 or DIP_BF16; a head a multiple of 16 bytes), x_stride /
 * out_stride elements apart (multiples of 16 bytes).  out may be x itself (equal pointers and strides), but may not overlap it in another way.
 */
int32_t dip_rotate_rows(const dip_rotary* rot, const void* x, int64_t x_stride, const int32_t* positions, int32_t n_rows,
                        int32_t n_heads, int32_t head_dim, int32_t dtype, void* out, int64_t out_stride, void* stream);

/*
 * dip_kv_append for one layer, with the step's queries and keys turned on the way: keys go into the cache
 * turned, values as they are, queries to q_out.  Row t of an entry is turned to position seq_len + t; with
 * parents (as in dip_tree_attention; NULL: none) to seq_len + its depth, an absent node to seq_len.
 * Which entries are passed over follows dip_kv_append; the queries of an entry that is passed over are turned all
 * the same, those of an entry whose sequence number is out of range are not written.
 *   q, q_out   n_rows rows of n_q_heads * head_dim elements of the cache's type, strides in elements
 *              (multiples of 16 bytes); q_out may be q itself, and overlaps neither it in another way nor k_new
 *              or v_new.  q and q_out NULL, n_q_heads 0: keys and values alone
 *   k_new, v_new   as in dip_kv_append: n_kv_heads * head_dim elements at r * row_stride
 */
int32_t dip_kv_append_rotary(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const int32_t* parents,
                             const dip_rotary* rot, const void* q, int64_t q_stride, int32_t n_q_heads, void* q_out,
                             int64_t q_out_stride, const void* k_new, const void* v_new, int64_t row_stride, void* stream);

/*
 * Keep keep[b] rows of every entry (device; values are clamped to its rows; NULL: all of them) and
 * commit: row path[row_start[b] + j] of the entry moves to row j, j < keep[b], in every layer (path:
 * device, n_rows entries, ascending within an entry, path[j] >= j; NULL: the first keep[b] rows
 * stay where they are), seq_len += keep[b], and pages beyond the new length are given up.  An
 * entry that dip_kv_append passes over keeps nothing: its length stays.
 */
int32_t dip_kv_compact(const dip_kv_cache* cache, const dip_batch* batch, const int32_t* path, const int32_t* keep,
                       void* stream);

/*
 * Attention of a step's rows over the cache, their own keys and values already in it.  Query head h
 * attends with key/value head h / (n_q_heads / n_kv_heads):
 *     out[r, h] = sum_j p_j v_j,   p = softmax over the visible j of scale * q[r, h] . k_j
 * dip_window_attention: row t of an entry stands at pos = seq_len + t and sees
 *     j <= pos  and  (j > pos - window  or  j < sinks).
 * dip_tree_attention: parents[r] is the entry's node that drafted node t (-1: none, any other value
 * outside [0, t): the node is absent, as are the nodes below an absent one); node t stands at pos =
 * seq_len + its depth, sees the ancestors that are nodes of the tree and itself, and of the committed
 * positions j < seq_len those with  j > pos - window  or  j < sinks.  A window shorter than the tree does not cut its
 * ancestors: a node that deep sees more than the same token would one at a time.
 * window 0 means no bound (sinks then change nothing).  A row that sees nothing, an absent node, and a row
 * whose scores are all -inf get zeros.  Positions that a row does not see do not matter to it, whatever they hold.
 * A value that is not finite at a position that a row sees makes that channel of the row what the sum gives
 * (infinite, or NaN where a NaN or both infinities meet, or where its weight vanishes in fp32); the other channels are as
 * they were.
 *   q, out   n_rows rows of n_q_heads * head_dim elements of the cache's type, q_stride / out_stride
 *            elements apart (multiples of 16 bytes); out may not overlap q
 *   scale > 0      n_q_heads a multiple of n_kv_heads      ws  *_workspace_bytes() bytes, 256-aligned
 * Scores, softmax statistics and sums are fp32; with a DIP_BF16 cache the weights p enter their product
 * with v as the sum of two bf16 terms (exact to 2^-15), and the output is rounded once.  Which kernel runs is chosen
 * by max_rows and the query heads per key/value head, for all entries of a call: many single tokens are faster in a
 * call without a prompt's rows among them.  The order of the sums is fixed
 * by shapes, all entries' rows and lengths, and max_len (bit-repeatable).
 */
size_t dip_attention_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch, int32_t n_q_heads,
                                     int32_t window, int32_t sinks);
int32_t dip_window_attention(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const void* q,
                             int64_t q_stride, int32_t n_q_heads, float scale, int32_t window, int32_t sinks,
                             void* out, int64_t out_stride, void* ws, size_t ws_bytes, void* stream);
int32_t dip_tree_attention(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const int32_t* parents,
                           const void* q, int64_t q_stride, int32_t n_q_heads, float scale, int32_t window,
                           int32_t sinks, void* out, int64_t out_stride, void* ws, size_t ws_bytes, void* stream);

/* ---- blocks of a long context ----
 * Attention that reads, of each row's past, a few blocks chosen by the row itself.  A block is `block` positions from a
 * multiple of `block` on: a power of two from 16 to the page size.  Of a sequence with `len` committed positions (the first
 * max_len of them) are read
 *     [0, front),       front = sinks, rounded up to whole blocks (and no more than tail),
 *     the chosen blocks of [front, tail),
 *     [tail, len),      tail = min(len - recent, the end of its last complete page), rounded down to whole blocks, >= 0,
 * and the step's own rows, as in dip_window_attention (up to the row itself) or dip_tree_attention (a node's ancestors).
 * So blocks are chosen from complete pages alone, whose positions no step changes.
 */

/* Bounds of the keys of every block, owned by the caller: of the cache's type, contiguous, 16-byte aligned,
 *     [n_layers][n_pages][n_kv_heads][page_size / block][2][head_dim],
 * the smallest number of each channel, then the largest (NaN not counted, an infinity as the largest finite number of its
 * sign; 0 and 0 where there is none).  They belong to the page, whichever sequences share it. */
size_t dip_block_bounds_bytes(const dip_kv_cache* cache, int32_t block);

/*
 * Work out the bounds of layers layer .. layer + n_layers - 1 for the complete pages of the n listed sequences (device
 * array, at most 65535; numbers out of range are skipped) that hold some of their last `back` committed positions (0: all of them).
 * To be called when positions were committed, with back as many as that (at least); pages copied by dip_kv_copy_pages take
 * theirs by a call like this too.
 */
int32_t dip_kv_block_bounds(const dip_kv_cache* cache, int32_t layer, int32_t n_layers, const int32_t* seqs, int32_t n,
                            int32_t back, int32_t block, void* bounds, void* stream);

/*
 * Choose blocks for every row and key/value head: of the blocks in [front, tail) the n_select (or all, if there are no more) with
 * the largest
 *     score = max over the query heads of the group of  sum_d max(q_d lo_d, q_d hi_d),
 * an upper bound of q . k over the block's keys; equal scores, the lower block first.  Sums are fp64, rounded
 * once to fp32; a sum that is NaN counts as -inf.
 *   q        as in dip_window_attention
 *   blocks   [n_rows][n_kv_heads][n_select], ascending, then -1; rows of an entry whose sequence is out of range: -1
 *   n_select 1 .. DIP_MAX_SELECT        sinks, recent >= 0        ws  *_workspace_bytes() bytes, 256-aligned
 */
#define DIP_MAX_SELECT 4096
size_t dip_select_blocks_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch, int32_t n_q_heads, int32_t block);
int32_t dip_select_blocks(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const void* q, int64_t q_stride,
                          int32_t n_q_heads, int32_t block, const void* bounds, int32_t n_select, int32_t sinks,
                          int32_t recent, int32_t* blocks, void* ws, size_t ws_bytes, void* stream);

/*
 * Attention over what the blocks leave: arguments, softmax, rounding and what is not finite as in dip_window_attention (parents
 * NULL) or dip_tree_attention.  blocks: as dip_select_blocks writes them, or of the caller's own making: ascending, unused
 * entries, -1, at the end; an entry outside [front, tail) or not above the one before it is passed over, and all others are read.
 * (So a list that is not ascending may read a block more than once: 5, 3, 5 reads block 5 twice.)
 * Every row reads its own blocks: meant for single tokens, trees and a few rows; the many rows of a prompt share what they
 * read in dip_window_attention.
 */
size_t dip_block_attention_workspace_bytes(const dip_kv_cache* cache, const dip_batch* batch, int32_t n_q_heads, int32_t block,
                                           int32_t n_select, int32_t sinks, int32_t recent);
int32_t dip_block_attention(const dip_kv_cache* cache, int32_t layer, const dip_batch* batch, const int32_t* parents,
                            const int32_t* blocks, int32_t n_select, int32_t block, const void* q, int64_t q_stride,
                            int32_t n_q_heads, float scale, int32_t sinks, int32_t recent, void* out, int64_t out_stride, void* ws,
                            size_t ws_bytes, void* stream);

/*
 * Verification of drafted trees (entries and parents as in dip_tree_attention, at most DIP_MAX_TREE
 * nodes).  Node t carries tokens[r]; p[r] is the target's distribution behind node t and q[r] the one
 * its children were drawn from, independently.  From node 0 on, the children of a node are tried in
 * order, child j (from 0) with its number u[r] in [0, 1):
 *     taken iff  u q(x) G_j < (p(x) - lam_j q(x))+ ,   lam_0 = 0, G_0 = 1,
 *     lam_{j+1} = lam_j + G_j,   G_j = sum_x (p(x) - lam_j q(x))+  for j >= 1,
 * which is the rule  r <- norm((r - q)+) after each refused child: the j-th r is (p - lam_j q)+ / G_j.
 * A child that is taken is the next node; where none is (m children), the next token is the first x with
 *     sum_{y <= x} w(y) > u_sample[b] * sum w,   w = (p - lam_m q)+  (p itself where that is all zero).
 *   p, q       n_rows rows of n_vocab probabilities (both DIP_F32 or DIP_BF16), p_stride / q_stride
 *              elements apart
 *   max_kids   1 .. DIP_MAX_TREE - 1: children of a node beyond that many are passed over
 *   keep       n_batch: nodes that stand, node 0 among them (0: the entry has no rows, or its node 0
 *              is no root)
 *   path       n_rows: the nodes that stand, then -1            token   n_batch: -1 where keep is 0 or
 *              p has no positive entry
 * Sums and comparisons are in 64 bits.  A token outside [0, n_vocab) is never taken.
 *   ws  *_workspace_bytes() bytes, 256-aligned
 */
size_t dip_verify_tree_workspace_bytes(const dip_batch* batch, int32_t n_vocab, int32_t max_kids);
int32_t dip_verify_tree(const dip_batch* batch, const int32_t* tokens, const int32_t* parents, const void* p,
                        int64_t p_stride, const void* q, int64_t q_stride, int32_t dtype, int32_t n_vocab,
                        const float* u, const float* u_sample, int32_t max_kids, int32_t* keep, int32_t* path,
                        int32_t* token, void* ws, size_t ws_bytes, void* stream);

/*
 * From logits to tokens, and to the probabilities that dip_verify_tree takes.  Row r: the words are ordered by their
 * logits l, the largest first, equal ones by number, and weigh w(x) = exp((l(x) - l(first)) / temperature).  Kept are
 *     the first top_k of them (top_k <= 0: all),
 *     of these the fewest first ones whose weights come to top_p of what all of these weigh, and one at least
 *     (top_p >= 1 or NaN: all),
 *     of these the ones with w >= min_p (min_p <= 0 or NaN: all; above 1 counts as 1).
 * token[r] = the first x, in order of the words' numbers, at which the running sum of the kept weights exceeds u[r] times
 * their sum; probs[r] = the kept weights divided by their sum, 0 elsewhere.  A temperature that is not above 0 keeps
 * the first word alone.  A logit of -inf is never kept, NaN counts as -inf; +inf outweighs all that is finite, and several
 * share alike.  A row of nothing but -inf gives -1 and zeros.
 * Weights are accurate to 2^-26 + 2^-50 |l / temperature| and summed in integers or fp64, so that results do not hang on the
 * order of sums (bit-repeatable).  A word whose l / temperature is 63.75 or more below the first's, its weight 2^-91 and less, may
 * count for nothing in the sums; it is not drawn then, whatever u, but keeps its probability.
 *   logits   n_rows (at most 65535) rows of n_vocab (at most 2^24), DIP_F32 or DIP_BF16, `stride` elements apart
 *   how      host; per-row settings, device arrays of n_rows entries; a NULL array, or NULL for all: none of it (temperature 1)
 *   u        n_rows numbers in [0, 1); may be NULL if token is
 *   token    n_rows, or NULL     probs    n_rows rows of n_vocab, DIP_F32 or DIP_BF16, probs_stride elements apart, or NULL;
 *            may be logits itself (same type and stride), but may not overlap it in another way
 *   ws       *_workspace_bytes() bytes, 256-aligned
 */
typedef struct dip_sampling {
    const float* temperature; /* device */
    const int32_t* top_k;     /* device */
    const float* top_p;       /* device */
    const float* min_p;       /* device */
} dip_sampling;
size_t dip_sample_workspace_bytes(int32_t n_rows, int32_t n_vocab);
int32_t dip_sample(const void* logits, int64_t stride, int32_t dtype, int32_t n_rows, int32_t n_vocab,
                   const dip_sampling* how /* host */, const float* u, int32_t* token, void* probs, int64_t probs_stride,
                   int32_t probs_dtype, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DIP_H_ */
