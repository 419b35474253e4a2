/*
 * mmee.h -- C ABI of the MI355X (gfx950) implementation of the hot path of MMEE,
 * "Matrix Multiplication Encoded Enumeration" (Fast Cross-Operator Optimization
 * of Attention Dataflow): exhaustive, pruned evaluation of the paper's analytical
 * buffer/DRAM/energy/latency model (Sec. V) over every fused-attention dataflow
 * (Sec. III-IV: tiling, loop order, buffering levels, recomputation, stationary
 * modes, fused or unfused softmax) and reduction to the optimum (Sec. VI).
 *
 * Conventions
 *  - Two chained matmuls per head (Sec. III-A):  C[i,l] = sum_k A[i,k] B[k,l],
 *    E[i,j] = sum_l C[i,l] D[l,j];  for attention A=Q, B=K^T, D=V, E=O, so the
 *    loop extents are I = L = N and K = J = d.  Dimensions are indexed
 *    i=0, k=1, l=2, j=3 everywhere.  Each extent is split in two levels,
 *    X = x_D * x_G: inter-tile count times intra-tile size (Sec. IV-A).
 *  - A candidate is one index in [0, space).  Mixed-radix digits, least
 *    significant first:
 *        t_i, t_k, t_l, t_j   position of x_G in the ascending divisor list of I,K,L,J
 *        p_A, p_B, p_D, p_E   buffering level 0..4 = number of innermost inter-tile
 *                             loops the operand's buffer spans (0 = one tile; the
 *                             paper's layers L3..L7, Sec. IV-B)
 *        order  0..23         lexicographic rank of the inter-tile loop sequence,
 *                             written outer -> inner over the symbols i<k<l<j
 *        r      0..1          recomputation of C tiles (Sec. III-C)
 *        s1,s2  0..2          stationary mode of Op1 / Op2: 0 weight, 1 input, 2 output (Sec. V-D)
 *        f      0..1          1 = softmax fused (C stays on chip), 0 = C staged through DRAM
 *    so space = (#tilings) * 540000.
 *  - All pointers are HOST pointers unless stated otherwise.  The library keeps
 *    none of them after a call returns.  Device scratch is cached inside the
 *    library and released by mmee_shutdown().
 *  - Every function returns 0 on success or a negative MMEE_E* code; nothing is
 *    thrown across this boundary.  Calls are serialised by an internal lock.
 *  - All the arithmetic runs in HIP kernels on the current HIP device; there is
 *    no CPU fallback: without a usable GPU the calls return MMEE_EDEVICE.
 */
#ifndef MMEE_H
#define MMEE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Attention workload (Sec. II-A): B batches of H heads, sequence length N, head dim d. */
typedef struct mmee_workload {
    uint32_t B, H, N, d;
    uint32_t word_bytes;    /* bytes per element, 2 for fp16                              */
    uint32_t tiling_mode;   /* 0: x_G ranges over power-of-two divisors, 1: all divisors   */
    uint32_t c_softmax;     /* softmax cost per element of C in MAC-energy units (Sec. V-D; the paper uses 10) */
    uint32_t reserved;      /* must be 0                                                   */
} mmee_workload;

/* Two chained matrix multiplications of free shape (Sec. VII-J, Table V: two GEMMs, or a
 * convolution chain turned into GEMMs by im2col): Op1 is I x K x L, Op2 is I x L x J, `batch`
 * independent instances.  An attention workload is the chain I = L = N, K = J = d, batch = B*H;
 * every mmee_* call on a workload is the mmee_chain_* call on that chain. */
typedef struct mmee_chain {
    uint32_t batch;
    uint32_t I, K, L, J;
    uint32_t word_bytes;
    uint32_t tiling_mode;   /* as in mmee_workload                                         */
    uint32_t c_softmax;     /* 0 when nothing sits between the two operators               */
} mmee_chain;

/* Spatial accelerator (Sec. II-B): PE arrays with register files, one global buffer, DRAM. */
typedef struct mmee_hw {
    uint32_t pe_rows, pe_cols;  /* one PE array                                            */
    uint32_t n_arrays;          /* heads are spread over the arrays (Sec. V)               */
    uint32_t rf_bytes;          /* register file per PE; half of it holds stationary data  */
    uint64_t gb_bytes;          /* global buffer capacity: BS * word_bytes <= gb_bytes     */
    double e_dram, e_gb, e_rf, e_mac;   /* pJ per word access at each level, pJ per MAC     */
    double dram_bw, gb_bw;      /* bytes per cycle; 0 drops that stream from the latency   */
} mmee_hw;

/* One decoded candidate (Sec. IV-A: loop boundaries, loop order, buffering levels). */
typedef struct mmee_mapping {
    uint64_t idx;
    uint32_t xG[4], xD[4];      /* i,k,l,j                                                 */
    uint8_t order[4];           /* inter-tile loops, outer -> inner, values 0..3 = i,k,l,j */
    uint8_t level[4];           /* p_A, p_B, p_D, p_E                                      */
    uint8_t recompute, stat1, stat2, fused;
} mmee_mapping;

/* Cost of one candidate.  The integer fields are per head (the model omits the head
 * dimension, Sec. V); energy and latency cover all B*H heads.  64 bytes. */
typedef struct mmee_cost {
    uint64_t bs_words;          /* buffer size requirement, Eq. (4)                        */
    uint64_t da_words;          /* DRAM access, Eq. (7) (+ DA_C when f = 0)                */
    uint64_t br_words;          /* buffer <-> register-file traffic                        */
    uint64_t mac_total;         /* N_op1 + N_op2, or j_D*N_op1 + N_op2 with recomputation  */
    uint64_t comp_cycles;       /* compute cycles on one array                             */
    double energy_pj;           /* +inf when valid == 0                                    */
    double latency_cycles;      /* +inf when valid == 0                                    */
    uint32_t valid;             /* 1 = feasible dataflow                                   */
    uint32_t reason;            /* 0 ok; 1 not a dataflow (r=1 with k outside j, or r=1 with f=0):
                                   all integer fields are 0; 2 exceeds the buffer capacity */
} mmee_cost;

typedef struct mmee_result {
    mmee_mapping best;
    mmee_cost cost;
    uint64_t space;             /* size of the index space                                 */
    uint64_t evaluated;         /* candidates the search decided over: costed, or settled without (over the
                                   buffer capacity, which costs +inf; over the surviving rows also those
                                   of a tiling that move more DRAM words than another one that fits) */
    double seconds;             /* host wall time of the call (upload, kernels, readback)  */
    double kernel_seconds;      /* device time of the search's kernels: by HIP events (start of the first
                                   to end of the last launch), or, where a call of one problem ends
                                   without events, by the device's clock from the first block to the last
                                   record (most pruned and most exhaustive searches of one problem, fronts
                                   over the surviving rows): some microseconds less          */
} mmee_result;

/* Counts of the offline stage (Sec. VI-B): loop-order x buffering-level rows per
 * (recompute, fused) group before and after symbolic pruning.  Group g = r + 2 f. */
typedef struct mmee_row_stats {
    uint32_t rows_total[4];     /* 15000 each                                              */
    uint32_t rows_valid[4];     /* rows that denote a dataflow                             */
    uint32_t rows_kept[4];      /* survivors of the dominance test                         */
} mmee_row_stats;

enum {
    MMEE_OBJ_ENERGY = 0,                /* key (energy, idx)            */
    MMEE_OBJ_LATENCY = 1,               /* key (latency, idx)           */
    MMEE_OBJ_LATENCY_THEN_ENERGY = 2,   /* key (latency, energy, idx)   */
    MMEE_OBJ_EDP = 3                    /* key (energy * latency, idx), the energy-delay product (Sec. VII-K) */
};

enum {
    MMEE_SEARCH_PRUNED = 0,             /* offline symbolic pruning on (the paper's method) */
    MMEE_SEARCH_EXHAUSTIVE = 1,         /* cost every candidate that denotes a dataflow (one that
                                           exceeds the buffer capacity costs +inf, whatever
                                           else it costs)                                   */
    /* When the four energies per access are whole numbers and the largest possible total stays
     * below 2^53, every term of the energy is an exact integer and the search adds a (row, tiling)
     * part and a (tiling, stationary modes) part per candidate; the result has the same bits as
     * the sum taken term by term in the order of Sec. V-D.  When only the size condition fails,
     * the searches for the energy, the latency and the (latency, energy) key still start that way
     * and keep the outcome if the optimal energy found is below 2^52 pJ: every candidate whose total
     * reaches 2^53 computes to more than that in either order, all others are exact, so the optimum
     * and its ties are those of the term-by-term sum; otherwise the search is repeated term by term.
     * This flag (may be or-ed with the others) keeps the term-by-term order in every case. */
    MMEE_SEARCH_ORDERED_SUM = 2
};

enum {
    MMEE_OK = 0,
    MMEE_EINVAL = -1,       /* null pointer, zero dimension, unsupported size, bad enum       */
    MMEE_ERANGE = -2,       /* index range outside [0, space)                                 */
    MMEE_ENOFEASIBLE = -3,  /* every candidate is masked; out->cost.valid = 0                 */
    MMEE_EDEVICE = -4,      /* HIP error or no device                                         */
    MMEE_EOVERFLOW = -5,    /* mmee_pareto: more front points than `capacity`                 */
    MMEE_ETOOBIG = -6,      /* mmee_search_noalloc: the problem exceeds its fixed scratch     */
    MMEE_EWORKSPACE = -7    /* a call with a mmee_*_workspace of its own: no workspace, or one smaller than asked for */
};

/* Number of candidates of (workload, hw): #tilings (integer factorisations, Sec. VI-A)
 * times 540000.  Pure host arithmetic. */
int mmee_space_size(const mmee_workload *w, const mmee_hw *hw, uint64_t *out);

/* *out = 1 when every search of (workload, hw) under these flags adds the energy regrouped (see
 * MMEE_SEARCH_ORDERED_SUM) and the sum is exact for every candidate beforehand: whole-number energies per
 * access, total energy of any candidate (Sec. V-D) below 2^53, and a power-of-two DRAM bandwidth and
 * array count; else 0.  With another bandwidth or array count only some searches regroup (the energy
 * key alone, and those of the full row set that take one or two keys per pass).  Results have the
 * same bits either way.  Pure host arithmetic. */
int mmee_energy_regrouped(const mmee_workload *w, const mmee_hw *hw, uint32_t flags, int *out);

/* On-device mixed-radix decode of n candidate indices (host arrays in and out): index -> loop
 * boundaries, loop order, buffering levels and options, the components of a pseudo nested loop
 * (Sec. IV-A).  A helper next to the three calls of the problem statement. */
int mmee_decode(const mmee_workload *w, const mmee_hw *hw, const uint64_t *idx, uint64_t n,
                mmee_mapping *out);

/* Cost of the n consecutive candidates first_idx .. first_idx+n-1 (Sec. V, Eq. (1)-(7),
 * energy and latency of Sec. V-D).  out_costs holds n records and may be host memory or
 * device memory of the current device (detected); device results are not copied back. */
int mmee_eval_batch(const mmee_workload *w, const mmee_hw *hw, uint64_t first_idx, uint64_t n,
                    mmee_cost *out_costs);

/* Optimal mapping under one objective; ties go to the lowest index (Sec. VI).
 * mmee_search uses the pruned row set.
 * A call of one problem, and a front over the surviving rows, keep a core of the host busy until the result is
 * there, for 20 ms at most; what takes longer (work of the caller's ahead of it on the stream) is then
 * waited for on the stream, as in the other calls.  Calls take turns: another thread's begins when this one returns. */
int mmee_search(const mmee_workload *w, const mmee_hw *hw, int objective, mmee_result *out);
int mmee_search_ex(const mmee_workload *w, const mmee_hw *hw, int objective, uint32_t flags,
                   mmee_result *out);

/* One pass over the space that reduces n_obj (1..4, distinct) objectives at once: all
 * metrics of a candidate are formed once and shared (Sec. VII-D).  out holds n_obj results. */
int mmee_search_multi(const mmee_workload *w, const mmee_hw *hw, const int *objectives,
                      uint32_t n_obj, uint32_t flags, mmee_result *out);

/* A helper for sweeps over hardware designs and sequence lengths (Sec. VII-I, Table IV; Sec. VII-H):
 * count independent searches (arrays of count workloads, hws, objectives, results) enqueued
 * back to back on one stream with a single synchronisation at the end.  Neighbouring entries
 * with identical workload and hw share one pass.  Pruned passes of problems on the same shape may
 * share the part of the search that hangs on the shape and the buffer capacity, whatever their keys; else
 * pruned passes for one key, or for energy and latency together, share kernel launches across
 * problems (one per kind of pass present).  Which way costs less is estimated per call from the
 * numbers of shapes, problems and tilings.  The remaining passes run problem by problem.
 * mmee_result::kernel_seconds of a pass that shared launches is the device time of all the
 * launches it shared.  Returns the first non-zero
 * per-entry code (per-entry codes are stored in rc[i] when rc is not null). */
int mmee_search_many(const mmee_workload *w, const mmee_hw *hw, const int *objectives,
                     uint32_t count, uint32_t flags, mmee_result *out, int *rc);

/* Energy-latency Pareto front (Sec. VI-A, Sec. VII-E): the feasible candidates that no other
 * candidate beats in both metrics; among candidates with identical (energy, latency) the lowest
 * index stands for all.  out receives at most `capacity` points by ascending latency (descending
 * energy), *n_points their number.  Over the surviving rows of a problem of at most 32768 tilings the
 * front comes out of one pass over the space; otherwise each point costs a pass.  `evaluated` counts
 * a pass per point and one that finds nothing more, either way.  Returns MMEE_EOVERFLOW (with the
 * first `capacity` points stored) when the front is longer. */
int mmee_pareto(const mmee_workload *w, const mmee_hw *hw, uint32_t flags, mmee_result *out,
                uint32_t capacity, uint32_t *n_points);

/* DRAM access versus buffer size requirement (Sec. VII-C): the dataflows that no other dataflow
 * beats in both Eq. (4) and Eq. (7), whatever the buffer capacity of hw (their cost records carry
 * valid = 0, reason = 2 where they exceed it).  Neither metric depends on the stationary modes;
 * the lowest index stands for equal pairs.  Points come by ascending buffer size (descending
 * DRAM access); conventions as for mmee_pareto.  `evaluated` counts (row, tiling) pairs. */
int mmee_front_bs_da(const mmee_workload *w, const mmee_hw *hw, uint32_t flags, mmee_result *out,
                     uint32_t capacity, uint32_t *n_points);

/* The same calls for a free chain shape (Sec. VII-J).  Semantics, layouts and error codes are
 * those of the workload calls above. */
int mmee_chain_space_size(const mmee_chain *c, const mmee_hw *hw, uint64_t *out);
int mmee_chain_energy_regrouped(const mmee_chain *c, const mmee_hw *hw, uint32_t flags, int *out);
int mmee_chain_decode(const mmee_chain *c, const mmee_hw *hw, const uint64_t *idx, uint64_t n,
                      mmee_mapping *out);
int mmee_chain_eval_batch(const mmee_chain *c, const mmee_hw *hw, uint64_t first_idx, uint64_t n,
                          mmee_cost *out_costs);
int mmee_chain_search_multi(const mmee_chain *c, const mmee_hw *hw, const int *objectives,
                            uint32_t n_obj, uint32_t flags, mmee_result *out);
int mmee_chain_search_many(const mmee_chain *c, const mmee_hw *hw, const int *objectives,
                           uint32_t count, uint32_t flags, mmee_result *out, int *rc);
int mmee_chain_pareto(const mmee_chain *c, const mmee_hw *hw, uint32_t flags, mmee_result *out,
                      uint32_t capacity, uint32_t *n_points);
int mmee_chain_front_bs_da(const mmee_chain *c, const mmee_hw *hw, uint32_t flags, mmee_result *out,
                           uint32_t capacity, uint32_t *n_points);

/* mmee_search_ex for callers that cannot allocate: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  This call allocates and frees nothing, on the host
 * side of HIP or on the device, and does not synchronise: it enqueues a handful of kernels on the
 * library's stream (mmee_set_stream) and returns.  All its working memory (row encodings, the
 * per-tiling tables, partial records) is one fixed array of at most 40 MiB that every GPU the
 * library is loaded on holds until the process ends; problems with more than 16384 tilings do not
 * fit and return MMEE_ETOOBIG (mmee_strerror says by how much) with nothing enqueued.
 *   out_dev   DEVICE pointer (current device) to one mmee_result, written by the last kernel;
 *             valid once the stream has been synchronised by the caller.  `seconds` and
 *             `kernel_seconds` are 0.  When no candidate is feasible the call still returns
 *             MMEE_OK and the record carries cost.valid = 0 (nothing is read back to tell).
 *   flags     as for mmee_search_ex; the regrouped energy sum is used only where it is exact
 *             beforehand (mmee_energy_regrouped), never on trust.
 * The first call on a device runs the offline stage into the array and reads its counts and row
 * numbers back (one synchronisation of that stream, still no allocation): make it outside any capture.  All calls on one GPU
 * share that GPU's array, which keeps the last call's contents; what must start at zero is cleared
 * by a kernel at the start of each call, or left at zero by the call before.  Calls that overlap on one GPU (different streams, or
 * a captured call replayed while an earlier launch of it still runs) race; so does this call against
 * any other search in flight on a different stream.  What a race spoils are the results of the calls in it, none after them. */
int mmee_search_noalloc(const mmee_workload *w, const mmee_hw *hw, int objective, uint32_t flags,
                        mmee_result *out_dev);

/* Runs the offline stage if needed (row encoding + symbolic pruning, once per process) and
 * reports its counts. */
int mmee_offline_stats(mmee_row_stats *out);

/* The offline stage's row lists (Sec. VI-A: listed ahead of time; Sec. VI-B): the rows of group
 * g = r + 2 f that denote a dataflow (which = 0) or that survive the symbolic pruning of Eq. (12)
 * (which = 1), ascending, as row numbers inside the group: p_A + 5 p_B + 25 p_D + 125 p_E +
 * 625 * order.  rows_out (host) receives at most `capacity` numbers, *n_rows the length of the
 * list; MMEE_EOVERFLOW when the list is longer than `capacity`. */
int mmee_offline_rows(uint32_t group, uint32_t which, uint32_t *rows_out, uint32_t capacity, uint32_t *n_rows);

/* Environment: MMEE_RESIDENT_BLOCKS=<even number>, read at the first call, lowers the number of
 * persistent blocks that searches of the full row set, pruned searches of few problems on a shape and
 * walked fronts are launched with (default: two per compute unit).  It changes how the work is split
 * and in which order partial results meet, never a result.  Problems that share their shape's part
 * and fronts over the surviving rows take one block per 64 tilings and do not look at it. */

/* ---- running the chains -------------------------------------------------------------------------
 * The two chained matrix products whose mappings the calls above search, run on this GPU: attention of queries over
 * keys of another length (I != L) with its gradient, the same over a paged cache with a tree of drafted tokens, and a gated
 * feed-forward block with its gradient.
 *
 * Conventions of these calls.  Every tensor pointer is a DEVICE pointer (current device); strides are in elements, the last
 * dimension is contiguous.  Pointers are 16-byte aligned and strides of 16-bit tensors multiples of 8, strides of inputs may be 0 (a
 * broadcast input: its gradient comes out unreduced); the stride of a dimension of extent 1 is not looked at.  The calls allocate nothing, enqueue kernels
 * on the library's stream (mmee_set_stream) and return without waiting; the caller keeps the buffers alive and orders other streams' work against
 * that stream.  They may be captured into a HIP graph.  `workspace` is device memory that the call uses while its kernels run; the
 * *_workspace calls say how much it needs (0: none) and look at no pointer.  What lies in the workspace before does not matter.
 * The same call on the same inputs gives the same bits.  Inputs and outputs are 16 bits, sums 32 bits. */
enum { MMEE_F16 = 0, MMEE_BF16 = 1 };   /* dtype */

/* Cross attention.  q [batch][q_len][heads][head_dim], k and v [batch][kv_len][kv_heads][head_dim], o as q; strides of the
 * first three dimensions.  heads is a multiple of kv_heads: query head a reads key/value head a / (heads / kv_heads).
 *   o = softmax(scale q k^T) v     over the keys l < kv_lens[batch] (when given; clamped to 0 .. kv_len) whose key_mask byte is
 *   not 0 (when given).  Keys that do not count are not read into any result, whatever they hold.  A row without keys gives zeros,
 *   and lse -inf.  head_dim: a multiple of 8 up to 128.  scale > 0. */
typedef struct mmee_attn {
    uint32_t dtype;
    uint32_t batch, heads, kv_heads, head_dim;
    uint32_t q_len, kv_len;
    float scale;
    const void *q, *k, *v;
    void *o;
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];     /* batch, token, head         */
    float *lse;                     /* [batch][heads][q_len] contiguous: log sum exp of the scaled scores; may be null for forward */
    const int32_t *kv_lens;         /* [batch] or null                                            */
    const uint8_t *key_mask;        /* [batch][kv_len] or null                                    */
    int64_t mask_stride;            /* bytes from one batch to the next, 0: one mask for all      */
    void *workspace;
    uint64_t workspace_bytes;
    uint64_t reserved;              /* must be 0                                                  */
} mmee_attn;

/* Gradients of mmee_attn: d_o as o; dq as q, dk and dv as k and v. */
typedef struct mmee_attn_grads {
    const void *d_o;
    void *dq, *dk, *dv;
    int64_t do_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
} mmee_attn_grads;

/* backward != 0: enough for the forward and the backward call. */
int mmee_attn_workspace(const mmee_attn *a, int backward, uint64_t *bytes);
int mmee_attn_forward(const mmee_attn *a);
/* Reads o and lse as the forward call left them. */
int mmee_attn_backward(const mmee_attn *a, const mmee_attn_grads *g);

/* Attention of a tree of drafted tokens over a paged cache: nodes rows per sequence, q and o [batch][nodes][heads][head_dim].
 * Keys and values lie in pages [n_pages][page_tokens][kv_heads][head_dim] (page_tokens a power of two, at most 65536);
 * position p of sequence b is token p % page_tokens of page page_table[b][p / page_tokens], pages_per_seq entries a sequence.
 * cache_lens[b] positions hold the sequence so far, node j's key and value are at position cache_lens[b] + j.  Row i sees
 * the positions of the sequence so far and node j where bit j % 64 of ancestors[b][i][j / 64] is set (its own bit too, if it
 * sees itself), j < node_counts[b].  ancestors is [batch][nodes][(nodes + 63) / 64] contiguous.  Rows i >= node_counts[b] give zeros, and lse -inf.
 * Lengths and counts are clamped to what there is room for; positions in a page outside 0 .. n_pages-1 are not read and count as masked, like those
 * past the last node and nodes that no row i < node_counts[b] sees.  The values of a node that some row sees must be finite also for the rows that do not see it.
 * Room that a batch leaves unused is best left out by node_counts: nodes that only their empty bits leave out are looked for among the rows.
 * nodes at most 1024. */
typedef struct mmee_tree_attn {
    uint32_t dtype;
    uint32_t batch, heads, kv_heads, head_dim;
    uint32_t nodes;
    uint32_t page_tokens, pages_per_seq, n_pages;
    float scale;
    const void *q, *k_pages, *v_pages;
    void *o;
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];     /* batch or page, token, head */
    const int32_t *page_table;
    int64_t table_stride;           /* entries from one sequence to the next                      */
    const int32_t *cache_lens;      /* [batch]                                                    */
    const int32_t *node_counts;     /* [batch], or null: nodes everywhere                         */
    const uint64_t *ancestors;
    float *lse;                     /* [batch][heads][nodes] or null                              */
    void *workspace;
    uint64_t workspace_bytes;
    uint64_t reserved;              /* must be 0                                                  */
} mmee_tree_attn;

int mmee_tree_attn_workspace(const mmee_tree_attn *a, uint64_t *bytes);
int mmee_tree_attn_forward(const mmee_tree_attn *a);

/* Gated feed-forward block of `rows` tokens:
 *   g = x w_gate^T, u = x w_up^T, hidden = act(g) u, y = hidden w_down^T
 * x [rows][in_dim], w_gate and w_up [hidden_dim][in_dim] (one row stride for both), w_down [out_dim][hidden_dim], y [rows][out_dim]; row strides
 * of at least a row.  hidden [rows][hidden_dim] is contiguous; so are gate and up, which keep g and u for the backward call, or null.
 * Widths: multiples of 8 up to 2^22. */
enum { MMEE_ACT_SILU = 0, MMEE_ACT_GELU = 1, MMEE_ACT_GELU_TANH = 2, MMEE_ACT_RELU = 3, MMEE_ACT_SIGMOID = 4 };

typedef struct mmee_ffn {
    uint32_t dtype, act;
    uint32_t rows, in_dim, hidden_dim, out_dim;
    const void *x, *w_gate, *w_up, *w_down;
    void *y, *hidden, *gate, *up;
    int64_t x_stride, gate_stride, up_stride, down_stride, y_stride;
    void *workspace;
    uint64_t workspace_bytes;
    uint64_t reserved;              /* must be 0                                                  */
} mmee_ffn;

/* dy as y, dx as x; dw_gate, dw_up and dw_down as the weights, contiguous. */
typedef struct mmee_ffn_grads {
    const void *dy;
    void *dx, *dw_gate, *dw_up, *dw_down;
    int64_t dy_stride, dx_stride;
} mmee_ffn_grads;

/* backward != 0: enough for the forward and the backward call. */
int mmee_ffn_workspace(const mmee_ffn *f, int backward, uint64_t *bytes);
int mmee_ffn_forward(const mmee_ffn *f);
/* Reads hidden, gate and up as the forward call left them. */
int mmee_ffn_backward(const mmee_ffn *f, const mmee_ffn_grads *g);

/* Norm of queries and keys per head and their rotation by position, in one pass over both: tokens rows, q [tokens][heads][head_dim], k
 * [tokens][kv_heads][head_dim], outputs likewise; strides of the first two dimensions.  With weights (both or none)
 *   z = x weight / sqrt(mean of the head's x^2 + eps),     without: z = x
 * and the first rot_dim values of a head turn in pairs by angle[i] = position * freqs[i]:
 *   (y_a, y_b) = (z_a cos - z_b sin, z_a sin + z_b cos)    (a, b) = (i, i + rot_dim / 2), or (2 i, 2 i + 1) with MMEE_PAIRS_NEIGHBOURS
 * the rest of the head is z.  freqs are radians a position in 64 bits, and so are the angles, whatever the position.  Positions may have several
 * axes (time, height, width): pair i turns by the position along axis axis_of[i] (clamped to axes - 1; null: all along the first).  head_dim: a
 * multiple of 8 up to 256; rot_dim: a multiple of 16 up to head_dim, 0: no rotation (freqs and positions may then be null).  eps at least 1e-30.
 * Tokens: up to 2^26 - 4.
 * An output may be its input's own buffer with the same strides, not one that overlaps it otherwise. */
enum { MMEE_PAIRS_HALVES = 0, MMEE_PAIRS_NEIGHBOURS = 1 };

typedef struct mmee_qk_rotate {
    uint32_t dtype, pairs;
    uint32_t tokens, heads, kv_heads, head_dim, rot_dim;
    uint32_t axes;                  /* 1 to 4 */
    float eps;
    const void *q, *k;
    void *q_out, *k_out;
    int64_t q_stride[2], k_stride[2], q_out_stride[2], k_out_stride[2];     /* token, head */
    const void *q_weight, *k_weight;                                        /* [head_dim], of the tensors' type, or null */
    const double *freqs;            /* [rot_dim / 2] */
    const int32_t *positions;       /* [axes][tokens] */
    int64_t axis_stride;            /* positions from one axis to the next */
    const uint8_t *axis_of;         /* [rot_dim / 2] or null */
    void *workspace;                /* of the backward call */
    uint64_t workspace_bytes;
    uint64_t reserved;              /* must be 0 */
} mmee_qk_rotate;

/* Gradients: dq_out and dk_out of the outputs, dq and dk as q and k, the weights' as the weights (null without weights).  dq may be dq_out's own
 * buffer, dk dk_out's, with the same strides. */
typedef struct mmee_qk_rotate_grads {
    const void *dq_out, *dk_out;
    void *dq, *dk, *dq_weight, *dk_weight;
    int64_t dq_out_stride[2], dk_out_stride[2], dq_stride[2], dk_stride[2];
} mmee_qk_rotate_grads;

/* Of the backward call; the forward call needs none. */
int mmee_qk_rotate_workspace(const mmee_qk_rotate *r, uint64_t *bytes);
int mmee_qk_rotate_forward(const mmee_qk_rotate *r);
/* Reads q and k as the forward call did, not its outputs. */
int mmee_qk_rotate_backward(const mmee_qk_rotate *r, const mmee_qk_rotate_grads *g);

/* Appends keys and values to a paged cache (pages, table and lengths as of mmee_tree_attn), the keys normed and rotated on the way as by
 * mmee_qk_rotate, the values as they are, and norms and rotates the queries beside them (q null: none; heads is then 0).  The new tokens of
 * `seqs` sequences lie one behind the other: sequence b's are starts[b] .. starts[b + 1] - 1, or, with starts null, tokens / seqs of each (without a
 * remainder).  Its j-th goes to position cache_lens[b] + j, which is also what it is rotated by unless positions are given.  Tokens
 * j >= counts[b] (when given) and tokens of no sequence leave everything as it was.  Positions past the page table and pages outside 0 .. n_pages-1 are
 * not written; the token's query is.  cache_lens stay as they are (clamped to 0 where they are below).  starts ascend and lie within 0 .. tokens.
 * Two new tokens at one place of the pool (sequences that share the page they write to) leave values of either there. */
typedef struct mmee_cache_append {
    uint32_t dtype, pairs;
    uint32_t tokens, seqs, heads, kv_heads, head_dim, rot_dim;
    uint32_t axes;
    uint32_t page_tokens, pages_per_seq, n_pages;
    float eps;
    const void *q, *k, *v;
    void *q_out, *k_pages, *v_pages;
    int64_t q_stride[2], k_stride[2], v_stride[2], q_out_stride[2];         /* token, head */
    int64_t k_pages_stride[3], v_pages_stride[3];                           /* page, token, head */
    const void *q_weight, *k_weight;
    const double *freqs;
    const int32_t *positions;       /* [axes][tokens], or null: positions in the cache (axes 1) */
    int64_t axis_stride;
    const uint8_t *axis_of;
    const int32_t *starts;          /* [seqs + 1] or null */
    const int32_t *counts;          /* [seqs] or null */
    const int32_t *cache_lens;      /* [seqs] */
    const int32_t *page_table;      /* [seqs][pages_per_seq] */
    int64_t table_stride;
    uint64_t reserved;              /* must be 0 */
} mmee_cache_append;

int mmee_cache_append_forward(const mmee_cache_append *c);

/* Attention of packed prompts: rows of sequence b are tokens q_starts[b] .. q_starts[b + 1] - 1 of q and o [q_tokens][heads][head_dim], its keys
 * tokens kv_starts[b] .. kv_starts[b + 1] - 1 of k and v [kv_tokens][kv_heads][head_dim] (kv_starts null: q_starts, and kv_tokens = q_tokens).
 * Heads, head_dim, scale as of mmee_attn; strides of the first two dimensions, between tokens 2^24 at most; up to 2^28 keys, and rows that share a
 * key/value head, in tiles that one launch can hold (kv_heads * (rows / 128 + keys / 128 + seqs) below 2^23 suffices).  causal != 0: row i of a sequence of m rows and n keys sees the
 * keys j <= i + n - m (the last row at the last key: a prompt over itself, or a prompt's next rows over all keys so far); 0: all n.  A row without keys
 * gives zeros, and lse -inf.  Starts ascend and lie within 0 .. tokens (beyond, they are clamped; a sequence whose end lies before its start is empty;
 * sequences that overlap are not looked for: which of them an output belongs to is then undefined).
 * What is not finite in a token may reach all rows of its sequence, none of another one.  Tokens of no sequence are not read, and outputs there are
 * left as they were; keys of a sequence without rows get zero gradients. */
typedef struct mmee_prompt_attn {
    uint32_t dtype, causal;
    uint32_t seqs, heads, kv_heads, head_dim;
    uint32_t q_tokens, kv_tokens;
    float scale;
    const void *q, *k, *v;
    void *o;
    int64_t q_stride[2], k_stride[2], v_stride[2], o_stride[2];             /* token, head */
    const int32_t *q_starts, *kv_starts;                                    /* [seqs + 1]  */
    float *lse;                     /* [heads][q_tokens] contiguous; may be null for forward */
    void *workspace;
    uint64_t workspace_bytes;
    uint64_t reserved;              /* must be 0 */
} mmee_prompt_attn;

/* d_o as o; dq as q, dk and dv as k and v. */
typedef struct mmee_prompt_attn_grads {
    const void *d_o;
    void *dq, *dk, *dv;
    int64_t do_stride[2], dq_stride[2], dk_stride[2], dv_stride[2];
} mmee_prompt_attn_grads;

/* backward != 0: enough for the forward and the backward call. */
int mmee_prompt_attn_workspace(const mmee_prompt_attn *a, int backward, uint64_t *bytes);
int mmee_prompt_attn_forward(const mmee_prompt_attn *a);
/* Reads o and lse as the forward call left them. */
int mmee_prompt_attn_backward(const mmee_prompt_attn *a, const mmee_prompt_attn_grads *g);

/* Use this HIP stream (a hipStream_t passed as void*) for all later launches; NULL = default.  Once a search, evaluation or front has
 * run, the call first waits for the stream used so far, whose scratch later launches share; before that, in a program that runs the
 * chains alone, it waits for nothing. */
int mmee_set_stream(void *hip_stream);

/* Free all cached device memory.  The library re-initialises itself on the next call. */
void mmee_shutdown(void);

const char *mmee_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* MMEE_H */
