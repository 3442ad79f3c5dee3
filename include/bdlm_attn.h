/*
 * bdlm_attn.h -- C ABI of the BDLM attention library for MI355X (gfx950).
 *
 * Block-diffusion LM training evaluates attention over a length-2L sequence:
 * a clean copy x and a corrupted copy x_t of L tokens, both split into blocks
 * of block_size tokens (arXiv 2609.19242, Sec. 3.2).  With 0-based positions
 * and blk(p) = p / block_size, a query row may attend to a key row when
 *
 *   clean query q,     clean key k:     k <= q                (token-causal; the paper's rule,
 *                                                              App. A eq:correctness-clean-attention)
 *                                       blk(k) <= blk(q)      (BDLM_CLEAN_INTRA_BLOCK reading)
 *   corrupted query q, corrupted key k: blk(k) == blk(q)      (own block, bidirectional)
 *   corrupted query q, clean key k:     blk(k) <  blk(q)      (clean prefix of earlier blocks)
 *   clean query,       corrupted key:   never
 *
 * (eq:correctness-corrupted-attention).  The library computes masked softmax
 * attention under this mask, its log-sum-exp, partial attention over one key
 * range, the J-way log-sum-exp merge of partials (eq:csbp-lse-merge), and the
 * exact backward from the saved output and LSE (App. C, fused backward).
 *
 * Mask generalisations (both keep every visible set an interval of positions):
 *  - window W > 0 (the sliding-window attention layers of the paper's
 *    DiffusionGemma runs, App. "Savings Breakdowns"): with e the end of the
 *    clean context the rules above give a query (q + 1 for a clean query under
 *    the token-causal rule, the end of its block under BDLM_CLEAN_INTRA_BLOCK,
 *    the start of its block for a corrupted query), only clean keys k with
 *    e - W <= k < e stay visible.  Corrupted keys are unaffected.
 *  - clean_prefix (the DFlash2 drafter attention, App. "DFlash2 Drafter
 *    Training Methodology", eq:dflash2-block-attention): corrupted block b is a
 *    draft block whose clean context (the target features) ends at
 *    clean_prefix[b] = a_b instead of at block_size * b; it still sees its own
 *    block bidirectionally.  The table must be non-decreasing with entries in
 *    [0, L] (draft blocks ordered by anchor: their losses are independent, so
 *    the order is free).  The asynchronous calls cannot check the contents:
 *    entries are clamped into [0, L] when read, and a decreasing table gives an
 *    unspecified mask (never an out-of-bounds access).  bdlm_visible_pairs
 *    checks the table and returns -1 when it breaks the contract.
 *
 * Rows and ranges.  A tensor's rows are described by bdlm_range records: a
 * range is `len` consecutive rows of one stream holding global positions
 * [pos0, pos0 + len).  Per batch element b, row i of a range lives at row
 * (b * batch_stride + i) of the pointer given for that range, where
 * batch_stride >= len (0 means len).  The packed joint layout [x_t ; x] of a
 * [batch][2L][heads][head_dim] tensor is two ranges {CORRUPTED, 0, L} at row 0
 * and {CLEAN, 0, L} at row L, both with batch_stride 2L.
 *
 * Layouts (all row-major, head_dim innermost, 16-byte aligned pointers):
 *   Q, O, dO, dQ : [batch][rows][heads][head_dim]
 *   K, V, dK, dV : [batch][rows][kv_heads][head_dim]
 *   Q, K, V, dO are in the problem's dtype; O, dQ, dK, dV are in that dtype,
 *   or fp32 when out_f32 = 1 (bdlm_attn_bwd reads O in the same type).
 *   LSE          : [batch][heads][rows] fp32, natural log; for a range with
 *                  batch stride R, element (b, h, i) is at b*heads*R + h*R + i.
 * Query head h reads KV head h / (heads / kv_heads).
 *
 * Ownership and execution.  Every buffer is device memory owned by the caller;
 * the library allocates and frees nothing.  Each call validates its arguments
 * on the host, then enqueues kernels on `stream` and returns without
 * synchronising.  Pointer arrays (`const void* const* q` ...) are host arrays
 * of device pointers, read during the call only.
 *
 * Errors.  A call returns BDLM_OK or a negative status.  Invalid or
 * unsupported arguments are rejected before anything is enqueued; a failed
 * launch returns BDLM_ERR_HIP.  bdlm_last_error() returns a message for the
 * calling thread's last failure.  No C++ exception crosses this interface.
 */
#ifndef BDLM_ATTN_H
#define BDLM_ATTN_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  BDLM_OK = 0,
  BDLM_ERR_INVALID = -1,     /* malformed argument: sizes, ranges, null or misaligned pointers */
  BDLM_ERR_UNSUPPORTED = -2, /* well-formed but not implemented: head_dim, dtype, too many ranges */
  BDLM_ERR_HIP = -3,         /* a HIP call or kernel launch failed */
  BDLM_ERR_WORKSPACE = -4    /* workspace missing or too small for the row statistics */
} bdlm_status;

typedef enum { BDLM_BF16 = 0, BDLM_F32 = 1 } bdlm_dtype;
typedef enum { BDLM_CLEAN = 0, BDLM_CORRUPTED = 1 } bdlm_stream;
typedef enum {
  BDLM_CLEAN_INTRA_CAUSAL = 0, /* clean query at position q sees clean keys at positions <= q */
  BDLM_CLEAN_INTRA_BLOCK = 1   /* clean query sees every clean key of its own and earlier blocks */
} bdlm_clean_intra;

/* Bits of bdlm_problem.hilo: which products carry P or dS as two bf16 terms. */
#define BDLM_HILO_PV 1   /* forward O += P V */
#define BDLM_HILO_DKDV 2 /* backward dV += P^T dO and dK += dS^T Q */
#define BDLM_HILO_DQ 4   /* backward dQ += dS K */
#define BDLM_HILO_ALL 7
/* With any of the bits above: a selected product carries the second term only where some
   probability P of the block of operands it contracts reaches 1/64, and a single bf16 term
   elsewhere.  The blocks are one wave's 32 query rows x 16 keys (P V, dS K) or 32 keys x 16 query
   rows of one query head (P^T dO, dS^T Q); the forward tests P against the row's running sum,
   which can only over-select.  An element left single-term has P < 1/64, so its rounding error is
   below 2^-15 in P and below 2^-15 |dP - D| in dS.  Same results as the all-tiles form up to
   rounding; fewer matrix products where large probabilities are rare. */
#define BDLM_HILO_ADAPTIVE 8

/* Limits of one call (kernel-argument capacity). */
#define BDLM_MAX_Q_RANGES 4
#define BDLM_MAX_K_RANGES 32
#define BDLM_MAX_MERGE_PARTS 32

/* Shape and mask description shared by every attention call. */
typedef struct {
  int64_t batch;      /* independent sequences, >= 1 */
  int64_t L;          /* tokens per copy: positions of both streams lie in [0, L) */
  int64_t block_size; /* tokens per block (the paper's M = L / B); L % block_size == 0 */
  int32_t heads;      /* query heads, a multiple of kv_heads */
  int32_t kv_heads;   /* key/value heads */
  int32_t head_dim;   /* 64 or 128 */
  int32_t dtype;      /* bdlm_dtype of Q, K, V and dO (and of the outputs unless out_f32) */
  float scale;        /* softmax scale; <= 0 selects 1 / sqrt(head_dim) */
  int32_t clean_intra;/* bdlm_clean_intra */
  int32_t out_f32;    /* 0: O, dQ, dK, dV in `dtype`; 1: in fp32 (the fp32 accumulators, unrounded) */
  int32_t hilo;       /* bf16 path: a mask of BDLM_HILO_* bits.  A product whose bit is clear takes
                         its operand P (softmax probabilities) or dS = P (dP - D) rounded to bf16;
                         a product whose bit is set takes it as a two-term bf16 sum hi + lo (about
                         16 significant bits, twice the matrix work of that product), on every
                         tile or, with BDLM_HILO_ADAPTIVE, only on tiles holding a large P.  For
                         inputs with large scores or |dS|, e.g. keys of large norm.  Ignored by
                         the fp32 path. */
  int64_t window;     /* 0: no limit.  > 0: a query sees only the last `window` positions of its clean
                         context (sliding-window layers; see "Mask generalisations" above) */
  const int32_t* clean_prefix; /* NULL, or a device array of L / block_size ints: the end of the clean
                         context of corrupted block b (DFlash2 anchors; see above).  Read by the kernels
                         during the call's execution; bdlm_visible_pairs reads it synchronously. */
} bdlm_problem;

/* A run of rows of one stream (see "Rows and ranges" above). */
typedef struct {
  int32_t stream;       /* bdlm_stream */
  int32_t reserved;     /* must be 0 */
  int64_t pos0;         /* global position of the range's first row, >= 0 */
  int64_t len;          /* rows, >= 0; pos0 + len <= L */
  int64_t batch_stride; /* rows between batch elements in this range's tensors; 0 means len */
} bdlm_range;

/*
 * Fused forward (Sec. 3.2 mask; eq:context-parallel-attention).
 * For every row of the n_q query ranges: O = softmax(scale * Q K^T + mask) V
 * and LSE = log sum exp(scale * Q K^T + mask), over all rows of the n_k key
 * ranges, in one pass with online softmax across ranges.  Tiles the mask
 * hides are skipped; only tiles it partly hides evaluate it.
 *   q[i], o[i], lse[i] : query range i's Q (in), O (out), LSE (out)
 *   k[j], v[j]         : key range j's K and V (in)
 * A query row that sees no key gets O = 0 and LSE = -inf.
 * Limits: 1 <= n_q <= BDLM_MAX_Q_RANGES, 1 <= n_k <= BDLM_MAX_K_RANGES.
 */
bdlm_status bdlm_attn_fwd(const bdlm_problem* p,
                          int32_t n_q, const bdlm_range* q_ranges,
                          const void* const* q, void* const* o, float* const* lse,
                          int32_t n_k, const bdlm_range* k_ranges,
                          const void* const* k, const void* const* v,
                          hipStream_t stream);

/*
 * Partial forward of one query range over one key range (App. A, step 2,
 * eq:correctness-online-softmax-merge; the per-launch normalised output O_j and
 * LSE z_j of App. C).  Same arithmetic as bdlm_attn_fwd restricted to key range
 * kr: O_j is normalised over the visible keys of kr only; rows that see none of
 * them get O_j = 0 exactly and z_j = -inf, so merging them is a no-op.
 *   q, o, lse : query range qr's Q (in), O_j (out), z_j (out)
 *   k, v      : key range kr's K and V (in)
 */
bdlm_status bdlm_attn_partial_fwd(const bdlm_problem* p,
                                  bdlm_range qr, const void* q, void* o, float* lse,
                                  bdlm_range kr, const void* k, const void* v,
                                  hipStream_t stream);

/*
 * J-way log-sum-exp merge of normalised partials over disjoint key sets
 * (eq:csbp-lse-merge generalised by eq:correctness-online-softmax-merge):
 *   m = max_j z_j,  w_j = exp(z_j - m) (0 where z_j = -inf),
 *   O = sum_j w_j O_j / sum_j w_j,  z = m + log(sum_j w_j),
 * in fp32 registers, one pass over the J inputs.  A row with every z_j = -inf
 * gets O = 0 and z = -inf.
 *   o_parts[j] : [batch][rows][heads][head_dim] in part_dtype
 *   lse_parts[j] : [batch][heads][rows] fp32
 *   o : [batch][rows][heads][head_dim] in out_dtype;  lse : [batch][heads][rows] fp32
 * o and lse may alias neither input.  1 <= n_parts <= BDLM_MAX_MERGE_PARTS;
 * batch * rows * heads < 2^31 (else BDLM_ERR_UNSUPPORTED, nothing launched).
 */
bdlm_status bdlm_lse_merge(int64_t batch, int64_t rows, int32_t heads, int32_t head_dim,
                           int32_t n_parts, const void* const* o_parts,
                           const float* const* lse_parts, int32_t part_dtype,
                           void* o, float* lse, int32_t out_dtype, hipStream_t stream);

/*
 * bdlm_lse_merge over rows laid out with batch strides, as the attention calls
 * write them (bdlm_range.batch_stride): part element (b, i, h, :) of O_j is at
 * row b * part_batch_stride + i of o_parts[j], z_j(b, h, i) at
 * (b * heads + h) * part_batch_stride + i of lse_parts[j]; the outputs likewise
 * with out_batch_stride.  A stride of 0 means rows (dense, as bdlm_lse_merge).
 * Strides below rows give BDLM_ERR_INVALID, above 2^30 BDLM_ERR_UNSUPPORTED;
 * otherwise the contract of bdlm_lse_merge, which is this call with both
 * strides 0.  Padding rows between batch elements are neither read nor written.
 */
bdlm_status bdlm_lse_merge_strided(int64_t batch, int64_t rows, int32_t heads, int32_t head_dim,
                                   int32_t n_parts, const void* const* o_parts,
                                   const float* const* lse_parts, int32_t part_dtype,
                                   int64_t part_batch_stride, void* o, float* lse,
                                   int32_t out_dtype, int64_t out_batch_stride,
                                   hipStream_t stream);

/* Workspace bytes bdlm_attn_bwd takes for these query ranges: per range two
 * fp32 arrays of batch * len * heads values (each rounded up to 256 bytes),
 * LSE * log2(e) and the row dots D = rowsum(dO * O), which every call needs;
 * and, for problems with too few key tiles to fill the card, the partial sums
 * of dK/dV walks that are cut into chunks and run side by side (arrays and
 * sums together at most BDLM_NOALLOC_SCRATCH_BYTES).  It is enough for any key
 * ranges, and a key range's dK and dV do not depend on which other ranges are
 * in the call.  bdlm_attn_bwd takes any size from the arrays' up; with less
 * than this function's, or with key ranges that overlap, it leaves the walks
 * whole: the same sums in another order, slower.  Ranges whose batch * len *
 * heads exceeds 2^28 are rejected by bdlm_attn_bwd. */
size_t bdlm_attn_bwd_workspace_bytes(const bdlm_problem* p, int32_t n_q, const bdlm_range* q_ranges);

/*
 * Backward from the saved (final, merged) O and LSE (App. C fused backward;
 * eqs. eq:correctness-corrupted-gradient .. eq:correctness-query-gradient).
 * With P = exp(scale * Q K^T + mask - LSE) and D = rowsum(dO * O):
 *   dV = P^T dO,  dS = P * (dO V^T - D),  dQ = scale * dS K,  dK = scale * dS^T Q,
 * summed over every query row of every query range, and over the query heads
 * of each KV head.  dq[i] like q[i]; dk[j], dv[j] like k[j]; all overwritten.
 * Key rows no query sees get dK = dV = 0.
 * workspace: device memory of bdlm_attn_bwd_workspace_bytes() (see there),
 * 256-byte aligned, contents ignored on entry.
 */
bdlm_status bdlm_attn_bwd(const bdlm_problem* p,
                          int32_t n_q, const bdlm_range* q_ranges,
                          const void* const* q, const void* const* o, const float* const* lse,
                          const void* const* dO, void* const* dq,
                          int32_t n_k, const bdlm_range* k_ranges,
                          const void* const* k, const void* const* v,
                          void* const* dk, void* const* dv,
                          void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * bdlm_attn_bwd without a workspace argument, for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc).  Same arguments, arithmetic, kernels and results as
 * bdlm_attn_bwd with the workspace of bdlm_attn_bwd_workspace_bytes(); the
 * workspace is a library-owned device array of BDLM_NOALLOC_SCRATCH_BYTES bytes
 * instead (one per GPU, held until the process ends).  The call allocates
 * nothing.  Query ranges whose D and LSE * log2(e)
 * need more than the array holds (more than about 8M (batch x row x head)
 * entries) are rejected with
 * BDLM_ERR_UNSUPPORTED before anything is enqueued.  The array of the device
 * current at the call is used, so `stream` must belong to that device.  Every
 * call on one GPU shares its array: calls that overlap in time on one GPU
 * (other streams, other threads) race and must be serialised by the caller.
 */
#define BDLM_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
bdlm_status bdlm_attn_bwd_noalloc(const bdlm_problem* p,
                                  int32_t n_q, const bdlm_range* q_ranges,
                                  const void* const* q, const void* const* o, const float* const* lse,
                                  const void* const* dO, void* const* dq,
                                  int32_t n_k, const bdlm_range* k_ranges,
                                  const void* const* k, const void* const* v,
                                  void* const* dk, void* const* dv, hipStream_t stream);

/*
 * Number of valid query-key pairs of the mask per (batch element, query head),
 * summed over the given ranges (the paper's unit of attention work, App. B
 * eq:block-work-by-position).  Host only; returns -1 on invalid arguments.
 */
int64_t bdlm_visible_pairs(const bdlm_problem* p, int32_t n_q, const bdlm_range* q_ranges,
                           int32_t n_k, const bdlm_range* k_ranges);

/*
 * Packed attention: sequences of different lengths in one call, without the
 * corrupted copy (prompts, packed training texts).  Sequence s has query rows
 * [q_start, q_start + q_len) and key rows [k_start, k_start + k_len) of the
 * call's tensors; its query row i is at position x = k_len - q_len + i (the
 * queries are the last q_len tokens), key row j at position j.  With blocks of
 * block_size tokens and e = block_size * (floor(x / block_size) + 1), row x sees
 * the keys j < e (block_size 1: j <= x), with a window only those with
 * j >= e - window and the first ones, j < sinks.  Rows at negative positions (q_len > k_len) see nothing.
 * A row that sees no key gets O = 0, LSE = -inf and dQ = 0; a key that no row
 * sees gets dK = dV = 0.  Rows that belong to no sequence are neither read nor
 * written.  The other rows must be finite: hidden pairs enter products as 0 times
 * their values, so a NaN or infinity in a key may reach rows of its sequence that
 * do not see it (keys that no row sees may hold anything in bf16 and fp32 alike, but for
 * those between the windows of blocks longer than a window).
 *
 *   Q, O, dO, dQ : [rows][heads][head_dim], K, V, dK, dV : [rows][kv_heads][head_dim],
 *     rows `stride` elements apart (a multiple of 16 bytes, at most 2^20), so
 *     that q, k and v may be parts of one fused projection
 *   LSE          : [heads][lse_pitch] fp32, natural log
 * Everything is in the problem's dtype (LSE fp32).
 *
 * Rounding.  bf16: scores, softmax statistics, D and all sums are fp32; P (and,
 * backward, dS) is rounded to bf16 for its second product, off by at most 2^-8 of
 * itself, as in bdlm_attn_fwd and bdlm_attn_bwd without hilo, which packed calls do
 * not have; outputs are rounded once.  Backward takes D = dO . O from the rounded O, off by up to
 * 2^-8 |dO||O|, but for rows of few keys, where it comes from the products: without sinks, rows all of
 * whose keys lie in one of the sequence's runs of 64, with sinks, rows that see at most 64.  fp32: fp64 between the inputs and the outputs,
 * but for the LSE that backward reads and D between its kernels, which are fp32.  The
 * same plan and inputs give the same bits.  In another batch a sequence's walks may
 * be cut elsewhere, so that its sums run in another order.
 */
typedef struct {
  int32_t heads, kv_heads, head_dim, dtype;
  float scale;         /* <= 0 selects 1 / sqrt(head_dim); positive scales below 2^-96 are unsupported */
  int32_t sinks;       /* with a window: the first keys of a sequence that stay visible */
  int64_t block_size;  /* tokens per block, 1 for token-causal attention */
  int64_t window;      /* 0: no limit */
} bdlm_packed;

/* Sequences come in the order of their rows and do not overlap; gaps are allowed. */
typedef struct {
  int64_t q_start, q_len, k_start, k_len;
} bdlm_packed_seq;

/* Chunks of query tiles' walks, where those are cut. */
typedef struct {
  int32_t items, sums, slots, reserved;
} bdlm_packed_chunks;

/* What bdlm_packed_plan_make found: passed on to the calls unchanged. */
typedef struct {
  bdlm_packed problem;
  int64_t q_rows, k_rows;    /* rows that the query and key tensors have at least */
  int32_t q_items, k_items, n_sums, slots, teams, reserved;
  bdlm_packed_chunks fwd, dq;
  size_t bytes;               /* of the items */
  size_t workspace_bytes;     /* of bdlm_packed_bwd */
  size_t fwd_workspace_bytes; /* of bdlm_packed_fwd */
} bdlm_packed_plan;

/* A tensor's first row and the elements between its rows. */
typedef struct {
  void* ptr;
  int64_t stride;
} bdlm_rows;

/*
 * The plan of packed calls over these sequences, for every layer and for
 * forward and backward.  Host only.  Fills *plan, and, unless items is null,
 * the plan->bytes bytes of work items at `items` (host memory, items_bytes
 * long); the caller copies those to device memory, 16-byte aligned, and keeps
 * them there while calls that use them run.
 */
bdlm_status bdlm_packed_plan_make(const bdlm_packed* p, int64_t n_seqs, const bdlm_packed_seq* seqs, void* items,
                                  size_t items_bytes, bdlm_packed_plan* plan);

/* O and LSE of a packed call.  items: the plan's items in device memory.
 * workspace: plan->fwd_workspace_bytes bytes (0 unless there are few query tiles with long walks), as in
 * bdlm_packed_bwd.  Deterministic. */
bdlm_status bdlm_packed_fwd(const bdlm_packed_plan* plan, const void* items, bdlm_rows q, bdlm_rows k, bdlm_rows v,
                            bdlm_rows o, float* lse, int64_t lse_pitch, void* workspace, size_t workspace_bytes,
                            hipStream_t stream);

/*
 * dQ, dK and dV of a packed call from its O and LSE (the formulas of
 * bdlm_attn_bwd).  workspace: plan->workspace_bytes bytes of device memory,
 * 256-byte aligned, contents ignored on entry; calls that may overlap in time
 * need one each.  Deterministic.  q_rows * heads <= 2^28.
 */
bdlm_status bdlm_packed_bwd(const bdlm_packed_plan* plan, const void* items, bdlm_rows q, bdlm_rows k, bdlm_rows v,
                            bdlm_rows o, const float* lse, int64_t lse_pitch, bdlm_rows dO, bdlm_rows dq, bdlm_rows dk,
                            bdlm_rows dv, void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * A paged cache of keys and values, and its pages' bookkeeping, all in device
 * memory owned by the caller.  Sequence s holds lens[s] tokens; token t is row
 * t % page_size of page table[s][t / page_size].  refs[p] counts the tables
 * that hold page p (0: free).  A page that is not full belongs to one sequence;
 * full ones may be shared, and what is written into a shared page, all its
 * sequences see.
 *
 * The page operations run in stream order and must not overlap in time with
 * each other or with attention over the same cache; they need no host round
 * trip and may be captured in a graph.  They check the lists that they are
 * given, which lie in device memory, on the device: status[0] becomes a
 * bdlm_cache_status, and, except for BDLM_CACHE_OK, grow and fork change nothing else.
 * status holds the outcome of the last grow, fork, free or compact.
 */
typedef enum {
  BDLM_CACHE_OK = 0,
  BDLM_CACHE_BAD_LIST = 1, /* a number out of range or listed twice, or against the call's rules */
  BDLM_CACHE_NO_PAGES = 2  /* too few free pages: status[1] more are needed (at most 2^31 - 1 are told) */
} bdlm_cache_status;

typedef struct {
  void *k, *v;      /* [layers][pages][page_size][kv_heads][head_dim], 16-byte aligned */
  int32_t* table;   /* [seqs][max_pages] */
  int32_t* lens;    /* [seqs] */
  int32_t* refs;    /* [pages] */
  int32_t* status;  /* [2] */
  int32_t* work;    /* bdlm_cache_work_bytes() bytes, contents ignored on entry */
  int64_t layers, pages, page_size, seqs, max_pages; /* seqs <= 2^19; max_pages * page_size < 2^30 */
  int32_t kv_heads, head_dim, dtype, reserved;       /* reserved must be 0 */
} bdlm_cache;

size_t bdlm_cache_work_bytes(int64_t pages, int64_t seqs);

/* Makes room for counts[i] >= 0 more tokens of sequence seqs[i] (n different
 * sequences): lens grows, and new pages come from the free ones, lowest
 * numbers first, to the sequences in the order of the list. */
bdlm_status bdlm_cache_grow(const bdlm_cache* c, int64_t n, const int32_t* seqs, const int32_t* counts,
                            hipStream_t stream);

/* Makes sequence children[i] a copy of parents[i]: full pages are shared, the
 * rows of a last partial page are copied, in all layers, to a page of its own
 * (free ones, lowest numbers first).  Children are different, empty and no
 * parents; a parent may have several. */
bdlm_status bdlm_cache_fork(const bdlm_cache* c, int64_t n, const int32_t* parents, const int32_t* children,
                            hipStream_t stream);

/* Empties sequences: their pages lose a reference each, their table entries
 * become -1.  One listed twice is freed once; a number out of range is passed
 * over (BDLM_CACHE_BAD_LIST, the others are freed). */
bdlm_status bdlm_cache_free(const bdlm_cache* c, int64_t n, const int32_t* seqs, hipStream_t stream);

/* Moves live pages to the lowest numbers: with L of them, the i-th free page
 * below L takes the data, in all layers, and the references of the i-th live page from L on; all
 * tables follow.  Afterwards pages L and up are free. */
bdlm_status bdlm_cache_compact(const bdlm_cache* c, hipStream_t stream);

/* Writes K and V rows of a layer: counts[i] rows from row starts[i] of k and v
 * on (starts NULL: from row i * rows / n on, at most rows / n) become the last
 * counts[i] tokens of sequence seqs[i] (after grow).  Rows out of `rows`, out
 * of the sequence or in pages out of the cache are passed over.  Sequences are
 * different. */
bdlm_status bdlm_cache_write(const bdlm_cache* c, int64_t layer, int64_t n, const int32_t* seqs, const int32_t* counts,
                             const int32_t* starts, int64_t rows, bdlm_rows k, bdlm_rows v, hipStream_t stream);

/*
 * Attention of decoding requests over the cache: request r is sequence
 * seqs[r], whose keys and values are in the cache, and its `rows` query rows
 * are its last tokens.  Row i sees the keys up to its own position, lens - rows
 * + i, or, with block = 1 (a block that is being denoised), all lens keys.  The
 * first `prefix` tokens are the same in all requests; they may be read through
 * the first request's table, once for all, which therefore has to hold them
 * all.  The result is that of attention over each request's own tokens.
 *   q, o : [requests][rows][heads][head_dim] in the cache's dtype
 *   lse  : [requests][heads][rows] fp32, natural log
 * Rows that see nothing (also: of a sequence number out of range) get O = 0
 * and LSE = -inf.  Keys and values of tokens that a sequence holds must be finite,
 * as in packed calls; rows of pages behind its last token may hold anything.  A page
 * number outside the cache reads as rows of zeros, and lens are taken between 0 and
 * what a table holds.
 * Rounding: as in packed calls, and where keys are cut into chunks their outputs are
 * kept in fp32 in both dtypes; fp32 calls join them in fp64, bf16 ones in fp32.  The
 * cuts follow the arguments and what a table can hold (the lengths are not known on
 * the host), so bits may differ with `prefix`, the table's size and the batch.
 * workspace: bdlm_prefix_attn_workspace_bytes() bytes, 256-byte aligned, contents ignored on
 * entry; calls that may overlap in time need one each.  It grows with what a table can
 * hold, by head_dim + 1 (fp32: + 2) words per chunk, row and head: 16 requests of 512
 * rows of 32 heads take 258 MiB with tables of 9,700 tokens, 1.1 GiB with 131,072.
 */
size_t bdlm_prefix_attn_workspace_bytes(const bdlm_cache* c, int64_t requests, int64_t rows, int32_t heads,
                                        int64_t prefix);
bdlm_status bdlm_prefix_attn(const bdlm_cache* c, int64_t layer, int64_t requests, const int32_t* seqs, int64_t rows,
                             int32_t heads, int64_t prefix, int32_t block, float scale, const void* q, void* o,
                             float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Attention of chunks of new tokens over the cache: request r is sequence seqs[r],
 * and its counts[r] new tokens are its last ones (after grow; their keys and values are in the
 * cache): one for a decoding request, many for a piece of a prompt.  The requests'
 * query rows lie one after the other in q, in the order of the list; rows behind
 * the last request's belong to none.  With len the sequence's tokens, row i of request
 * r is at position x = len - counts[r] + i; it sees the keys that a row at x sees in packed calls:
 * with e = block_size * (floor(x / block_size) + 1), j < min(e, len), with a window only
 * j >= e - window or j < sinks.  Rows that see nothing (negative positions, a sequence
 * number out of range) get O = 0 and LSE = -inf.  Negative counts count as 0; rows past `rows` are passed over.
 *
 * A plan is made on the device from the lengths and counts, in stream order, for all
 * layers of a step; it may be captured in a graph.  It holds while the lengths it was
 * made from do; the table is read by the calls.  After BDLM_CHUNK_STARTS bytes it holds the requests'
 * first rows (int32 [requests], at most `rows`), as bdlm_cache_write takes them.
 * A call takes a plan that was made with its own bdlm_chunk (but for scale) and a cache of its own's sizes (but for
 * layers and pages).  With another one (a captured call that is replayed after its plan was made anew with another
 * window, say), or one that no call has made, every row becomes NaN, whatever `fill` is.
 *   q, o : [rows][heads][head_dim] in the cache's dtype, rows `stride` elements apart
 *   lse  : [heads][lse_pitch] fp32, natural log
 *   fill : 1: rows behind the last request's become 0 (LSE -inf), 0: they stay as they are
 * Keys and values that no row of a request sees may hold anything (but for those between
 * the windows of blocks longer than a window); the others of its sequence must be finite.  A page number outside the cache reads as rows of zeros, and lens are
 * taken between 0 and what a table holds; the cache has at most 2^34 tokens' room.  Rounding as in bdlm_prefix_attn; the cuts follow the
 * plan, so bits may differ with the batch.
 * workspace: bdlm_chunk_workspace_bytes() bytes, 256-byte aligned, contents ignored on
 * entry; calls that may overlap in time need one each (they may share a plan).
 */
#define BDLM_CHUNK_STARTS 64
typedef struct {
  int64_t requests, rows;
  int64_t block_size, window;
  int32_t heads, sinks;
  float scale;         /* <= 0 selects 1 / sqrt(head_dim) */
  int32_t reserved;    /* must be 0 */
} bdlm_chunk;

size_t bdlm_chunk_plan_bytes(const bdlm_cache* c, const bdlm_chunk* p);
size_t bdlm_chunk_workspace_bytes(const bdlm_cache* c, const bdlm_chunk* p);
/* plan: bdlm_chunk_plan_bytes() bytes of device memory, 16-byte aligned. */
bdlm_status bdlm_chunk_plan(const bdlm_cache* c, const bdlm_chunk* p, const int32_t* seqs, const int32_t* counts,
                            void* plan, size_t plan_bytes, hipStream_t stream);
bdlm_status bdlm_chunk_attn(const bdlm_cache* c, const bdlm_chunk* p, int64_t layer, const void* plan, size_t plan_bytes,
                            bdlm_rows q, bdlm_rows o, float* lse, int64_t lse_pitch, int32_t fill, void* workspace,
                            size_t workspace_bytes, hipStream_t stream);

/*
 * Norms of queries and keys for each head with the position rotation, in one
 * pass: what comes between the projections and any of the attention calls.
 * For a head's row x with weight w (null: ones), at position p_a on axis a:
 *   r = 1 / sqrt(mean x^2 + eps),  n = x r w     (eps 0: no norm, n = x; else within [2^-100, 2^100]),
 * and of the first `dim` elements pair i, on axis axis[i], turns by
 * t = p_axis[i] * freq[i]: (n1, n2) -> (n1 cos t - n2 sin t, n2 cos t + n1 sin t).
 *   q, k, outputs : [rows][heads or kv_heads][head_dim], rows `stride` elements apart
 *     (parts of one fused projection, say).  Outputs may be the inputs (the same
 *     pointer and stride); other overlaps are the caller's error.
 *   positions     : [axes][rows] int32 in device memory, of any sign
 *   weights       : [head_dim] in `dtype`
 * Rounding: angles are formed in 64 bits and reduced there; in bf16 sums and products are
 * fp32 (|x|, and backward |g w|, must be below 2^60), in fp32 the sums over a row are fp64; outputs are rounded
 * once.  A NaN or infinity stays in its head's row (and reaches the weights' gradient).
 */
typedef struct {
  int32_t head_dim;    /* 64 or 128 */
  int32_t dim;         /* elements that turn, a multiple of 16 in [16, head_dim] */
  int32_t interleaved; /* pair i: 0: elements i and i + dim / 2, 1: elements 2 i and 2 i + 1 */
  int32_t axes;        /* 1 to BDLM_MAX_AXES */
  double freq[64];     /* radians per position of pairs 0 .. dim / 2 - 1 */
  int32_t axis[64];
} bdlm_rotary;
#define BDLM_MAX_AXES 4

bdlm_status bdlm_qk_rotate_fwd(const bdlm_rotary* r, int32_t dtype, int64_t rows, const int32_t* positions, int32_t heads,
                               int32_t kv_heads, bdlm_rows q, bdlm_rows k, const void* q_weight, const void* k_weight,
                               double eps, bdlm_rows q_out, bdlm_rows k_out, hipStream_t stream);

/*
 * Backward from the same inputs and the outputs' gradients dq_out, dk_out: dq and dk
 * (which may be dq_out and dk_out), and the weights' gradients [head_dim] in fp32 (null:
 * not wanted; without a norm they must be), the same bits in every call.  However many rows and heads: at most 64
 * products are added one after the other in fp32, those sums in fp64, and the additions are off by less than 2^-17 of
 * the sum of the products' sizes.  workspace:
 * bdlm_qk_rotate_workspace_bytes(), 256-byte aligned, contents ignored on entry, one per call that may
 * overlap in time; not needed where no weight's gradient is wanted.
 */
size_t bdlm_qk_rotate_workspace_bytes(int32_t head_dim);
bdlm_status bdlm_qk_rotate_bwd(const bdlm_rotary* r, int32_t dtype, int64_t rows, const int32_t* positions, int32_t heads,
                               int32_t kv_heads, bdlm_rows q, bdlm_rows k, const void* q_weight, const void* k_weight,
                               double eps, bdlm_rows dq_out, bdlm_rows dk_out, bdlm_rows dq, bdlm_rows dk,
                               float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes,
                               hipStream_t stream);

/*
 * Kernel timing (observability).  While enabled for the calling thread, every
 * kernel the library enqueues is bracketed by two hipEvents recorded on its
 * stream.  bdlm_timing_collect() waits for the recorded events, writes up to
 * max_records (kernel id, milliseconds) pairs in launch order, forgets them and
 * returns how many it wrote (or a negative status).  bdlm_kernel_name() maps an
 * id to a name.  Disabled by default; events are created on first use and
 * reused.
 */
bdlm_status bdlm_timing_enable(int32_t on);
int32_t bdlm_timing_collect(int32_t max_records, int32_t* kernel_ids, float* ms);
const char* bdlm_kernel_name(int32_t kernel_id);

/* Message for the calling thread's last failed call ("" if none). */
const char* bdlm_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* BDLM_ATTN_H */
