/*
 * specverify -- the target model's verify step of speculative decoding with a
 * draft length gamma that changes every step (GammaTune, "Token-Driven
 * GammaTune: Adaptive Calibration for Enhanced Speculative Decoding").
 *
 * C ABI of a CUDA library for NVIDIA B200 (sm_100a).  Three operations make up
 * one verify step; they run back to back on one stream and never synchronise
 * with or read back to the host:
 *
 *   spec_verify_attn    attention of the gamma+1 draft positions against the
 *                       paged bf16 KV cache                     (Section 3 / 5)
 *   spec_accept_sample  accept / reject the drafts, resample or draw the bonus
 *                       token                                   (Section 3)
 *   gamma_tune_update   choose the next gamma from the number accepted
 *                                                               (Section 4.1, Algorithm 1)
 * and, for GammaTune+, spec_draft_stop in front of them         (Section 4.2).
 *
 * General conventions
 *   - Pointers named "device" point to device memory owned by the caller; the
 *     library allocates no device memory and keeps no state between calls
 *     except registered KV-pool handles (host memory), a few per-device facts
 *     it caches on the host (multiprocessor count, occupancy), and the one
 *     built-in scratch array of spec_accept_sample_static with its cached
 *     device address (see there).
 *   - "host" pointers are plain host memory (spec_verify_step_host prefers
 *     pinned memory so that its copies are asynchronous).
 *   - Every call is asynchronous on the given stream (a cudaStream_t passed as
 *     void*; NULL = the default stream) and returns after enqueueing.
 *   - A negative sv_status is an error found on the host before anything was
 *     launched.  Conditions found on the device (a page id outside the pool, a
 *     token id outside the vocabulary, a non-finite softmax sum, gamma outside
 *     [0, gamma_max], a bounded wait that expired) set bits in the caller's
 *     device_status word; the affected sequence is skipped or clamped and the
 *     kernel returns normally.  Nothing traps or asserts on the device.
 *   - Batch notation: B sequences; sequence b has draft length gamma[b] and
 *     R_b = gamma[b]+1 query / target rows starting at row cu_q[b], and
 *     gamma[b] draft rows / tokens / uniforms starting at cu_d[b].  seq_len[b]
 *     is the KV length INCLUDING those R_b positions (their K/V are already in
 *     the cache).  gamma, seq_len, cu_q, cu_d live on the device.
 */
#ifndef SPECVERIFY_H
#define SPECVERIFY_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t sv_status;
enum {
    SV_OK = 0,
    SV_EINVAL = -1,        /* null pointer, non-positive size, inconsistent arguments */
    SV_EUNSUPPORTED = -2,  /* head_dim not 64/128, page_size not 16, hq % hkv != 0, ... */
    SV_EALIGN = -3,        /* a pointer or stride misses the alignment stated below */
    SV_ECUDA = -4,         /* a CUDA runtime / driver call failed (launch, tensor map) */
    SV_EWORKSPACE = -5     /* workspace missing or smaller than the size query says */
};

/* bits of the device status word */
enum {
    SV_DEV_BAD_GAMMA = 1,   /* gamma[b] outside [0, gamma_max]: clamped */
    SV_DEV_BAD_PAGE = 2,    /* block-table entry outside [0, n_pages): attention reads that page as zeros
                               and the outputs of that sequence are unspecified (other sequences are
                               unaffected); the cache append skips that position */
    SV_DEV_BAD_TOKEN = 4,   /* draft token outside [0, vocab): position rejected */
    SV_DEV_NONFINITE = 8,   /* softmax sum not finite (NaN / +Inf logit): sequence emits -1 */
    SV_DEV_TIMEOUT = 16,    /* a bounded device-side wait expired (also: a kernel found its shared
                               memory misaligned and did nothing) */
    SV_DEV_BAD_LEN = 32,    /* seq_len[b] < gamma[b]+1 or beyond the block table: sequence skipped */
    SV_DEV_NO_PAGES = 64    /* fewer free pages than a sequence asks for: its pages stay as they were */
};

const char *sv_status_str(sv_status s);

/* ---------------------------------------------------------------- KV pool */
/*
 * A paged KV pool: K and V arrays of n_pages pages, each page holding
 * page_size (= 16) token slots for hkv heads of head_dim bf16 values.
 * strides[4] = element strides for (page, kv head, slot, dim); dim stride must
 * be 1, the others multiples of 8 elements (16 bytes); both base pointers
 * 16-byte aligned.  [page, head, slot, dim] and [page, slot, head, dim] are
 * both expressible.  Registration builds the TMA tensor maps on the host; the
 * handle is host memory released by spec_kv_pool_release.  Slots past a
 * sequence's seq_len inside its last page are read (and multiplied by zero
 * weights), so pool memory must hold finite values.
 */
typedef struct sv_kv_pool *sv_kv_pool_t;

sv_status spec_kv_pool_register(const void *k_pool_device, const void *v_pool_device,
                                int64_t n_pages, int32_t page_size, int32_t hkv, int32_t head_dim,
                                const int64_t strides[4], sv_kv_pool_t *out);
sv_status spec_kv_pool_release(sv_kv_pool_t pool);

/* ---------------------------------------------------------------- norm, rotation and append in one pass */
/*
 * What a target layer does between its projection and the verify attention
 * (KV caching, paper Section 5), for every row r with slot_map[r] >= 0:
 *   y = x * w / sqrt(mean_d(x_d^2) + eps)    each query head with q_weight, each key head with
 *                                            k_weight; y = x where that pointer is NULL
 *   for each frequency f < rot_dim / 2, with the pair (a, b) = (f, f + rot_dim/2), or (2f, 2f+1)
 *   if interleaved, and the angle t = positions[axis of f][r] * inv_freq[f]:
 *       z_a = scale * (y_a cos t - y_b sin t) ;  z_b = scale * (y_b cos t + y_a sin t)
 *   z_d = y_d for d >= rot_dim
 * Queries go to q_out, keys to slot slot_map[r] % 16 of page slot_map[r] / 16 of the pool, values
 * there unchanged.  Rows with a negative slot (padding, as spec_kv_pages_update marks it) write
 * nothing: their part of q_out stays as it is.  A row is any position: draft blocks, single tokens, prompts.
 * bf16 inputs, float32 arithmetic, one rounding to bf16 at the end.  The angle keeps its digits at
 * far positions: a frequency becomes a 64-bit fraction of a turn, and the product with the
 * position, in 64-bit integers, drops whole turns exactly before the rest goes to float32.
 * Slots of different rows must differ.  q_out may be q itself where q's rows are contiguous; it
 * must not overlap q otherwise, nor k_new or v_new (SV_EINVAL).
 * A slot at or beyond n_pages * 16 -> SV_DEV_BAD_PAGE, row skipped.  One launch; n_rows == 0
 * returns SV_OK without one.
 */
typedef struct sv_rope_append_params {
    const void *q;              /* device bf16, row r at r * q_stride: [hq, head_dim] contiguous */
    int64_t q_stride;           /* elements between rows (a fused projection's width, for one), a multiple of 8 */
    const void *k_new;          /* device bf16, rows of [hkv, head_dim] */
    int64_t k_stride;
    const void *v_new;          /* device bf16, rows of [hkv, head_dim] */
    int64_t v_stride;
    void *q_out;                /* device bf16 [n_rows, hq, head_dim]; all four 16-byte aligned */
    sv_kv_pool_t pool;          /* head_dim a multiple of 16 */
    int32_t hq;                 /* at most 2^20, as the pool's heads */
    int64_t n_rows;             /* <= 2^30 */
    const int64_t *slot_map;    /* device [n_rows] */
    const int32_t *positions;   /* device [n_axes, n_rows] */
    int32_t n_axes;             /* position axes (1; 3 for time, height, width) */
    const uint8_t *freq_axis;   /* device [rot_dim/2]: axis of each frequency (one >= n_axes: the last), or NULL: axis 0 */
    const double *inv_freq;     /* device [rot_dim/2]; NULL if rot_dim is 0 */
    int32_t rot_dim;            /* rotated dims: a multiple of 16, 0 .. head_dim */
    int32_t interleaved;        /* 0: pairs (f, f + rot_dim/2); 1: pairs (2f, 2f+1) */
    float rope_scale;           /* factor of the rotated dims, usually 1 */
    const void *q_weight;       /* device [head_dim], 16-byte aligned, or NULL: queries are not normalised */
    const void *k_weight;       /* device [head_dim], 16-byte aligned, or NULL: keys are not normalised */
    int32_t weights_f32;        /* 0: the weights are bf16, 1: float32 */
    float eps;                  /* >= 0 */
    uint32_t *device_status;    /* device, one word, OR-ed into; may be NULL */
} sv_rope_append_params;

sv_status spec_rope_append(const sv_rope_append_params *p, void *stream);

/* ---------------------------------------------------------------- block tables and slot maps */
/*
 * The controller moves every seq_len[b] on the device (gamma_tune_update), so the
 * pages behind the sequences have to follow there as well (KV caching, paper
 * Section 5).  This call brings the block table to the lengths of the coming
 * step, taking pages from a stack of free ones and giving back those that a
 * shorter or finished sequence no longer needs, and lists where each row of the
 * step goes.  With need[b] = ceil(seq_len[b] / 16):
 *   1. release, in the order of b: columns need[b] .. n_held[b]-1 of row b (if any)
 *      are pushed on the stack free_list[0 .. n_free) in column order and their
 *      table entries become -1;
 *   2. acquire, in the order of b: columns n_held[b] .. need[b]-1 (if any) are
 *      popped one after the other.  A sequence gets all the pages it asks for or
 *      none, and the first that goes without stops the acquisition for those
 *      behind it (SV_DEV_NO_PAGES; they keep what they held);
 *   3. n_held[b] = need[b] where that succeeded, *n_free the pages left.
 * seq_len[b] = 0 is a sequence that is not (or no longer) there: it gives back
 * all its pages.  Pages released by a call serve the acquisitions of the same call.
 * The outcome does not depend on the launch: ids move in the order stated.
 * Rows (only with slot_map / positions): row r belongs to the sequence b with
 * cu_q[b] <= r < cu_q[b+1] as its position i = r - cu_q[b]; for i <= gamma[b]
 *     positions[r] = seq_len[b] - (gamma[b]+1) + i
 *     slot_map[r]  = page * 16 + positions[r] % 16
 * and both are -1 in every other row below n_rows (padding, rows behind the last
 * sequence, sequences that are absent, skipped or without their pages).
 * Device-detected: seq_len[b] < 0 or beyond the table row, or n_held[b] outside
 * [0, block_table_stride] -> SV_DEV_BAD_LEN, sequence left as it is; 0 <
 * seq_len[b] < gamma[b]+1 -> SV_DEV_BAD_LEN, its rows are -1; gamma[b] out of
 * range -> SV_DEV_BAD_GAMMA, clamped; *n_free outside [0, n_pages] or more pages
 * given back than the pool has -> SV_DEV_BAD_PAGE, clamped / dropped; a table
 * entry under a row outside [0, n_pages) -> SV_DEV_BAD_PAGE, its slot is -1.
 * block_table, n_held, free_list and n_free are the caller's state; a new pool
 * starts with n_held = 0, table entries -1, free_list = the page ids in any order
 * and *n_free their number.  One launch up to 384 sequences, two above; no workspace.
 */
typedef struct sv_kv_pages_params {
    const int32_t *seq_len;     /* device [batch]: lengths to provide for (draft block included) */
    int32_t batch;              /* at most 8192 */
    int32_t *block_table;       /* device in/out [batch, block_table_stride] */
    int64_t block_table_stride; /* elements between rows; batch * block_table_stride <= 2^30 */
    int32_t *n_held;            /* device in/out [batch]: pages each sequence holds */
    int32_t *free_list;         /* device in/out [n_pages]: the stack; entries at and above *n_free are scratch */
    int32_t *n_free;            /* device in/out, one word */
    int64_t n_pages;            /* pages of the pool, < 2^30 */
    int32_t page_size;          /* 16 */
    const int32_t *gamma;       /* device [batch]; gamma and cu_q may be NULL when slot_map and positions are */
    const int32_t *cu_q;        /* device [batch+1], not decreasing */
    int32_t gamma_max;          /* upper bound of gamma[b] */
    int64_t *slot_map;          /* device out [n_rows], or NULL */
    int32_t *positions;         /* device out [n_rows], or NULL */
    int64_t n_rows;             /* rows of slot_map / positions, < 2^31 */
    uint32_t *device_status;    /* device, one word, OR-ed into; may be NULL */
} sv_kv_pages_params;

sv_status spec_kv_pages_update(const sv_kv_pages_params *p, void *stream);

/* ---------------------------------------------------------------- attention */
/*
 * Paper Section 3: the target verifies the gamma drafted tokens in one parallel
 * forward; with KV caching (Section 5) the context-dependent part of it is
 * this causal attention.  For sequence b, row i in [0, gamma[b]], query head h:
 *     pos = seq_len[b] - (gamma[b]+1) + i ;  kv head = h / (hq / hkv)
 *     s_j = sm_scale * <q, k_j>   for j = 0 .. pos
 *     o   = sum_j softmax(s)_j v_j ;   lse = ln sum_j exp(s_j)
 * bf16 inputs, fp32 accumulation and softmax, bf16 output.  A row with a score that is NaN or +inf, or with nothing but
 * scores of -inf, gives NaN.
 */
typedef struct sv_attn_params {
    const void *q;              /* device bf16 [n_rows, hq, head_dim], 16-byte aligned */
    void *o;                    /* device bf16 [n_rows, hq, head_dim], 16-byte aligned */
    float *lse;                 /* device fp32 [n_rows, hq], or NULL */
    sv_kv_pool_t pool;
    const int32_t *block_table; /* device [batch, block_table_stride]: physical page of logical page */
    int64_t block_table_stride; /* elements between rows; >= ceil(max_seq_len / 16) */
    const int32_t *seq_len;     /* device [batch] */
    const int32_t *gamma;       /* device [batch] */
    const int32_t *cu_q;        /* device [batch+1] */
    int32_t batch;
    int32_t gamma_max;          /* upper bound of gamma[b]; sizes the row tile */
    int32_t hq, hkv, head_dim;
    int32_t max_seq_len;        /* upper bound of seq_len[b]; sizes the grid and the workspace */
    float sm_scale;             /* usually 1/sqrt(head_dim) */
    uint32_t *device_status;    /* device, one word, OR-ed into; may be NULL */
} sv_attn_params;

/* Bytes of device scratch spec_verify_attn needs for these bounds (partial
 * results of sequences whose keys are split over several thread blocks). */
size_t spec_verify_attn_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t hq, int32_t hkv,
                                        int32_t head_dim, int32_t max_seq_len);

sv_status spec_verify_attn(const sv_attn_params *p, void *workspace_device, size_t workspace_bytes,
                           void *stream);

/* ---------------------------------------------------------------- cache append */
/*
 * KV caching (paper Section 5, experimental setup): before the verify
 * attention runs, the keys and values of the gamma[b]+1 new positions are
 * written behind each sequence's context.  New row i of sequence b (row
 * cu_q[b]+i of k_new / v_new) is token
 *     pos = seq_len[b] - (gamma[b]+1) + i
 * (seq_len already counts the block) and goes to physical page
 * block_table[b][pos / 16], slot pos % 16 of every kv head.  A copy of bf16
 * bit patterns; nothing else in the pools is touched.  Rolling rejected
 * positions back needs no copy: gamma_tune_update shortens seq_len, and the
 * next append overwrites them.
 * The pool memory (registered through const pointers for the attention) is
 * written by this call; the caller owns it and orders the call before the
 * attention on the same stream.
 * Device-detected: gamma[b] out of range -> SV_DEV_BAD_GAMMA, clamped;
 * seq_len[b] < gamma[b]+1 or a position beyond the block table row ->
 * SV_DEV_BAD_LEN, sequence skipped; a page id outside [0, n_pages) ->
 * SV_DEV_BAD_PAGE, that position skipped.
 */
typedef struct sv_kv_append_params {
    const void *k_new;          /* device bf16 [n_rows, hkv, head_dim], 16-byte aligned */
    const void *v_new;          /* device bf16 [n_rows, hkv, head_dim], 16-byte aligned */
    sv_kv_pool_t pool;          /* head_dim a multiple of 8 */
    const int32_t *block_table; /* device [batch, block_table_stride] */
    int64_t block_table_stride;
    const int32_t *seq_len;     /* device [batch] */
    const int32_t *gamma;       /* device [batch] */
    const int32_t *cu_q;        /* device [batch+1] */
    int32_t batch;
    int32_t gamma_max;          /* upper bound of gamma[b]; sizes the grid */
    uint32_t *device_status;    /* device, one word, OR-ed into; may be NULL */
} sv_kv_append_params;

sv_status spec_kv_append(const sv_kv_append_params *p, void *stream);

/* ---------------------------------------------------------------- bounds of every page's keys */
/*
 * Long contexts (KV caching, paper Section 5): instead of all of its cache a row may read the pages that matter to it,
 * found by a cheap score on a summary of every page.  This call keeps the summary, next to the cache append.  For every
 * page of sequence b that holds a position of [start, seq_len[b]), with start = seq_len[b] - (gamma[b]+1), or first[b]
 * where first is given (gamma NULL), and for every kv head, over the page's positions below seq_len[b]:
 *     M_d = max k_d,  m_d = min k_d,  scale = max_d max(|M_d|, |m_d|) * (1/127)
 *     bounds[page][head][0][d] = round(M_d / scale),  bounds[page][head][1][d] = round(m_d / scale)
 * float32, each operation and the constant 1/127 rounded once, round half to even.  The bounds are 0 where scale is 0 or
 * not finite; a key that is NaN makes it NaN.  Other pages' entries stay.  seq_len[b] = 0 is an absent sequence.  A page
 * that two sequences bring up to date is written by both; they have to fill it alike.
 * Device-detected: gamma[b] outside [0, max_new) -> SV_DEV_BAD_GAMMA, clamped; a start below 0, more than max_new
 * positions or a length beyond the table row -> SV_DEV_BAD_LEN, sequence skipped; a page id outside the pool ->
 * SV_DEV_BAD_PAGE, page skipped.  One launch.
 */
typedef struct sv_page_bounds_params {
    sv_kv_pool_t pool;          /* head_dim 64 or 128 */
    int8_t *bounds;             /* device in/out [n_pages, hkv, 2, head_dim], 16-byte aligned */
    float *scales;              /* device in/out [n_pages, hkv] */
    const int32_t *block_table; /* device [batch, block_table_stride] */
    int64_t block_table_stride;
    const int32_t *seq_len;     /* device [batch] */
    const int32_t *gamma;       /* device [batch], or NULL: first */
    const int32_t *first;       /* device [batch], or NULL: gamma */
    int32_t batch;
    int32_t max_new;            /* upper bound of the positions of a sequence (gamma_max + 1 behind a draft block); sizes the grid */
    uint32_t *device_status;    /* device, one word, OR-ed into; may be NULL */
} sv_page_bounds_params;

sv_status spec_page_bounds_update(const sv_page_bounds_params *p, void *stream);

/* ---------------------------------------------------------------- pages that a row reads */
/*
 * For row i of sequence b's block at position pos = seq_len[b] - (gamma[b]+1) + i (the pages 0 .. pos / 16 are before it)
 * and kv head g, with the group's query heads h:
 *     s = max_{h,d} |q_hd| * (1/127),  qi_hd = round(q_hd / s)                (as above; at most 127 in magnitude; all 0
 *                                                                              where one of the queries is not finite)
 *     score(page) = scales[page] * max_h sum_d max(qi_hd bounds[page][g][0][d], qi_hd bounds[page][g][1][d])
 * The row reads the first n_first pages, the last n_last up to and including its own, and of the others those with the
 * highest scores (one that is NaN, as the scale of a page whose keys are not all finite gives it, counts as the highest),
 * the lower page on ties, n_select in all (all of them where there are no more).  The sum is of whole numbers and the
 * product with the scale is rounded once, so a row of a block reads the pages that the same position would have read
 * decoded alone: n_last >= 1 keeps pages with keys behind the row out of the comparison.
 * Choice and listed pages together are worth it (B200, 64 pages a row) for single tokens from some 20000 tokens of one
 * sequence, 4000 of 16 or 2000 of 128; for blocks where the pages of all rows together are a small part of the cache.
 * Output per sequence and kv head: the pages that any row of the block reads, in ascending order (indices into the block
 * table row), and for each the rows that do (bit i: row i).  Entries at and beyond n_list are left as they are.  A skipped
 * sequence has n_list 0.
 * Device-detected: gamma[b] out of range -> SV_DEV_BAD_GAMMA, clamped; seq_len[b] < gamma[b]+1 or > max_seq_len ->
 * SV_DEV_BAD_LEN, sequence skipped; a page id outside [0, n_pages) -> SV_DEV_BAD_PAGE, that page's score is 0.
 * Two launches; one where max_seq_len tokens have no more than n_select pages.
 */
typedef struct sv_page_select_params {
    const void *q;              /* device bf16 [n_rows, hq, head_dim], 16-byte aligned: what the attention reads */
    const int8_t *bounds;       /* device [n_pages, hkv, 2, head_dim], 16-byte aligned */
    const float *scales;        /* device [n_pages, hkv] */
    int64_t n_pages;
    const int32_t *block_table; /* device [batch, block_table_stride] */
    int64_t block_table_stride; /* elements between rows; >= ceil(max_seq_len / 16) */
    const int32_t *seq_len;     /* device [batch] */
    const int32_t *gamma;       /* device [batch] */
    const int32_t *cu_q;        /* device [batch+1] */
    int32_t batch;
    int32_t gamma_max;          /* at most 63 */
    int32_t hq, hkv, head_dim;  /* head_dim 64 or 128, hq / hkv at most 128 */
    int32_t max_seq_len;        /* upper bound of seq_len[b]; sizes the grid and the workspace */
    int32_t n_select;           /* pages of a row, >= n_first + n_last */
    int32_t n_first;            /* >= 0 */
    int32_t n_last;             /* >= 1 */
    int32_t *page_list;         /* device out [batch, hkv, list_stride] */
    uint64_t *row_mask;         /* device out [batch, hkv, list_stride] */
    int32_t *n_list;            /* device out [batch, hkv] */
    int64_t list_stride;        /* >= min(ceil(max_seq_len / 16), (gamma_max+1) * n_select) */
    uint32_t *device_status;    /* device, one word, OR-ed into; may be NULL */
} sv_page_select_params;

/* Bytes of device scratch for these bounds (the scores of all rows). */
size_t spec_page_select_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t hkv, int32_t max_seq_len);

sv_status spec_page_select(const sv_page_select_params *p, void *workspace_device, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------- attention over listed pages */
/*
 * spec_verify_attn where row i of sequence b reads, for kv head g, only the keys of those listed pages whose mask has bit
 * i set (and, as there, none behind its position): j runs over the positions of pages page_list[b][g][e], e <
 * n_list[b][g], with bit i of row_mask[b][g][e].  A row without any key gives o = 0 and lse = -inf (so does one whose
 * scores are all -inf); one with a score that is NaN or +inf gives NaN in both.  The lists are those of spec_page_select,
 * or any others: pages in any order, each once.
 * Arguments of attn as in spec_verify_attn; gamma_max at most 63, hq / hkv at most 128, max_seq_len at most 2^31 - 65.
 * Device-detected: as spec_verify_attn; a listed page outside the sequence's pages -> SV_DEV_BAD_PAGE, not read; n_list
 * outside [0, list_stride] -> SV_DEV_BAD_LEN, clamped.  Two launches.
 */
typedef struct sv_attn_pages_params {
    sv_attn_params attn;
    const int32_t *page_list;   /* device [batch, hkv, list_stride] */
    const uint64_t *row_mask;   /* device [batch, hkv, list_stride] */
    const int32_t *n_list;      /* device [batch, hkv] */
    int64_t list_stride;
} sv_attn_pages_params;

size_t spec_verify_attn_pages_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t hq, int32_t hkv, int32_t head_dim);

sv_status spec_verify_attn_pages(const sv_attn_pages_params *p, void *workspace_device, size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------- attention behind shared prefixes */
/*
 * spec_verify_attn (the same result up to rounding) of a batch in which groups of sequences share the pages of a long
 * prefix: the prefix's keys and values are read once per group and meet all of its rows together.
 * Sequence b belongs to group[b] (0 .. n_groups-1; -1: to none).  The first prefix_len[g] / 16 entries (whole pages; a
 * rest counts to the sequences) of the members' block table rows must be the same pages.  A member whose block begins
 * inside these pages (seq_len[b] - (gamma[b]+1) < 16 * pages) is computed by itself; so is the only member of a group.
 * Worth it (B200) where spec_verify_attn would read (members - 1) * prefix_len * hkv * head_dim * 4 bytes again that are
 * 300 MB or more, with up to some 40 rows (positions * hq / hkv) to a member and kv head; 1 GB with 136 rows, and not for a
 * hundred such members.
 * Device-detected: as spec_verify_attn; group[b] outside [-1, n_groups) or prefix_len[g] negative or beyond the table
 * row -> SV_DEV_BAD_LEN, the sequence or group is computed without sharing.  Five launches.
 */
typedef struct sv_attn_prefix_params {
    sv_attn_params attn;        /* batch at most 8192, gamma_max at most 4095, hq / hkv at most 128, max_seq_len at most 2^31 - 65 */
    const int32_t *group;       /* device [batch] */
    const int32_t *prefix_len;  /* device [n_groups], tokens */
    int32_t n_groups;           /* 1 .. batch */
} sv_attn_prefix_params;

size_t spec_verify_attn_prefix_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t hq, int32_t hkv, int32_t head_dim,
                                               int32_t n_groups);

sv_status spec_verify_attn_prefix(const sv_attn_prefix_params *p, void *workspace_device, size_t workspace_bytes,
                                  void *stream);

/* ---------------------------------------------------------------- all layers of a step */
/*
 * A target model keeps one KV cache per layer (KV caching, paper Section 5), all
 * with the same paging: one block table, one set of lengths.  This call runs the
 * cache append and the verify attention of n_layers caches in one enqueue: first
 * ONE launch writes every layer's new keys and values (spec_kv_append for all
 * layers at once; skipped when k_new is NULL), then the attention of layer 0, 1,
 * ... in order, each reading its own pool, queries and writing its own output.
 * In a real model layer l+1's queries depend on layer l's output through the
 * projections in between, which are outside this library; here they are inputs.
 * pools / q / o / k_new / v_new / lse are HOST arrays of n_layers entries
 * (device pointers inside); everything else is shared and means what it means in
 * sv_attn_params.  The workspace is the one spec_verify_attn asks for (it is
 * reused layer after layer).  Errors: as spec_verify_attn / spec_kv_append; the
 * pools must agree in hkv and head_dim.
 */
typedef struct sv_attn_layers_params {
    int32_t n_layers;
    const sv_kv_pool_t *pools;    /* host [n_layers] */
    const void *const *q;         /* host [n_layers] of device bf16 [n_rows, hq, head_dim] */
    void *const *o;               /* host [n_layers] of device bf16 [n_rows, hq, head_dim] */
    float *const *lse;            /* host [n_layers] of device fp32 [n_rows, hq], or NULL */
    const void *const *k_new;     /* host [n_layers] of device bf16 [n_rows, hkv, head_dim], or NULL: no append */
    const void *const *v_new;     /* host [n_layers], NULL exactly when k_new is */
    sv_attn_params shared;        /* q, o, lse and pool of this struct are ignored */
} sv_attn_layers_params;

sv_status spec_verify_attn_layers(const sv_attn_layers_params *p, void *workspace_device,
                                  size_t workspace_bytes, void *stream);

/* ---------------------------------------------------------------- penalties, biases and grammar masks */
/*
 * What a request asks for on top of the model's distribution, applied to the
 * logits that spec_accept_sample (target rows) or spec_draft_step (draft rows)
 * then reads (paper Section 3: both sides sample from these rows).  For element
 * k of a row, with C the times token k stands in the row's history, and S = k is
 * in the history or in the prompt:
 *     x1 = S ? (x > 0 ? x / repetition : x * repetition) : x
 *     x2 = x1 - (frequency * C + (C > 0 ? presence : 0))
 *     x3 = x2 + bias[k]
 *     out = mask bit k is clear ? -inf : x3
 * The history of target row i of a block is what the sequence has generated
 * (token_counts) and the drafts x_0 .. x_{i-1} in front of the row, so that the
 * row is what decoding token by token would have seen; that of a draft row is
 * token_counts and the n_drafted[b] tokens drafted so far.
 * A masked element is -inf whatever it held (NaN too); a row with nothing
 * allowed is all -inf, which spec_accept_sample reports (SV_DEV_NONFINITE).
 * float32 arithmetic, one rounding to the logits' type at the end.
 * Target rows (n_drafted == NULL): rows cu_q[b] .. cu_q[b] + gamma[b]; rows of
 * no sequence are left as they are.  Draft rows (n_drafted != NULL): row b.
 * out may be logits itself (same stride): what does not change is then neither
 * read nor written where the mask and the counts show it and 128-bit access is
 * enabled, and written as it was elsewhere.  Otherwise the two must not overlap,
 * from the first element to the last (SV_EINVAL).
 * A bias list that names a token twice: the later entry counts.
 * Device-detected: gamma[b], or with penalties n_drafted[b], outside [0, gamma_max]
 * -> SV_DEV_BAD_GAMMA, clamped; a block with rows beyond n_rows -> SV_DEV_BAD_LEN,
 * left as it is; drafts beyond n_d_rows -> SV_DEV_BAD_LEN, not counted; a draft or bias token outside
 * [0, vocab) -> SV_DEV_BAD_TOKEN, ignored.  One launch, no workspace.
 */
typedef struct sv_logits_adjust_params {
    const void *logits;         /* device [n_rows, row_stride] float32, or bf16 if logits_bf16 */
    void *out;                  /* device [n_rows, out_stride], the same type */
    int64_t row_stride;         /* elements between rows (>= vocab); both strides multiples of 4 (bf16: 8) with 16-byte */
    int64_t out_stride;         /* aligned bases enable 128-bit access */
    int64_t n_rows;
    int32_t vocab;              /* at most 2^30 (SV_EUNSUPPORTED, as the next limit); 128-bit access needs a multiple of 4 (bf16: 8) */
    int32_t logits_bf16;
    int32_t batch;
    int32_t gamma_max;          /* at most 64 */
    const int32_t *gamma;       /* device [batch]; target rows only */
    const int32_t *cu_q;        /* device [batch+1]; target rows only */
    const int32_t *cu_d;        /* device [batch+1]: first draft token of each sequence; with penalties and gamma_max > 0 */
    const int32_t *n_drafted;   /* device [batch]: draft rows; NULL: target rows */
    const int32_t *active;      /* device [batch] or NULL: the rows of sequences with active[b] == 0 are left as they are */
    const int32_t *draft_tokens;/* device [n_d_rows]; with penalties and gamma_max > 0 */
    int64_t n_d_rows;
    const int16_t *token_counts;/* device [batch, count_stride], see spec_token_counts_update; needed by the penalties */
    int64_t count_stride;       /* a multiple of 8, >= vocab; base 16-byte aligned */
    const float *repetition;    /* device [batch], > 0 (1: none), or NULL */
    const float *frequency;     /* device [batch] or NULL */
    const float *presence;      /* device [batch] or NULL */
    const int32_t *bias_tokens; /* device [batch, bias_stride], or NULL */
    const float *bias_values;   /* device [batch, bias_stride] */
    const int32_t *n_bias;      /* device [batch]: entries of each list, at most bias_stride (more: clamped, SV_DEV_BAD_LEN) */
    int32_t bias_stride;        /* at most 2^30 */
    const uint32_t *mask;       /* device [n_rows, mask_stride]: bit k % 32 of word k / 32 set = token k allowed; 4-byte aligned, or NULL */
    int64_t mask_stride;        /* words between rows, >= ceil(vocab / 32) */
    uint32_t *device_status;    /* device, one word, OR-ed into; may be NULL */
} sv_logits_adjust_params;

sv_status spec_logits_adjust(const sv_logits_adjust_params *p, void *stream);

/*
 * The counts behind the penalties, kept on the device: token_counts[b][k] holds
 * the times token k was generated in its low 15 bits (saturating at 32767) and in
 * bit 15 whether it stands in the prompt.  One call, per sequence b:
 *   reset[b] != 0: the row's vocab entries are cleared first (a request is admitted);
 *   then each of its tokens is counted (prompt == 0), or marked (prompt != 0).
 * Tokens of b: row b of tokens [batch, token_stride], max_tokens of them, or, with
 * cu_tokens, tokens[cu_tokens[b]] .. tokens[cu_tokens[b+1] - 1].  Entries of -1
 * are skipped, so out_tokens of spec_accept_sample (token_stride = max_tokens =
 * gamma_max + 1) is counted as it stands, padding and all.
 * The result does not depend on the order in which tokens are counted.
 * Device-detected: another token outside [0, vocab) -> SV_DEV_BAD_TOKEN, skipped;
 * a range of cu_tokens outside [0, n_tokens] or longer than max_tokens ->
 * SV_DEV_BAD_LEN, none of that sequence's tokens are counted.  One launch.
 */
typedef struct sv_token_counts_params {
    int16_t *token_counts;      /* device in/out [batch, count_stride], 16-byte aligned */
    int64_t count_stride;       /* elements between rows: a multiple of 8, >= vocab */
    int32_t vocab;              /* at most 2^30, as max_tokens */
    int32_t batch;
    const int32_t *tokens;      /* device; may be NULL if max_tokens is 0 (reset alone) */
    int64_t token_stride;       /* elements between rows, >= max_tokens; not used with cu_tokens */
    const int32_t *cu_tokens;   /* device [batch+1], or NULL */
    int64_t n_tokens;           /* entries of tokens; used with cu_tokens */
    int32_t max_tokens;         /* most tokens of a sequence; sizes the grid (without reset, a warp per 32 of them and sequence) */
    const int32_t *reset;       /* device [batch] or NULL: nothing is cleared */
    int32_t prompt;
    uint32_t *device_status;    /* device, one word, OR-ed into; may be NULL */
} sv_token_counts_params;

sv_status spec_token_counts_update(const sv_token_counts_params *p, void *stream);

/* ---------------------------------------------------------------- accept / resample */
/*
 * Speculative sampling (paper Section 3, after Leviathan et al. and Chen et
 * al.).  Per sequence, with T = its temperature, target rows t_0..t_gamma and
 * draft rows d_0..d_{gamma-1}, draft tokens x_i, uniforms u_i and u_s:
 *   T > 0:  p_i = softmax(t_i / T), q_i = softmax(d_i / T)
 *           ratio_i = min(1, p_i[x_i] / q_i[x_i]); accept while u_i < ratio_i;
 *           n = index of the first rejection (gamma if none)
 *           n < gamma: next ~ normalise(max(0, p_n - q_n))  (p_n if that is all zero)
 *           n = gamma: next ~ p_gamma                        (the bonus token)
 *           both by inverse CDF in vocabulary order with u_s
 *           (smallest k with sum_{j<=k} w_j > u_s * sum_j w_j).
 *   T == 0: n = first i with argmax(t_i) != x_i (lowest index wins ties),
 *           next = argmax(t_n); draft logits and uniforms are not read.
 * Softmax sums are accumulated in float64 from float32 exponentials; the
 * ratio, the comparison and the sampled row are evaluated in float64.
 * The paper's largest target runs with reduced precision (Section 5); logits
 * stored as bf16 are accepted too (logits_bf16), which halves the bytes of
 * this step.
 */
typedef struct sv_accept_params {
    const float *target_logits;   /* device fp32 [n_q_rows, row_stride] */
    const float *draft_logits;    /* device fp32 [n_d_rows, row_stride]; may be NULL if all T == 0 */
    int64_t row_stride;           /* elements between rows (>= vocab); a multiple of 4 with
                                     16-byte aligned bases enables 128-bit loads */
    int32_t vocab;
    const int32_t *draft_tokens;  /* device [n_d_rows] */
    const float *u_accept;        /* device [n_d_rows], in [0,1) */
    const float *u_sample;        /* device [batch], in [0,1) */
    float temperature;            /* used when temperature_per_seq is NULL */
    const float *temperature_per_seq; /* device [batch] or NULL */
    const int32_t *gamma;         /* device [batch] */
    const int32_t *cu_q;          /* device [batch+1] */
    const int32_t *cu_d;          /* device [batch+1] */
    int32_t batch;
    int32_t gamma_max;
    int32_t *n_accepted;          /* device out [batch]: accepted drafts, 0..gamma (extra token not counted) */
    int32_t *out_tokens;          /* device out [batch, gamma_max+1]: accepted drafts, next token, then -1 */
    double *ratio;                /* device out [n_d_rows] or NULL (NaN past the first rejection) */
    double *logZ_p;               /* device out [n_q_rows] or NULL: ln sum exp(t/T) */
    double *logZ_q;               /* device out [n_d_rows] or NULL: ln sum exp(d/T) */
    uint32_t *flag_count;         /* device, one word or NULL: += positions with |u - ratio| < 1e-6 */
    uint32_t *device_status;      /* device, one word or NULL */
    int32_t logits_bf16;          /* 0: the logits are float32 (as declared).  1: target_logits / draft_logits
                                     point to bf16 values (2 bytes each, row_stride still in elements; a
                                     multiple of 8 with 16-byte aligned bases enables 128-bit loads); every
                                     value is widened exactly to float32 and the arithmetic is unchanged, so
                                     the result is that of the float32 call on the widened values at half
                                     the bytes */
} sv_accept_params;

size_t spec_accept_sample_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t vocab);

sv_status spec_accept_sample(const sv_accept_params *p, void *workspace_device,
                             size_t workspace_bytes, void *stream);

/*
 * spec_accept_sample without a workspace argument and without any allocation.
 * The paper has no counterpart to this entry point; it exists for callers that
 * are not able to obtain device scratch memory themselves: code running where
 * every device buffer was fixed at start-up (a serving engine whose memory pool
 * is fully handed out, a plugin that is only given its input and output
 * tensors), or code that must not call cudaMalloc at this point because an
 * allocation would synchronise the device or is forbidden by the host
 * framework's rules.  The computation and the results are those of
 * spec_accept_sample; only the place of the intermediate slice statistics
 * differs: they go to an array of SV_ACCEPT_STATIC_SCRATCH_BYTES bytes that is
 * built into the library (each GPU that loads the library carries it until the
 * process ends).
 *   - Limit: the intermediate results -- 32 bytes per (row, slice of the
 *     vocabulary) with batch * (2*gamma_max + 1) rows and slices of 2048 to 16384
 *     elements (the library picks larger slices when there are many rows), plus
 *     24 bytes per 128 vocabulary entries per sequence for the sampling pass --
 *     must fit in SV_ACCEPT_STATIC_SCRATCH_BYTES.  The largest configuration of
 *     the tests (batch 128, gamma_max 16, vocab 128256) needs about 4.2 MB.  A
 *     larger problem is refused with SV_EWORKSPACE before anything is launched;
 *     use spec_accept_sample then.
 *   - The first call on each device looks up the array's device address
 *     (cudaGetSymbolAddress) with that device current; make that first call
 *     outside any stream capture.  No call allocates or frees memory.
 *   - All calls on one device share the array and it keeps whatever the previous
 *     call left there.  Nothing needs clearing: every record a call reads was
 *     written earlier in that same call.  Two calls whose kernels can overlap on
 *     the GPU (different streams without an ordering between them) race on the
 *     array and give wrong results; keep such calls on one stream or order them
 *     with events.
 */
#define SV_ACCEPT_STATIC_SCRATCH_BYTES (8u << 20)
sv_status spec_accept_sample_static(const sv_accept_params *p, void *stream);

/* ---------------------------------------------------------------- GammaTune */
/*
 * Paper Section 4.1, Algorithm 1, one update per sequence, state on the device:
 *   SV_GT_PROPOSED  A' = A + delta if A == gamma else A      (Eq. 7 feeding the average,
 *                   gbar <- min(gmax, max(gmin, (1-eta) gbar + eta A'))   (Eq. 8)   as the prose says)
 *                   gamma <- ceil(gbar)
 *   SV_GT_LITERAL   the listing as printed: the average is fed A itself
 *   SV_GT_FIXED     gamma and gbar stay (plain speculative decoding)
 * binary64 throughout, each product and the sum rounded separately (no fused
 * multiply-add), so trajectories are reproducible bit for bit.
 * Bookkeeping done in the same kernel:
 *   seq_len <- seq_len - (gamma+1) + (A+1) + (gamma_next+1)
 *   cu_q, cu_d <- prefix sums of gamma_next+1 / gamma_next, or b*(gamma_max+1) /
 *   b*gamma_max when padded_rows != 0 (fixed row slabs per sequence).
 */
enum { SV_GT_FIXED = 0, SV_GT_PROPOSED = 1, SV_GT_LITERAL = 2 };

typedef struct sv_gamma_config {
    double eta;          /* adaptation rate in [0, 1] */
    double delta;        /* expansion offset */
    int32_t gamma_min;   /* >= 0 */
    int32_t gamma_max;   /* >= gamma_min */
    int32_t mode;        /* SV_GT_* */
    int32_t padded_rows; /* row-offset convention, see above */
} sv_gamma_config;

typedef struct sv_gamma_params {
    const int32_t *n_accepted;  /* device [batch] */
    double *gamma_bar;          /* device in/out [batch] */
    int32_t *gamma;             /* device in/out [batch] */
    int32_t *seq_len;           /* device in/out [batch], or NULL */
    int32_t *cu_q;              /* device out [batch+1] */
    int32_t *cu_d;              /* device out [batch+1] */
    int32_t batch;
    sv_gamma_config config;
    int32_t *trajectory;        /* device out or NULL: gamma_next written to trajectory[step*batch + b] */
    int32_t *accepted_log;      /* device out or NULL: A written to accepted_log[step*batch + b] */
    int32_t step;
    uint32_t *device_status;    /* device, one word or NULL */
    const int32_t *n_drafted;   /* device [batch] or NULL: drafts actually produced this step when
                                   drafting stopped early (spec_draft_stop); gamma[b] stays the
                                   length the controller issued and is what A is compared with,
                                   n_drafted[b]+1 is the number of positions the cache gained */
} sv_gamma_params;

sv_status gamma_tune_update(const sv_gamma_params *p, void *stream);
/* gamma = gamma0 and gamma_bar = gamma0 for every sequence, cu_q / cu_d built; n_accepted,
 * seq_len, trajectory are not touched. */
sv_status gamma_tune_init(const sv_gamma_params *p, int32_t gamma0, void *stream);

/* ---------------------------------------------------------------- GammaTune+ early stop */
/*
 * Paper Section 4.2 (GammaTune+): drafting stops when the draft model's top
 * probability falls below a threshold tau.  For sequence b and draft position
 * i < gamma[b] the confidence is c_i = max_k softmax(d_i / T)_k (one streaming
 * pass over the draft row: running max and sum).  The paper does not say
 * whether the low-confidence token itself is kept; here it is, and nothing is
 * drafted after it:
 *     n_drafted[b] = min(gamma[b], 1 + first i with c_i < tau)   (gamma[b] if none).
 * T == 0 (greedy draft): c_i = 1, drafting never stops early.
 * The verify step then runs with n_drafted as its gamma array (attention,
 * accept) and gamma_tune_update takes both (see sv_gamma_params.n_drafted).
 * Confidences are float32 exponentials summed in float64; c_i and the
 * comparison with tau are evaluated in float64.
 */
typedef struct sv_draft_stop_params {
    const float *draft_logits;    /* device fp32 [n_d_rows, row_stride] */
    int64_t row_stride;           /* elements between rows (>= vocab) */
    int32_t vocab;
    float temperature;            /* used when temperature_per_seq is NULL */
    const float *temperature_per_seq; /* device [batch] or NULL */
    float tau;                    /* threshold in [0, 1] */
    const int32_t *gamma;         /* device [batch]: draft lengths issued by the controller */
    const int32_t *cu_d;          /* device [batch+1] */
    int32_t batch;
    int32_t gamma_max;
    int32_t *n_drafted;           /* device out [batch] */
    double *top_prob;             /* device out [n_d_rows] or NULL: c_i of every draft row */
    uint32_t *device_status;      /* device, one word or NULL */
    int32_t logits_bf16;          /* as in sv_accept_params: 1 = draft_logits holds bf16 values */
} sv_draft_stop_params;

size_t spec_draft_stop_workspace_bytes(int32_t batch, int32_t gamma_max, int32_t vocab);

sv_status spec_draft_stop(const sv_draft_stop_params *p, void *workspace_device, size_t workspace_bytes,
                          void *stream);

/* ---------------------------------------------------------------- GammaTune+ drafting step */
/*
 * Paper Section 4.2, the draft side: one drafting step of every sequence that
 * is still drafting.  Row b of draft_logits holds sequence b's draft logits for
 * its next position.  For every b with active[b] != 0 and n_drafted[b] < gamma[b]:
 *     q = softmax(d_b / T);  token ~ q by inverse CDF in vocabulary order with
 *     u_sample[b] (the smallest k with sum_{j<=k} q_j > u * sum_j q_j;
 *     T == 0: token = argmax, lowest index on ties);  c = max_k q_k (T == 0: 1)
 *     draft_tokens[cu_d[b] + n_drafted[b]] = token, top_prob[same] = c,
 *     n_drafted[b] += 1,  active[b] = (c >= tau) && (n_drafted[b] < gamma[b]).
 * The token drawn at a position whose confidence is below tau is kept, as in
 * spec_draft_stop; a loop of these steps from n_drafted = 0 and active = 1 ends
 * with the n_drafted that spec_draft_stop gives for the same rows, and with the
 * tokens where spec_accept_sample reads them.  Sequences that are not active are
 * not read and not written; one with n_drafted[b] >= gamma[b] only has active[b]
 * cleared.  A row whose softmax sum is not finite (NaN or +inf logits) sets
 * SV_DEV_NONFINITE, stores token -1 and clears active[b].
 * Arithmetic: the top probability from float32 exponentials summed in float64
 * (as spec_draft_stop), evaluated and compared with tau in float64; the token
 * from a float64 pass over the row (as the bonus token of spec_accept_sample).
 */
typedef struct sv_draft_step_params {
    const float *draft_logits;    /* device fp32 [batch, row_stride] (bf16 values if logits_bf16) */
    int64_t row_stride;           /* elements between rows (>= vocab) */
    int32_t vocab;
    float temperature;            /* used when temperature_per_seq is NULL */
    const float *temperature_per_seq; /* device [batch] or NULL */
    float tau;                    /* threshold in [0, 1] */
    const float *u_sample;        /* device [batch], in [0,1); may be NULL if every temperature is 0 */
    const int32_t *gamma;         /* device [batch]: draft lengths issued by the controller */
    const int32_t *cu_d;          /* device [batch+1]: first draft row of each sequence */
    int32_t batch;
    int32_t gamma_max;            /* bound on gamma[b] */
    int32_t *n_drafted;           /* device in/out [batch] */
    int32_t *active;              /* device in/out [batch] */
    int32_t *draft_tokens;        /* device out [n_d_rows] */
    double *top_prob;             /* device out [n_d_rows] or NULL */
    uint32_t *device_status;      /* device, one word or NULL */
    int32_t logits_bf16;          /* as in sv_accept_params */
} sv_draft_step_params;

size_t spec_draft_step_workspace_bytes(int32_t batch, int32_t vocab);

/* Four launches on `stream`; nothing is read back.  Errors before any launch: SV_EINVAL (null pointers,
 * sizes <= 0, row_stride < vocab, tau outside [0, 1], u_sample NULL with a positive temperature),
 * SV_EWORKSPACE, SV_EALIGN (workspace not 16-byte aligned). */
sv_status spec_draft_step(const sv_draft_step_params *p, void *workspace_device, size_t workspace_bytes,
                          void *stream);

/* ---------------------------------------------------------------- whole step from host buffers */
/*
 * One verify step whose per-step inputs start in HOST memory: copies q,
 * logits, draft tokens and uniforms to the caller's device staging buffers,
 * runs spec_verify_attn, spec_accept_sample, gamma_tune_update on `stream`,
 * and copies n_accepted, out_tokens, gamma (next) and the attention output
 * back to host buffers.  All asynchronous; the caller synchronises the stream
 * before reading the host outputs.  The KV pool, block table and controller
 * state stay resident on the device (that is what a KV cache is).
 * n_q_rows / n_d_rows are the numbers of rows to copy (host knows the layout
 * it filled).  Device pointers inside attn / accept / gamma are used as the
 * staging destinations.
 */
typedef struct sv_step_host_io {
    const void *q_host;             /* bf16 [n_q_rows, hq, head_dim] */
    const float *target_logits_host;
    const float *draft_logits_host;
    const int32_t *draft_tokens_host;
    const float *u_accept_host;
    const float *u_sample_host;
    int64_t n_q_rows, n_d_rows;
    int32_t *n_accepted_host;       /* out [batch] */
    int32_t *out_tokens_host;       /* out [batch, gamma_max+1] */
    int32_t *gamma_next_host;       /* out [batch] */
    void *o_host;                   /* out bf16 [n_q_rows, hq, head_dim], or NULL */
} sv_step_host_io;

sv_status spec_verify_step_host(const sv_step_host_io *io, const sv_attn_params *attn,
                                void *attn_workspace, size_t attn_workspace_bytes,
                                const sv_accept_params *accept, void *accept_workspace,
                                size_t accept_workspace_bytes, const sv_gamma_params *gamma,
                                void *stream);

/*
 * Self-test of the bounded waits (no counterpart in the paper).  Every wait of
 * the tensor-core kernels has a cycle budget; when it runs out the kernel sets
 * SV_DEV_TIMEOUT and returns instead of hanging.  This call launches one thread
 * block that waits, with a budget of limit_cycles (1 .. 2e9 SM cycles), on a
 * barrier nothing ever arrives at.  Afterwards *device_status has
 * SV_DEV_TIMEOUT set and *device_result is 0 (1 would mean the wait was
 * satisfied); the context stays usable.
 */
sv_status sv_selftest_wait_expiry(uint32_t *device_status, int32_t *device_result, int64_t limit_cycles,
                                  void *stream);

/* Kernel launches issued by the library since it was loaded (for reporting). */
uint64_t sv_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* SPECVERIFY_H */
