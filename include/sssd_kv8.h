/*
 * sssd_kv8.h -- a KV cache held in 8 bits, attention over it, and rotary positions, as kernel-level
 * operations of libsssd_verify.  Same conventions as sssd_verify.h: device pointers are caller-owned,
 * calls enqueue on `stream` and return 0 or a negative SSSD_E*, nothing is allocated, nothing waits
 * (but sssd_kv8_sync), every call may be captured into a graph.
 *
 * One layer of a model that keeps its context in such a cache does, per step of B sequences x n rows
 * (the last accepted token and n-1 drafts, a chain or a tree):
 *   sssd_kv8_append     rotate the new K rows, quantise K and V into the cache, rotate the queries
 *   sssd_kv8_attention  every new row's attention over the cached rows it sees
 * and after acceptance, once for all layers, sssd_kv8_commit_tree.  Where sequences continue one another (several answers
 * to a prompt, many users behind a system prompt), sssd_kv8_fork makes them, sssd_kv8_reserve gives the next rows room of
 * their own, sssd_kv8_attention_shared reads what they share once, and sssd_kv8_compact closes a pool's holes.
 *
 * Stored values.  Positions are kept in blocks of 32, a page each (of one sequence, all kv heads).  A
 * block's K of one kv head, and its V, have one scale each, a power of two: with A the largest finite
 * magnitude among the block's live rows, the smallest power of two s >= 2^-126 with A <= 448 s
 * (SSSD_KV8_E4M3) or A <= 127 s (SSSD_KV8_INT8), and s = 1 for A = 0.  A value x is held as the code
 * nearest to x / s, ties to the even code; it stands for code * s, which bf16 holds exactly.  A live row is one
 * below lens[b] when a step begins, or new in it; rows at or beyond are dead and leave no trace in what
 * is written later.  When a step's new rows change a block's scale, the block's older rows move to the
 * new scale: exactly where it shrinks, and where it grows too for SSSD_KV8_E4M3 but for the smallest
 * values (below 2^-6 of the new scale); SSSD_KV8_INT8 then drops low bits, and none when the scale
 * shrinks and grows back.  So the order in which rows came, and drafts that were rejected, however many,
 * put an integer code less than one step of the largest scale its row was held at off the row's own value
 * (half a step for the largest, a quarter for one half as large, ...).  A value that is no number is held as
 * 0, and an infinite one, or of a magnitude above 2^127, as the largest code of its sign; neither counts
 * for A, both raise the status.
 */
#ifndef SSSD_KV8_H
#define SSSD_KV8_H

#include "sssd_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SSSD_KV8_E4M3 0 /* 8-bit floats: 1 sign, 4 exponent, 3 mantissa bits, largest 448 */
#define SSSD_KV8_INT8 1 /* 8-bit integers -127 .. 127 */

/* head_dim 64 or 128; n_q_heads a multiple of n_kv_heads, at most 64 times as many; n_pages: pages of a layer's pool, 0 for
 * max_batch * ceil(max_seq / 32). */
typedef struct {
    int32_t format; /* SSSD_KV8_E4M3 or SSSD_KV8_INT8 */
    int32_t n_layers, n_q_heads, n_kv_heads, head_dim;
    int32_t max_batch, max_seq, n_pages;
} sssd_kv8_config;

/* Bytes of the cache (all layers) and of the workspace, and the geometry of a block table: int32
 * [max_batch][blocks_per_seq], entries 0 .. n_pages-1.  Host computation only; any out pointer may be NULL. */
int sssd_kv8_sizes(const sssd_kv8_config *cfg, size_t *cache_bytes, size_t *ws_bytes, int32_t *blocks_per_seq,
                   int32_t *n_pages);

/* A cache as the calls take it (host struct, read during the call only). */
typedef struct {
    sssd_kv8_config cfg;
    void *cache;                /* device, 256-byte aligned, at least cache_bytes; any contents           */
    size_t cache_bytes;
    void *workspace;            /* device, 256-byte aligned, at least ws_bytes; zero-filled once by the
                                   caller; calls that share it must be ordered                            */
    size_t ws_bytes;
    const int32_t *block_table; /* device, or NULL: sequence b owns pages b*blocks_per_seq and following;
                                   NULL needs n_pages >= max_batch * blocks_per_seq                       */
    int32_t *status;            /* device int32 [1], zero-filled once by the caller: what sssd_kv8_sync reports */
    uint32_t flags;             /* 0 or SSSD_NO_WAIT, as for sssd_verify_init: the same results, slower     */
} sssd_kv8;

/* Rows of heads in device memory: element (b, j, head, channel) lies `b*batch_stride + j*row_stride +
 * head*head_stride + channel` elements behind `data`.  Strides are any (0 among them, for what is read); where
 * data and strides are multiples of 16 bytes rows are moved 16 bytes at a time. */
typedef struct {
    void *data;
    int32_t type; /* SSSD_F32 or SSSD_BF16 */
    int64_t batch_stride, row_stride, head_stride;
} sssd_rows;

/* ------------------------------------------------------------------------- rotary positions -- */
#define SSSD_ROPE_HALVES 0     /* pairs (i, i + rotary_dims/2), as everywhere else in this library */
#define SSSD_ROPE_NEIGHBOURS 1 /* pairs (2i, 2i + 1)                                              */

#define SSSD_ROPE_PLAIN 0  /* f_i = base^(-2i / rotary_dims) radians per position, i < rotary_dims/2              */
#define SSSD_ROPE_LINEAR 1 /* f_i / factor                                                                        */
#define SSSD_ROPE_BANDS 2  /* by the turns a pair makes in `original` positions, t = original * f_i / 2 pi:
                              f_i (w + (1 - w) / factor), w = (t - low) / (high - low) clamped to 0 .. 1          */
typedef struct {
    int32_t rotary_dims; /* even, 2 .. 1024 */
    float base;          /* > 1 */
    int32_t scaling;     /* SSSD_ROPE_* */
    float factor;        /* LINEAR, BANDS: > 0 */
    float low, high;     /* BANDS: 0 <= low < high */
    int32_t original;    /* BANDS: > 0 */
} sssd_rope_config;

/* The frequencies in turns per position, f_i / 2 pi, as float64 [rotary_dims/2] in HOST memory; the caller
 * keeps a device copy, and may as well fill one by a rule of its own. */
int sssd_rope_frequencies(const sssd_rope_config *cfg, double *turns);

/* Channels at or beyond rotary_dims pass unchanged; the others are rotated by 2 pi * frac(position * turns[i])
 * (the product in 64 bits, so that far positions keep their angle) and multiplied by `magnitude`. */
typedef struct {
    const double *turns; /* device, [rotary_dims/2] */
    int32_t rotary_dims; /* even, 2 .. head_dim, at most 1024 */
    int32_t pairs;       /* SSSD_ROPE_HALVES or SSSD_ROPE_NEIGHBOURS */
    float magnitude;     /* 1, or what a scaling for long contexts asks for */
} sssd_rope;

/* out = x rotated: [B][n][heads][head_dim] each (heads <= 65535, head_dim <= 8192), of one type; out may be x itself (same data and strides), else
 * they must not overlap.  positions: device int32 [B][n]. */
int sssd_op_rope(const sssd_rows *x, const sssd_rows *out, int32_t B, int32_t n, int32_t heads, int32_t head_dim,
                 const int32_t *positions, const sssd_rope *rope, void *stream);

/* --------------------------------------------------------------------------------- the cache -- */
/*
 * Write n rows of each of B sequences, slots first .. first+B-1 of the cache, into `layer`.
 *   k, v     [B][n][n_kv_heads][head_dim], of one type
 *   lens     device int32 [B]; live rows of every sequence before the call; row j goes to lens[b] + j.  Not changed.
 *   counts   device int32 [B] or NULL; rows of sequence b, 0 .. n: rows from counts[b] on are not read (NULL: n)
 *   rope     NULL: rows are stored as they are.  Else k is rotated first, row j at position lens[b] + depth(j)
 *   parents  NULL: chains, depth(j) = j.  Else device int32 [B][n] as in sssd_verify_step_tree (n <= 32)
 *   q, q_out both NULL, or with rope: [B][n][n_q_heads][head_dim], q_out = q rotated likewise (rows below counts[b]
 *            only), of one type, which need not be k's; q_out may be q itself
 * n is any (a prompt comes in one call; above max_seq only with counts).  A sequence with lens[b] < 0, lens[b] + counts[b] > max_seq, counts[b] outside
 * 0..n or a page outside the pool for a block it writes is rejected: nothing of it is stored, and the status raised (its
 * queries are rotated all the same in the last case, and left alone in the others); a parent outside [0, j) is treated as j-1 and raises the status.  Sequences of one call must not share a page they write.
 */
int sssd_kv8_append(const sssd_kv8 *kv, int32_t layer, int32_t first, int32_t B, int32_t n, const sssd_rows *k,
                    const sssd_rows *v, const int32_t *lens, const int32_t *counts, const sssd_rope *rope,
                    const int32_t *parents, const sssd_rows *q, const sssd_rows *q_out, void *stream);

/*
 * Read rows start[b] .. start[b]+counts[b]-1 of slots first .. first+B-1 back into k, v ([B][n][n_kv_heads][head_dim],
 * of one type): the values that the codes stand for.  start, counts: device int32 [B] or NULL (0 and n); rows from
 * counts[b] on are left as they were.  Sequences are rejected as by sssd_kv8_append, and then left as they were too.
 */
int sssd_kv8_read(const sssd_kv8 *kv, int32_t layer, int32_t first, int32_t B, int32_t n, const int32_t *start,
                  const int32_t *counts, const sssd_rows *k, const sssd_rows *v, void *stream);

/*
 * Attention of n <= 32 new rows of each of the sequences in slots 0 .. B-1, which are in the cache (sssd_kv8_append):
 * softmax(q . k / sqrt(head_dim)) over what a row sees, times v.
 *   q, out   [B][n][n_q_heads][head_dim], of one type; q already rotated.  They must not overlap.  Scores, softmax and sums are
 *            held to 32-bit accuracy for SSSD_F32, q and probabilities to 22 bits; for SSSD_BF16 probabilities are rounded to 11
 *            bits.  For both, a channel of q is held to 2^-39 of its row's largest at the finest, a probability to 2^-32 of its
 *            row's largest.  Any finite q will do whose scores are in float32's range; a row of q that is no finite number spoils
 *            its own results alone.  The scales of V's blocks may lie anywhere; values of blocks 2^80 and more below the largest
 *            scale that any row of the call sees may count as 0
 *   lens, counts, parents  as in sssd_kv8_append: row j sees the old rows (below lens[b]) and, of the new ones, itself
 *            and its ancestors
 *   window   0: all of them.  Else those fewer than `window` positions behind the row's own (a new row's position is
 *            lens[b] + depth), and the first `sinks` positions
 * Rows from counts[b] on are left as they were.  A rejected sequence's rows are set to 0 (for a page outside the pool:
 * are meaningless), and the status raised.  A sequence's results are the same bits whatever the others hold.
 */
int sssd_kv8_attention(const sssd_kv8 *kv, int32_t layer, int32_t B, int32_t n, const sssd_rows *q,
                       const sssd_rows *out, const int32_t *lens, const int32_t *counts, const int32_t *parents,
                       int32_t window, int32_t sinks, void *stream);

/*
 * Commit a step of n = k+1 <= 32 rows, all layers at once, as sssd_kv_commit_tree does: the rows of the accepted nodes
 * accepted_path[b][1..a], a = accepted_len[b], move to lens[b]+1 .. lens[b]+a; then lens[b] += a + 1 (device int32 [B],
 * in-out).  accepted_path [B][n], or NULL for chains: only lens advances.  A path that is not strictly increasing within
 * 1..n-1 or whose last row lies at or beyond max_seq, a outside 0..n-1, lens[b] < 0, or a page outside the pool for a block of
 * the path leaves that sequence untouched and raises the status.
 */
int sssd_kv8_commit_tree(const sssd_kv8 *kv, int32_t B, int32_t n, int32_t *lens, const int32_t *accepted_len,
                         const int32_t *accepted_path, void *stream);

/* ----------------------------------------------------------------- prefixes that sequences share -- */
/*
 * sssd_kv8_attention for a batch whose sequences share prefixes: the same rows and results (but for the order of sums), without a window,
 * each prefix read once for all rows of its group, or by each sequence where that is the faster way for sequences of up to max_seq positions.  Sequences of a group lie next to each other: group g is the slots starts[g] ..
 * starts[g+1]-1 below B, and the first shared[g] positions of all of them are the same rows.  They are read, in whole blocks
 * (shared[g] / 32 of them), through the block table's row of the group's first sequence, whose other state plays no part.
 *   groups      0 .. B; sequences in no group, groups of one and empty groups share nothing
 *   starts      device int32 [groups + 1], ascending from >= 0 to <= B
 *   shared      device int32 [groups], 0 .. max_seq
 *   workspace   device, 256-byte aligned, any contents, at least what sssd_kv8_shared_sizes asks for this B and n (a larger B or n asks
 *               for more); calls that share it must be ordered, as those of one kv, whose own workspace is used too
 * starts or shared out of range raise the status, and nothing is shared in that call.  A sequence shorter than its group's shared blocks is rejected
 * like the others (sssd_kv8_attention).  Pages outside the pool among a prefix's blocks raise the status and spoil the rows of the group.
 */
int sssd_kv8_shared_sizes(const sssd_kv8_config *cfg, int32_t B, int32_t n, size_t *ws_bytes);
int sssd_kv8_attention_shared(const sssd_kv8 *kv, int32_t layer, int32_t B, int32_t n, const sssd_rows *q, const sssd_rows *out,
                              const int32_t *lens, const int32_t *counts, const int32_t *parents, int32_t groups,
                              const int32_t *starts, const int32_t *shared, void *workspace, size_t ws_bytes, void *stream);

/* ---------------------------------------------------------------------------------- pages of the pool -- */
/*
 * Who has which pages.  refs[p] counts the entries of the table that name page p, and whatever else the caller holds it for; pages of count 0
 * are free.  A new pool has a table of -1 and counts of 0.  Entries behind a sequence's pages are -1.  The three calls change table, counts
 * and pages on the device, in all layers, and each either does all of what it says or, where it cannot, nothing but raise the status.  Pages
 * are taken from the lowest free ones, in the order of slots and blocks.
 */
typedef struct {
    int32_t *table;   /* device int32 [max_batch][blocks_per_seq]: the cache's block_table, which has to point at it */
    int32_t *refs;    /* device int32 [n_pages] */
    void *workspace;  /* device, 256-byte aligned, at least ws_bytes; zero-filled once by the caller; calls that share it must be ordered */
    size_t ws_bytes;
} sssd_kv8_pages;

/* The calls take pools of up to 2^30 pages. */
int sssd_kv8_pages_sizes(const sssd_kv8_config *cfg, size_t *ws_bytes);

/*
 * All slots 0 .. max_batch-1 at once: slot b becomes a continuation of what slot origins[b] was before the call (b: stays itself; -1:
 * empty, its length 0), with lens[b] = lens[origins[b]].  Its whole blocks are shared with all who continue the same slot; of its last block, where
 * that is partly filled, one has the page (the origin itself if it stays, else the lowest slot) and the others get copies.  Pages behind the new length,
 * and pages that nobody names any more, are free afterwards.
 *   origins, lens   device int32 [max_batch]; lens in-out
 * Nothing is done where an origin is outside -1 .. max_batch-1, the length of one outside 0 .. max_seq, an entry of the table outside
 * -1 .. n_pages-1 or of a page that counts 0, a live block without a page, or where there are too few free pages.  max_batch <= 65535.
 */
int sssd_kv8_fork(const sssd_kv8 *kv, const sssd_kv8_pages *pages, const int32_t *origins, int32_t *lens, void *stream);

/*
 * Room for rows lens[b] .. lens[b]+counts[b]-1 (counts NULL: n) of the sequences in slots first .. first+B-1: every block of these rows gets a page that no
 * other entry names.  Missing pages are taken; a page that others share is replaced, by a copy where live rows (below lens[b]) are in it.  Where all
 * who share a page ask for it in this call, the first of them (by slot and block) keeps it.  lens is not changed.
 * Nothing is done where lens[b], counts[b] or lens[b] + counts[b] is out of range as for sssd_kv8_append, an entry that is looked at is outside
 * -1 .. n_pages-1 or of a page that counts 0, or where there are too few free pages.
 */
int sssd_kv8_reserve(const sssd_kv8 *kv, const sssd_kv8_pages *pages, int32_t first, int32_t B, int32_t n, const int32_t *lens,
                     const int32_t *counts, void *stream);

/*
 * A pool without holes.  With U pages in use (counts above 0), to NULL: the i-th of those in use at or behind U moves into the i-th free one in front
 * of it; the others stay.  Else the i-th page in use goes to page i of another cache (the same format, layers, kv heads, head_dim, max_batch and
 * blocks per sequence, any n_pages >= U), whose table and counts are written whole; kv and its pages stay as they were.
 *   moved    device int32 [n_pages] or NULL: where each page is now, -1 for free ones
 *   in_use   device int32 [1] or NULL: U, written also where nothing else is done
 * Nothing is done where the table has an entry outside -1 .. n_pages-1 or of a page that counts 0, or U is above the other's n_pages.  The status is kv's.
 */
int sssd_kv8_compact(const sssd_kv8 *kv, const sssd_kv8_pages *pages, const sssd_kv8 *to, const sssd_kv8_pages *to_pages, int32_t *moved,
                     int32_t *in_use, void *stream);

/* Wait for `stream`, then clear the status and return SSSD_ENOSPACE if a call raised it for a sequence, page, count,
 * path or parent out of range, else SSSD_EINVAL if it was raised for rows that are no finite numbers, SSSD_EHIP if the
 * runtime reported an error, else SSSD_OK. */
int sssd_kv8_sync(const sssd_kv8 *kv, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SSSD_KV8_H */
