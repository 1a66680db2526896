/*
 * spd_q8.h - 8-bit serving operators of the SPD library: a paged KV cache that is quantised (to 8 or 4 bits) as it
 * is written, attention of chunks of new tokens over its pages, plans of steps on the host or the device, rows
 * brought to 8-bit integers, and the product of such rows with 8-bit weights.
 *
 * Together they make up a rank's share of a decoder block (spd.h) with 8-bit projections:
 *
 *   a    = q8(RMSNorm(X; g1))                       spd_q8_norm
 *   qkv  = a Wqkv                                   spd_q8_matmul
 *   q'   = rope(q); pages <- quantised rope(k), v   spd_pages_write
 *   A    = attention(q', pages)                     spd_pages_attention
 *   Y    = q8(A) Wo                                 spd_q8_rows, spd_q8_matmul
 *   m    = q8(RMSNorm(X + Y; g2))                   spd_q8_norm with a summand (the fold of an SPD block, Sec. 4.1.1)
 *   u    = q8(silu(m Wg) * (m Wu))                  spd_q8_matmul, spd_q8_swiglu
 *   slot = Y + u Wd                                 spd_q8_matmul with a summand
 *
 * The conventions are those of spd.h: error codes, host checks before anything is enqueued, caller-owned
 * buffers, nothing allocated, freed or waited for by a device call, work enqueued on `stream` alone.
 * A call that has nothing to do (no tokens, no rows) needs no addresses but its plan's.
 * The device calls may be captured into a HIP graph, which is then bound to what its calls were given on the host: the launches of a plan made
 * there are those of its lengths, another such plan takes another capture; a graph with plans made on the device holds for every step
 * within their limits.  Results are bit-reproducible.
 */
#ifndef SPD_Q8_H
#define SPD_Q8_H

#include "spd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of these operators, besides SPD_F32 and SPD_BF16. */
#define SPD_F16 2  /* IEEE binary16 */
#define SPD_E4M3 3 /* 8 bits, 4 of exponent, 3 of fraction, largest finite value 448; a page's keys and values only */
#define SPD_E2M1 4 /* 4 bits, 2 of exponent, 1 of fraction: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; a page's keys and values only */

/* ---------------------------------------------------------------- pool of pages (host only)
 *
 * The pool is one device buffer of n_pages pages.  A page holds page_size consecutive positions of one
 * sequence for every KV head of the rank; which page holds which positions is the caller's to say, call
 * by call, in a page table.  Pages may be shared between sequences for reading (a common prefix).
 *
 * What a page holds of a position and head is the key's and the value's codes, and a scale (fp32) for each:
 * the value read back is code * scale.  With cache_dtype SPD_E4M3 the scale is a / 448, a the row's largest
 * magnitude (2^-90 if that is larger), and the code is the e4m3 value nearest to x * (448 / a).  With a
 * 16-bit cache_dtype the code is x rounded to that type and the scale is 1.  A row that holds a value that is
 * not finite (or becomes infinite in a 16-bit type) is stored as codes 0 with scale NaN: it reads back as
 * NaN and makes NaN of the output of every query that sees it, and of no other.
 *
 * With cache_dtype SPD_E2M1 every 32 consecutive features of a row have a scale of their own, a power of two 2^e: e is the least with
 * a <= 7 * 2^e, a the largest magnitude among them, -100 to 125 with dtype SPD_BF16 and -23 to 13 with SPD_F16 (the least for a = 0), so that code *
 * scale is a value of dtype.  The code is the e2m1 value nearest to x * 2^-e, ties to the even one, 6 for what is beyond (in SPD_F16
 * what lies above 57344 becomes 49152).  Keys are rotated in 64 bits for it.  A row that holds a value that is not finite, or
 * becomes infinite in dtype, has codes 0 and scales NaN.  A position takes 136 bytes of a head of 128 where e4m3 takes 264 and 16 bits 520; code *
 * scale is at most a / 5 off (e4m3: a / 28), of normally distributed rows 11 % in the root mean square (e4m3: 2.6 %).
 *
 * Layout, per page and head: keys [page_size/16 blocks][head_dim/64 (e4m3) | /32 (16-bit)][4][16 positions][16 bytes
 * of consecutive features]; values [blocks][same][4 groups][16 features][features 16 apart: 4 | 2][4 consecutive positions];
 * page_size key scales; page_size value scales.  With SPD_E2M1: keys [blocks][4][16 positions][head_dim/8 bytes of consecutive features, two to a byte,
 * the first in its low half]; values [blocks][4 groups][16 features][head_dim/32 pairs of features 16 apart][4 consecutive positions], a byte for each pair;
 * key scales [page_size][head_dim/32], bytes e + 127 (255: NaN); value scales the same.
 * The pool must be zero-filled once before its first use. */
typedef struct spd_pages_config {
    int32_t n_q_heads;   /* query heads of the rank */
    int32_t n_kv_heads;  /* KV heads of the rank; divides n_q_heads, at most 16 query heads per KV head */
    int32_t head_dim;    /* 64 or 128 */
    int32_t page_size;   /* positions per page: 16, 32, 64, 128 or 256 */
    int32_t n_pages;
    int32_t dtype;       /* SPD_BF16 | SPD_F16: queries and attention output */
    int32_t cache_dtype; /* SPD_E4M3, SPD_E2M1, or the same as dtype */
    int32_t max_ctx;     /* positions a sequence may reach (length of the rotary table) */
    float rope_base;     /* 10000 for LLaMA2 */
} spd_pages_config;

typedef struct spd_pages_sizes {
    size_t pool_bytes;
    size_t rope_bytes;   /* rotary table: fp32 [max_ctx][head_dim / 2][cos, sin] */
} spd_pages_sizes;

typedef struct spd_pages spd_pages;

/* Checks the configuration; touches no device.  The handle is immutable and may be shared between threads.
 * SPD_EINVAL: NULL, non-positive sizes, n_q_heads not a multiple of n_kv_heads, unknown types, rope_base not positive.
 * SPD_EUNSUPPORTED: head_dim, page_size, cache_dtype or the number of query heads per KV head outside the above. */
int spd_pages_create(const spd_pages_config *cfg, spd_pages **out);
void spd_pages_destroy(spd_pages *pages);
int spd_pages_get_sizes(const spd_pages *pages, spd_pages_sizes *out);
/* Writes the rotary table (rope_bytes, host): angle position * rope_base^(-2j/d), computed in double. */
int spd_pages_rope_table(const spd_pages *pages, float *host);

/* ---------------------------------------------------------------- plan of a step (host only)
 *
 * A plan says what a step's calls work on: which sequences, where their new tokens sit, in which pages, and how
 * the work is cut into workgroups.  Every layer of a model uses the same plan, and every step needs one of its own: it is as long
 * as its page table and its pieces of work, and takes the host 5 to 35 us for one to some hundred pieces (a call that asks for the size alone as long).
 *   batch       sequences; 0 is a plan of nothing
 *   positions   host, [batch]: position of each sequence's first new token = positions already in its pages
 *   q_lens      host, [batch]: new tokens of each sequence, 0 or more.  The tokens of a step are rows
 *               0 .. sum(q_lens) - 1 of the calls' matrices, sequence after sequence.
 *   page_table  host, [batch][ld_table]: page_table[b][i] is the page of positions [i * page_size, (i + 1) * page_size) of
 *               sequence b; the first ceil((positions[b] + q_lens[b]) / page_size) entries are read
 *   window      0: a token sees every position up to its own.  w > 0: only the w last of them (its own among them) ...
 *   sinks       ... and the first `sinks` positions of the sequence
 *   plan_host   receives the plan, or NULL: only *bytes is written
 *   capacity    bytes of plan_host
 *   bytes       receives the size of the plan
 * The caller copies the plan to the device; calls take both copies.
 * SPD_EINVAL: NULL, negative sizes, positions[b] + q_lens[b] > max_ctx, ld_table too small, a page outside the pool, a
 * page that would be written by two sequences or in two places or is written while another sequence reads it,
 * sinks without a window, capacity too small, more than 2^24 tokens or 65535 sequences. */
int spd_pages_plan(const spd_pages *pages, int32_t batch, const int32_t *positions, const int32_t *q_lens, const int32_t *page_table,
                   int32_t ld_table, int32_t window, int32_t sinks, void *plan_host, size_t capacity, size_t *bytes);

typedef struct spd_pages_plan_info {
    int32_t batch;
    int32_t tokens;          /* sum of q_lens: rows of qkv, queries and outputs */
    int64_t held;            /* sum of positions + q_lens: rows that spd_pages_read() writes */
    size_t workspace_bytes;  /* scratch of spd_pages_attention(), may be 0 */
} spd_pages_plan_info;
int spd_pages_plan_get_info(const spd_pages *pages, const void *plan_host, spd_pages_plan_info *out);

/* ---------------------------------------------------------------- plan of a step, made on the device
 *
 * Where lengths are on the device (a step's tokens were drawn there, requests end there), so can the plan be made: spd_pages_reserve() says once, on the
 * host, how large steps may get, and spd_pages_build() turns the requests' lengths into a step's plan, as often as there are steps, without the host. It takes pages
 * from a free list for positions that have none yet, writes them into the page table, takes back those of requests that have ended, and says
 * which row of the step's matrices is which position and slot.  spd_pages_write() and spd_pages_attention() take the plan as they take one
 * that was made on the host, and give the same bits.  A captured graph holds for every step within the limits. */
typedef struct spd_pages_limits {
    int32_t batch;    /* requests: entries of the arrays below; at most 4096 */
    int32_t tokens;   /* rows of the step's matrices */
    int32_t q_len;    /* new tokens of a request.  With up to 16 / (query heads per KV head) steps take one launch of attention, else two */
    int32_t entries;  /* pages of a request: columns of the page table */
    int32_t window, sinks;      /* as for spd_pages_plan() */
} spd_pages_limits;

/* Host only.  plan_host: receives what the calls take for plan_host, or NULL; capacity: its bytes; bytes: receives its size; device_bytes: receives the size of
 * plan_dev, which spd_pages_build() fills.  tokens of the plan's info are the limit's, its workspace_bytes serve every step within the limits, held is 0.
 * SPD_EINVAL: NULL, sizes that are not positive, q_len above tokens, sinks without a window, capacity too small.
 * SPD_EUNSUPPORTED: more than 4096 requests, 2^24 tokens, 2^28 entries in all, or 8192 pieces of 128 rows (tokens * query heads per KV head / 128, and one
 * for every request that can have more than 16 rows). */
int spd_pages_reserve(const spd_pages *pages, const spd_pages_limits *limits, void *plan_host, size_t capacity, size_t *bytes, size_t *device_bytes);

#define SPD_STEP_RELEASE (-1)  /* q_lens[b]: the request has ended, its pages come back */
#define SPD_STEP_LENGTHS (-1)  /* served[b]: lengths out of range, or more rows than there are */
#define SPD_STEP_PAGE (-2)     /* served[b]: a page of the request, in the table or from the free list, is not of the pool */
#define SPD_STEP_NO_PAGES (-3) /* served[b]: not enough free pages */

/* Device arrays, int32 but for row_slot. */
typedef struct spd_pages_step {
    const int32_t *positions;  /* [batch] positions that are in a request's pages already */
    const int32_t *q_lens;     /* [batch] its new tokens: 1 .. q_len of the limits, 0 (no part in the step), or SPD_STEP_RELEASE */
    int32_t *page_table;       /* [batch][ld_table] pages of the request's positions; entries for positions that are new and in no page yet are written */
    int64_t ld_table;          /* at least the limits' entries */
    int32_t *free_pages;       /* [n_pages] a stack of free pages: the first *n_free are free.  NULL, with n_free and n_free_out: the table has every page */
    const int32_t *n_free;
    int32_t *n_free_out;       /* free pages after the step; may be n_free */
    int32_t *positions_out;    /* [batch] positions + q_lens for requests that are served, 0 for those that have ended; may be positions, or NULL, as may the others */
    int32_t *served;           /* [batch] new tokens of the request, or why it has no part in the step */
    int32_t *first_row;        /* [batch + 1] where its rows begin; last, rows in use */
    int32_t *row_seq;          /* [tokens] of each row: its request, */
    int32_t *row_pos;          /* [tokens] its position, */
    int64_t *row_slot;         /* [tokens] its place in the pool, page * page_size + position % page_size.  -1 for rows that are no request's, or of one not served */
} spd_pages_step;

/* Device call.  Rows go to requests in order, max(q_len, 0) to each, whether it is served or not (within the limit).  Pages that come back are pushed in the
 * requests' order, each request's in the order of its positions; then pages are popped in the same order, for requests that need more than
 * are left and for all that need any after them none (SPD_STEP_NO_PAGES).  A request that is not served keeps its positions, its rows of outputs stay as they were.
 * SPD_STEP_PAGE tells of a table or a free list that is not sound: new pages have been written into the request's row all the same.  Where the page that is none is one that
 * it had, later steps hand it no others as long as a page lies in the first place behind ceil(positions / page_size); where it came from the free list (of
 * which a request that ended with such an entry makes it part) it is gone with the step, and so are the new pages beside it.  Who mends the table makes the free list anew of the pages that
 * are in nobody's first ceil(positions / page_size) entries.  Two requests may share pages for reading; that the page of a new token is one request's alone, and a page at most once in the
 * free list and the tables of those that have ended, is the caller's to see to: it is not checked.
 * plan_dev: device_bytes, 16-byte aligned; calls on other streams that still read the plan of the step before have to be over.  Arrays may share no memory but
 * for what is said above.
 * SPD_EINVAL: NULL, a plan made on the host, alignment, ld_table, shared memory. */
int spd_pages_build(const spd_pages *pages, const void *plan_host, void *plan_dev, const spd_pages_step *step, void *stream);

/* ---------------------------------------------------------------- device calls on pages
 * plan_host / plan_dev: the plan and its copy on the device (16-byte aligned).  pool: pool_bytes, 256-byte aligned. */

/* Rotates queries and keys and puts keys and values away, quantised.
 *   qkv     [tokens][ld]: n_q_heads query heads, n_kv_heads keys, n_kv_heads values of head_dim each; in_dtype SPD_F32, or the
 *           pool's dtype; 16-byte aligned, ld * element size a multiple of 16
 *   rope    device copy of the rotary table, 16-byte aligned, or NULL: keys go in as they are, and q_out has to be NULL
 *   q_out   [tokens][ld_q] in the pool's dtype, receives the rotated queries, 16-byte aligned rows; may be qkv itself (with its
 *           ld) when in_dtype is the pool's dtype, else it may share no memory with qkv (columns beside it in rows of the same stride in
 *           bytes do not); NULL: not wanted
 * Must be enqueued ahead of the step's spd_pages_attention(). */
int spd_pages_write(const spd_pages *pages, const void *plan_host, const void *plan_dev, int32_t in_dtype, const void *qkv,
                    int64_t ld, const float *rope, void *pool, void *q_out, int64_t ld_q, void *stream);

/* Reads every position of every sequence back: k_out, v_out [held][n_kv_heads][head_dim], sequence after sequence, out_dtype
 * SPD_F32 or the pool's dtype, code * scale rounded once; 16-byte aligned.  SPD_EUNSUPPORTED: a plan made on the device, whose lengths the host does not know. */
int spd_pages_read(const spd_pages *pages, const void *plan_host, const void *plan_dev, const void *pool, int32_t out_dtype,
                   void *k_out, void *v_out, void *stream);

/* out[token] = softmax over the visible positions of (q . k / sqrt(head_dim)) v, query head j on KV head
 * j / (n_q_heads / n_kv_heads).
 *   q, out     [tokens][ld_q], [tokens][ld_out] in the pool's dtype, 16-byte aligned, strides multiples of 8.  out may share no memory
 *              with q (other columns of rows of the same stride do not: keys and values that are put away leave theirs).
 *   workspace  workspace_bytes of the plan, 256-byte aligned; may be NULL when that is 0.  One per stream, of use to any plan that
 *              it is large enough for, zero-filled once before its first use (calls leave its counters at zero).
 * Sums, maxima and outputs are kept in fp32; probabilities (times the value's scale) are rounded to the pool's dtype
 * for the second product, in fp16 beside e4m3 relative to the largest of these products. */
int spd_pages_attention(const spd_pages *pages, const void *plan_host, const void *plan_dev, const void *q, int64_t ld_q,
                        const void *pool, void *out, int64_t ld_out, void *workspace, void *stream);

/* ---------------------------------------------------------------- rows to 8-bit integers (device calls)
 * Each row of n values v gets scale = a / 127, a its largest magnitude (2^-90 if that is larger), and codes
 * rint(v * (127 / a)), so that code * scale is the value to half a step.  A row with a value that is not finite gets
 * scale NaN.  Everything is computed in fp32.
 *   dtype    SPD_F32 | SPD_BF16 | SPD_F16, of the input rows
 *   ld*      row strides in elements; rows need no alignment beyond their elements'
 *   codes    int8 [rows][ld_codes]; they share no memory with the rows, nor does a sum that is none of them (other columns of rows
 *            of the same stride in bytes do not)
 *   scales   fp32 [rows]
 * rows (at most 2^23) = 0 or n = 0: nothing is done. */

/* v = s / sqrt(mean(s^2) + eps) * gain with s = x + add.  s * gain has to be finite in fp32, the sum of squares does not: a row of any finite size
 * has its norm (without an eps, down to the least normal number).
 *   add   [rows][ld_add] or NULL (s = x);   sum   receives s in `dtype` or NULL, may be x or add (same stride) */
int spd_q8_norm(int32_t dtype, int32_t rows, int32_t n, const void *x, int64_t ld_x, const void *add, int64_t ld_add, const float *gain,
                float eps, void *sum, int64_t ld_sum, int8_t *codes, int64_t ld_codes, float *scales, void *stream);
/* v = x */
int spd_q8_rows(int32_t dtype, int32_t rows, int32_t n, const void *x, int64_t ld_x, int8_t *codes, int64_t ld_codes, float *scales,
                void *stream);
/* v = silu(gate) * up, a row of x holding n gates and then n ups */
int spd_q8_swiglu(int32_t dtype, int32_t rows, int32_t n, const void *x, int64_t ld_x, int8_t *codes, int64_t ld_codes, float *scales,
                  void *stream);

/* ---------------------------------------------------------------- product of 8-bit integers
 * out[m][j] = (sum_i codes[m][i] * w[i][j]) * scales[m] * w_scale[j] (+ add[m][j]).  The sums are exact (32-bit integers: K at
 * most 131071); they are scaled in fp32 and rounded once.
 *
 * Weights are quantised and laid out once, on the host: */
#define SPD_Q8_MAX_K 131071
/* bytes of the packed weights of a K x N matrix, 0 for sizes out of range */
size_t spd_q8_weight_bytes(int32_t K, int32_t N);
/* w: host fp32 [K][ld], y = x W; every column gets scale = largest magnitude / 127 and codes rint(w / scale).
 * SPD_EINVAL: NULL, sizes out of range, ld < N, a weight that is not finite. */
int spd_q8_pack(int32_t K, int32_t N, const float *w, int64_t ld, void *packed_host);
/* the same from codes and scales: int8 [K][ld], fp32 [N] */
int spd_q8_pack_codes(int32_t K, int32_t N, const int8_t *w, int64_t ld, const float *w_scale, void *packed_host);
/* inverse of spd_q8_pack_codes() */
int spd_q8_unpack(int32_t K, int32_t N, const void *packed_host, int8_t *w, int64_t ld, float *w_scale);
/* scratch of a product of at most `rows` rows on one stream, may be 0 (and is for every size: none of the kernels needs any) */
size_t spd_q8_matmul_workspace(int32_t rows, int32_t K, int32_t N);
/* Device call.
 *   rows       at most 2^28, rows * N at most 2^38
 *   codes      int8 [rows][ld_codes], 16-byte aligned, ld_codes a multiple of 16 and at least K rounded up to that (bytes past K
 *              may hold anything)
 *   packed     device copy of the packed weights, 256-byte aligned
 *   out_dtype  SPD_F32 | SPD_BF16 | SPD_F16, of add ([rows][ld_add], or NULL) and out ([rows][ld_out]); out may be add (same
 *              stride), and shares no memory with it or with the codes otherwise
 *   workspace  spd_q8_matmul_workspace(rows, K, N) bytes, 256-byte aligned; may be NULL when that is 0 */
int spd_q8_matmul(int32_t rows, int32_t K, int32_t N, const int8_t *codes, int64_t ld_codes, const float *scales, const void *packed,
                  int32_t out_dtype, const void *add, int64_t ld_add, void *out, int64_t ld_out, void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPD_Q8_H */
