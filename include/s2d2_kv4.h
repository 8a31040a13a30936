/*
 * s2d2_kv4.h - a prefix key / value cache held in 4 bits, and the operators on it (MI355X, gfx950).
 *
 *   s2d2_kv4_append     quantises rows of K and V and appends them to the cache
 *   s2d2_kv4_read       entries of the cache back as bf16 or fp32
 *   s2d2_kv4_attention  attention of a batch of ragged windows over the cached entries and the window itself
 *   s2d2_kv4_weigh      adds the attention weight that the windows give every cached entry to its `mass`
 *   s2d2_kv4_evict      cuts every list of entries down to a budget, by that mass
 *   s2d2_set_kv4        the forwards and appends of a context (s2d2.h) run on such a cache
 *
 * The conventions of s2d2.h hold: caller-owned device memory, host-side checks, work enqueued on a stream without
 * synchronising, no memset / memcpy nodes, no float atomics (same inputs, same bits), 0 or a negative S2D2_E* code with the
 * reason in s2d2_last_error().  The calls without a context take the stream (a hipStream_t, NULL: the default stream);
 * its device must be current and hold the memory.
 *
 * Format.  The head_dim values of an entry (one token, one KV head, K or V) are cut into groups of 32.  With a the
 * largest |x| of a group, its exponent e is the smallest whole number with 6 * 2^e >= a, cut to [-23, 13]; its scale byte is
 * e + 127.  Every value becomes a 4-bit code: bit 3 the sign, bits 0-2 the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to
 * |x| / 2^e, ties to the even code, larger values to 6 (|x| up to 49152 stays in range).  The even dimension lies in the low
 * half of a byte.  A group that holds a NaN or an infinity gets the scale byte 255 and reads as NaN.  The value of a code is
 * exact in bf16 and in half.  (This is the microscaling format of 4-bit E2M1 elements with E8M0 scales, with a range of scales cut to what
 * half holds.)  4.25 bits a value.
 *
 * Entries.  Sequence n holds entries[n] entries; entry i lies in page page_table[n, i / page_size], slot i % page_size, of
 * every layer and KV head.  Keys are stored after their rotation, so attention does not depend on the order of the
 * entries, and an entry need not lie at its position: seq_len[n] counts the tokens that were appended (the position of the next one),
 * entries[n] those that are still held.  They differ once entries were evicted.
 * A page that s2d2_kv4_append, s2d2_kv4_weigh or s2d2_kv4_evict writes may be in no other sequence's table.
 * entries outside [0, capacity] are read as the nearest end; a page number outside [0, n_pages) is read as the nearest page and
 * never written.
 */
#ifndef S2D2_KV4_H
#define S2D2_KV4_H

#include "s2d2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  void* k_codes;             /* device [n_layers, n_pages, n_kv_heads, page_size, head_dim / 2] bytes, 16-byte aligned, as v_codes */
  void* v_codes;
  void* k_scales;            /* device [n_layers, n_pages, n_kv_heads, page_size, head_dim / 32] bytes, 8-byte aligned, as v_scales */
  void* v_scales;
  float* mass;               /* device [n_layers, n_pages, n_kv_heads, page_size]: attention weight gathered, or NULL */
  int32_t* position;         /* device, the same shape: position of the token, or NULL */
  const int32_t* page_table; /* device [N, max_pages_per_seq] */
  int32_t* entries;          /* device [N] */
  int32_t* seq_len;          /* device [N] */
  int32_t* status;           /* device [N] or NULL: set to S2D2_ENOSPC by an append without room, else left unchanged */
  int32_t n_layers, n_pages, page_size, max_pages_per_seq;  /* max_pages_per_seq * page_size < 2^30 */
  int32_t n_kv_heads, head_dim;                             /* head_dim 32, 64, 128 or 256 */
} s2d2_kv4_view;

/* Windows of N sequences: the rows of sequence n are row0[n] .. row0[n] + n_rows[n] - 1 of q, k, v, out, lse.  n_rows outside [0, T]
 * is read as the nearest end; a sequence whose rows leave [0, rows) is skipped.  Rows of no sequence are not touched.
 *   q       [rows, n_q_heads, head_dim] in `dtype`, q_stride elements from row to row; head h reads KV head h / (n_q_heads / n_kv_heads)
 *   k, v    [rows, n_kv_heads, head_dim] in `dtype`, kv_stride elements from row to row: the window's own keys (after
 *           rotation) and values; both NULL: the rows see the cached entries only
 *   lo, hi  [rows] or both NULL: row r sees the rows [lo[r], hi[r]) of its sequence's window, and itself; NULL: the rows up to itself
 *   scale   > 0, at most 2.35e38; scores are scale * q.k
 *   out     [rows, n_q_heads, head_dim] in `dtype`, out_stride elements from row to row.  A row that sees nothing: 0
 *   lse     [rows, n_q_heads] fp32 or NULL: natural logarithm of the sum of exp(score); -inf for a row that sees nothing
 * q, k, v, out are 16-byte aligned, their strides whole 16 bytes.  A window row with a NaN or an infinity in v makes the rows that see it NaN,
 * and no others; finite values of v up to 2^100 in magnitude do not overflow (the largest weight of a row stands for 2^7 to 2^15 in sums of 32 bits).  S2D2_F32: products and sums as in 32 bits; S2D2_BF16: products of bf16 queries, softmax weights in half, sums in 32 bits. */
typedef struct {
  int32_t N, T, rows, n_q_heads, dtype;
  float scale;
  const void *q, *k, *v;
  int64_t q_stride, kv_stride, out_stride;
  const int32_t *row0, *n_rows, *lo, *hi;
  void* out;
  float* lse;
} s2d2_kv4_rows;

/* Rows n_rows[n] (values outside [0, T] are cut) of k, v [n_layers, rows, n_kv_heads, head_dim] in `dtype` from row row0[n] on, layer_stride and
 * row_stride elements apart (16-byte aligned, strides whole 16 bytes), become entries of all layers behind those of sequence n;
 * entries[n] and seq_len[n] advance.  mass of a new entry: 0 (what the rows of its own window gave it is not known here; an eviction right behind
 * an append should protect its rows, by `recent`); position: seq_len[n] + i.  Without room for all of them nothing of that
 * sequence is written and status[n] is set to S2D2_ENOSPC.  A sequence whose rows leave [0, rows) is skipped.  N <= 1024, N * T below 2^26. */
int32_t s2d2_kv4_append(void* stream, const s2d2_kv4_view* kv, int32_t N, int32_t T, int32_t rows, int32_t dtype, const void* k, const void* v,
                        int64_t layer_stride, int64_t row_stride, const int32_t* row0, const int32_t* n_rows);

/* Entries first[n] .. first[n] + T - 1 of every sequence and layer to k, v [n_layers, N, T, n_kv_heads, head_dim] in `dtype`, contiguous and
 * 16-byte aligned.  Places of entries that there are not are left as they were. */
int32_t s2d2_kv4_read(void* stream, const s2d2_kv4_view* kv, int32_t N, int32_t T, int32_t dtype, const int32_t* first, void* k, void* v);

/* Bytes of scratch that s2d2_kv4_attention needs for N windows of up to T rows on this cache; negative S2D2_E* on bad arguments. */
int64_t s2d2_kv4_attention_bytes(const s2d2_kv4_view* kv, int32_t N, int32_t T, int32_t n_q_heads);

/* Attention of the windows over the entries of `layer` and over themselves.  scratch: device, 16-byte aligned, s2d2_kv4_attention_bytes() or
 * more; its contents do not matter and nothing is kept in it.  Calls that run at the same time need a scratch each.  N <= 1024, T <= 8192,
 * N * (max_pages_per_seq * page_size + T + 64) below 2^36, N * T * n_q_heads at most 2^25. */
int32_t s2d2_kv4_attention(void* stream, const s2d2_kv4_view* kv, int32_t layer, const s2d2_kv4_rows* rows, void* scratch, size_t scratch_bytes);

/* mass of every cached entry of `layer` and KV head += sum over the rows of its sequence's window and the query heads of the KV head of
 * exp(scale * q.k - lse): with the lse that s2d2_kv4_attention wrote, the softmax weights that the rows gave the entry.  A row of lse -inf adds
 * nothing.  The window's own rows, which are no entries yet, get nothing (a single token can be appended first, and then attend to the entries alone).  k, v, lo, hi and out are not looked at (out may be NULL).  N <= 1024, T <= 8192. */
int32_t s2d2_kv4_weigh(void* stream, const s2d2_kv4_view* kv, int32_t layer, const s2d2_kv4_rows* rows);

/* Every sequence with more than budget + slack entries is cut to `budget`, list by list (a list: one layer, one KV head).  Kept are the entries of the
 * first `sink` positions (position < sink) and of the last `recent` (position >= seq_len[n] - recent), then those of the largest mass; ties: the
 * lower entry first; a NaN counts as less than any other mass.  The i-th entry below `budget` that goes is replaced by the i-th one from `budget` on that stays
 * (codes, scales, mass and position as they are); all others stay where they are.  entries[n] becomes budget.  Needs mass and position;
 * budget >= 1, slack >= 0, sink + recent <= budget.  N <= 1024, N * n_layers * n_kv_heads below 2^22.  scratch: device, 4-byte aligned, s2d2_kv4_evict_bytes() or more; its contents do not
 * matter and nothing is kept in it.  Calls that run at the same time need a scratch (and a cache) each. */
int32_t s2d2_kv4_evict(void* stream, const s2d2_kv4_view* kv, int32_t N, int32_t budget, int32_t slack, int32_t sink, int32_t recent, void* scratch,
                       size_t scratch_bytes);

/* Bytes of scratch that s2d2_kv4_evict needs for N sequences of this cache, whatever the budget (4 bytes for every place of a list and 4 for the
 * list); negative S2D2_E* on bad arguments. */
int64_t s2d2_kv4_evict_bytes(const s2d2_kv4_view* kv, int32_t N);

/* From this call on the calls of s2d2.h on `ctx` that take an s2d2_kv_view keep the prefix in this cache (NULL: in the view's own pages again).
 * Their views then have to describe it: k_pages = k_codes, v_pages = v_codes, the same page_table, seq_len, n_pages, page_size and
 * max_pages_per_seq (else S2D2_EINVAL).  n_layers, n_kv_heads and head_dim must be the model's.  Rows of a window are attended to as
 * the model's operand mode has them (by default queries and window keys as half: 11 bits, up to 65504; act_planes 1, 2: bf16 queries of one or two planes, bf16 keys) and quantised when they are appended.  With mass, s2d2_verify, s2d2_prefill and s2d2_block_complete add the weights of their windows' rows
 * (the drafting forward adds none), to the cached entries and to the rows that they see among themselves: the context's next append enters its rows with the mass
 * that the last of these forwards gave them (0 if there was none since this call).  s2d2_kv4_evict on the same cache may follow an append at any time: positions go by seq_len.
 * lse: device [s2d2_stage_rows(max_batch, max_block), n_q_heads] fp32, needed with mass; scratch: device, 16-byte aligned, at least
 * s2d2_kv4_attention_bytes(kv, max_batch, 3 * max_block, n_q_heads) bytes.  Both belong to the context while it runs. */
int32_t s2d2_set_kv4(s2d2_ctx* ctx, const s2d2_kv4_view* kv, void* scratch, size_t scratch_bytes, float* lse);

#ifdef __cplusplus
}
#endif
#endif /* S2D2_KV4_H */
