/*
 * brq_attn.h -- C ABI of the attention side of a block-rotated MXFP4 layer for MI355X (gfx950).
 *
 * What stands between the W4A4 products of brq.h: the norm of every query and key head with the
 * position rotation, a cache of keys and values in MXFP4, attention over that cache, and the
 * bookkeeping of its pages.  The conventions of brq.h hold (device pointers, caller-owned buffers,
 * nothing allocated, work enqueued on `stream`, argument errors found on the host before anything is
 * launched), and these besides:
 *   - A set of heads (brq_heads) is x[t][h][d] = data[t * token_stride + h * head_stride + d] of one
 *     dtype, d < D contiguous; strides are in elements and any multiples of 16 bytes from 0 on, so that
 *     queries, keys and values may be views of one packed projection.  Outputs may not overlap inputs.
 *     T tokens of a set have T * heads < 2^25 heads together.
 *   - What the host cannot see is checked on the device where memory depends on it: a position outside
 *     the tables, a slot or page number outside the cache, a length or offset outside its table is
 *     never used to address memory; what comes out instead is stated at each call.
 *   - Block rotations are those of brq_block_rotate inside each head: B = 1 none, else a power of two,
 *     8 <= B <= D.  They leave attention unchanged when queries and keys take the same one
 *     ((q R)(k R)^T = q k^T); values rotated on their way into the cache give outputs in the rotated
 *     basis, which is what brq_rotate_quantize_fused makes online in front of the output projection:
 *     brq_mxfp4_quantize on them is enough there, with the same projection weights (rotated by Bv).
 */
#ifndef BRQ_ATTN_H
#define BRQ_ATTN_H

#include "brq.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    void* data;
    int64_t heads, token_stride, head_stride;
} brq_heads;

/*
 * Rotation by position of the first `rot` channels of a head: channel pair i < rot/2 of a token at
 * position p, (a, b) -> (a cos[p][i] - b sin[p][i], b cos[p][i] + a sin[p][i]); the pair is channels
 * (i, i + rot/2), or (2i, 2i + 1) where `interleaved`.  rot % 16 == 0, rot <= D.
 * cos, sin: [rows][rot/2] fp32, contiguous, 16-byte aligned; positions: [T], 0 <= positions[t] < rows.
 */
typedef struct {
    const float *cos, *sin;
    const int64_t* positions;
    int64_t rows, rot;
    int32_t interleaved;
} brq_rope;

/*
 * Queries and keys of T tokens on their way to attention, one pass:
 *     n = x / sqrt(mean_d x^2 + eps) * w        (w NULL: n = x)
 *     y = rope(n) * diag(H_B, ..., H_B) / sqrt(B)          (rope NULL: no rotation by position)
 * in fp32, rounded once to ydt.  q and q_out, k and k_out: the same number of heads; k and k_out may be
 * NULL together.  wq, wk: [D] fp32, each may be NULL.  D = 64, 128 or 256.
 * A token whose position is outside the tables comes out as NaN.
 */
brq_status brq_qk_norm_rope(const brq_heads* q, const brq_heads* k, brq_dtype xdt, int64_t T, int64_t D,
                            const float* wq, const float* wk, float eps, const brq_rope* rope, int64_t B,
                            const brq_heads* q_out, const brq_heads* k_out, brq_dtype ydt, void* stream);

/*
 * Its gradients: from those of the outputs (gq, gk, of gdt) and the inputs (q, k, of xdt),
 *     gn = rope^-1(g * diag(H_B, ..., H_B) / sqrt(B)),      dw[d] = sum_{t,h} gn x / sqrt(mean x^2 + eps),
 *     dx = (gn w - x * mean_d(gn w x) / (mean x^2 + eps)) / sqrt(mean x^2 + eps)        (w NULL: dx = gn)
 * dq, dk of xdt; dwq, dwk [D] fp32 are set, not added to (NULL: not wanted; must be NULL where the weight is).
 * The sums over tokens and heads are made in an order that depends on the sizes alone.
 * A token whose position is outside the tables has NaN for its dx, and dw has it in its sums.
 * workspace: brq_qk_norm_rope_backward_workspace bytes, 16-byte aligned; may be NULL where dwq and dwk are.
 */
brq_status brq_qk_norm_rope_backward(const brq_heads* q, const brq_heads* k, brq_dtype xdt, int64_t T, int64_t D,
                                     const float* wq, const float* wk, float eps, const brq_rope* rope, int64_t B,
                                     const brq_heads* gq, const brq_heads* gk, brq_dtype gdt, const brq_heads* dq,
                                     const brq_heads* dk, float* dwq, float* dwk, void* workspace,
                                     int64_t workspace_bytes, void* stream);
brq_status brq_qk_norm_rope_backward_workspace(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t* bytes);

/*
 * The cache: num_pages pages of BRQ_KV4_PAGE tokens in one buffer (16-byte aligned), each page
 * brq_kv4_page_bytes = Hk * 68 * D bytes, contiguous.  A head of a page is 68 * D bytes: with t the token's
 * place in the page, codes packed as in brq.h, G = D/32 scale groups, P = D/32 code bytes a column:
 *     key code byte j        at              t * D/2 + j
 *     key scale of group n   at   32 D       + (n * 16 + t % 16) * 4 + t / 16
 *     value code byte j      at   34 D       + ((t / 4 * 16 + j / P) * 4 + t % 4) * P + j % P
 *     value scale of group n at   66 D       + ((t / 4 % 4 * G + n) * 4 + t / 16) * 4 + t % 4
 * These are the orders in which the matrix cores take them: 16 tokens of keys, or 4 tokens of a column of
 * values, are one load of a lane each.  Bytes of tokens that were never written are never used.
 * A slot is page * BRQ_KV4_PAGE + place.  D = 64 or 128.
 */
#define BRQ_KV4_PAGE 64
brq_status brq_kv4_page_bytes(int64_t Hk, int64_t D, int64_t* bytes);

/*
 * Writes the keys and values of T tokens to slots[t] (distinct; a slot outside the cache: the token is not
 * written):  keys as brq_qk_norm_rope makes them, kept in fp32, then brq_mxfp4_quantize; values v H_Bv /
 * sqrt(Bv), then the same, except that no scale is above 2^125, the largest under which all codes are finite
 * (infinities and NaN saturate): what a token's value holds is nothing to rows that do not see it.
 * Queries of the same tokens may come along (q, q_out of xdt; NULL together: none).
 * Everything else as in brq_qk_norm_rope.  A token whose position is outside the tables is not written.
 */
brq_status brq_kv4_append(const brq_heads* q, const brq_heads* k, const brq_heads* v, brq_dtype xdt, int64_t T,
                          int64_t D, const float* wq, const float* wk, float eps, const brq_rope* rope, int64_t B,
                          int64_t Bv, const int64_t* slots, uint8_t* pool, int64_t num_pages,
                          const brq_heads* q_out, void* stream);

/*
 * The values that stand in the cache: k_out, v_out of BRQ_BF16 or BRQ_F32 (exact in either), [T][Hk][D] as
 * their heads' strides say.  A slot outside the cache reads as NaN.
 */
brq_status brq_kv4_read(const uint8_t* pool, int64_t num_pages, int64_t T, int64_t D, const int64_t* slots,
                        const brq_heads* k_out, const brq_heads* v_out, brq_dtype ydt, void* stream);

/*
 * Attention of T query rows of S sequences over the cache.  Sequence s has query rows cu_q[s] ... cu_q[s+1] - 1
 * (cu_q: [S + 1], ascending, or rows may be left unwritten; NULL: one row each, T = S) and the tokens
 * 0 ... kv_lens[s] - 1, token j in page table[s * table_cols + j / 64].  Its queries are the last of them: row i
 * of n stands at position p = kv_lens[s] - n + i.  With Hk heads in the cache, q.heads a multiple of it, query
 * head h reads head h / (q.heads / Hk):
 *     a_j = scale * q . k_j  for the j that the row sees,   o = sum_j exp(a_j) v_j / sum_j exp(a_j),
 *     lse = log sum_j exp(a_j)
 * The row sees j < kv_lens[s]; with `causal` j <= p, and with window > 0 (causal only) j > p - window.  Lengths
 * below 0 count as 0; rows in front of the first token (p < 0) are rows like others.  A row that sees nothing
 * has o = 0, lse = -infinity; a NaN in a query makes its row NaN and no other.  Tokens whose page number is
 * outside the cache are not seen.
 * q and out are BRQ_BF16; lse [T][q.heads] fp32 or NULL; scale is a finite number (of magnitude below 2^-126, 0
 * included: taken for 2^-126).  Arithmetic: products exact, summed in the matrix cores' fp32, softmax in fp32, its
 * weights rounded to bf16 in front of the product with the values (of up to 32 rows, query rows x heads of a group,
 * to a sequence at most: divided by the sum of the rounded weights; of more: by the weights' own).
 * max_q, max_kv: what the host knows of the longest query and context; rows beyond max_q of a sequence, and rows
 * that are no sequence's, are not written, tokens at max_kv and beyond not seen.  They size the grid and the workspace.
 * T * q.heads < 2^25, q.heads and Hk < 2^16, S * Hk < 2^22, max_q and table_cols < 2^25, max_kv < 2^31 - 64.
 * workspace: brq_kv4_attention_workspace bytes (may be 0, then NULL), 16-byte aligned.
 */
brq_status brq_kv4_attention(const brq_heads* q, int64_t T, int64_t D, const uint8_t* pool, int64_t num_pages,
                             int64_t Hk, const int32_t* table, int64_t table_cols, const int32_t* kv_lens,
                             const int32_t* cu_q, int64_t S, float scale, int causal, int64_t window, int64_t max_q,
                             int64_t max_kv, const brq_heads* out, float* lse, void* workspace,
                             int64_t workspace_bytes, void* stream);
brq_status brq_kv4_attention_workspace(int64_t T, int64_t S, int64_t Hq, int64_t Hk, int64_t D, int64_t max_q,
                                       int64_t max_kv, int64_t* bytes);

/*
 * Pages.  A scheduler's state is on the device: table [S][table_cols] int32 page numbers (-1: none), lens [S]
 * int32 tokens, refs [num_pages] int32 how many table entries name a page (0: free).  A sequence has
 * ceil(len / 64) pages, or more after a reservation.  Pages are taken lowest number first, by the order of the
 * calls' lists, so that results do not depend on the schedule.  Sequence numbers outside 0 ... S - 1 and page
 * numbers outside the cache are passed over.
 *
 * copy:    page dst[i] = page src[i].  No dst may be another pair's src or dst.
 * fork:    sequence child[i] (distinct, not a parent, without pages) becomes a copy of parent[i]: full pages
 *          are shared (refs + 1), a last page that is not full is copied to a page taken from the free ones.
 *          failed[0] (int32) is set to the number of pairs for which none was left: their child stays empty.
 * free:    the pages of seq[i] are given up (refs - 1), its row becomes -1, its length 0.
 * reserve: in the rows of sequences seq[i] (distinct) every column below ceil(tokens[i] / 64) that has no page gets one
 *          (lengths are not changed).  A sequence gets all it needs or nothing: nothing where its need and those of
 *          the sequences before it in the list are more than the free pages, or where the table has too few
 *          columns; failed[0] (int32) is set to the number of those.
 * compact: the live pages move to the lowest numbers: the k-th free page below their count gets the k-th
 *          live page above it.  table and refs follow; live[0] (int32) is set to the count.
 * workspace: brq_kv4_pages_workspace bytes (compact: n = 0), 16-byte aligned.  S and S * table_cols < 2^31,
 * num_pages < 2^29, table_cols < 2^25, n < 2^21; page_bytes is a multiple of 16 below 2^31.
 */
brq_status brq_kv4_pages_workspace(int64_t n, int64_t num_pages, int64_t* bytes);
brq_status brq_kv4_pages_copy(uint8_t* pool, int64_t page_bytes, int64_t num_pages, const int32_t* src,
                              const int32_t* dst, int64_t n, void* stream);
brq_status brq_kv4_pages_fork(uint8_t* pool, int64_t page_bytes, int64_t num_pages, int32_t* table, int64_t S,
                              int64_t table_cols, int32_t* lens, int32_t* refs, const int32_t* parent,
                              const int32_t* child, int64_t n, int32_t* failed, void* workspace, void* stream);
brq_status brq_kv4_pages_free(int32_t* table, int64_t S, int64_t table_cols, int32_t* lens, int32_t* refs,
                              int64_t num_pages, const int32_t* seq, int64_t n, void* stream);
brq_status brq_kv4_pages_reserve(int32_t* table, int64_t S, int64_t table_cols, int32_t* refs, int64_t num_pages,
                                 const int32_t* seq, const int32_t* tokens, int64_t n,
                                 int32_t* failed, void* workspace, void* stream);
brq_status brq_kv4_pages_compact(uint8_t* pool, int64_t page_bytes, int64_t num_pages, int32_t* table, int64_t S,
                                 int64_t table_cols, int32_t* refs, int32_t* live, void* workspace, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BRQ_ATTN_H */
