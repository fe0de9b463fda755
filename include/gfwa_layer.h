/*
 * gfwa_layer.h -- the operators that an attention layer of a model has directly around the calls of gfwa.h: from its
 * projection's output to the Q, K, V that the attention reads, back again for training, and the same work on a paged
 * key/value cache for serving.  Part of libgfwa; the conventions of gfwa.h hold (device pointers, the caller's stream,
 * status codes, nothing allocated, nothing launched on an error) except where a strided layout is named.  What a call writes
 * (outputs, cache, workspace) may not overlap what it reads, nor each other, judged by the ranges of bytes that the tensors span:
 * GFWA_ERR_OVERLAP (dq, dk and dv among each other are the one exception: there the first and last rows of each are looked for among the others' rows).
 * A workspace belongs to its call until that is done on the stream: calls that may run at the same time (two streams, two captured graphs) need one each.
 * Sizes: N (new tokens of a call) up to 2^24, B * H up to 2^24 (2^22 with a paged cache), B * H * ceil(N / 32) and B * N below 2^31: GFWA_ERR_DIM.
 */
#ifndef GFWA_LAYER_H
#define GFWA_LAYER_H

#include "gfwa.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A tensor of heads as a projection leaves it: element e of head h of token n of sequence b stands at
 * data + b * batch + n * token + h * head + e (strides in elements; e is contiguous).  The struct is host memory, read during
 * the call.  data must be 16-byte aligned and every stride of a dimension longer than one a multiple of 16 bytes, from 0
 * (outputs: rows must not overlap) up; the largest offset has to stay below 2^40 elements.
 */
typedef struct {
    void *data;
    long long batch, token, head;
} gfwa_heads_t;

enum {
    GFWA_HEAD_NORM = 1,   /* root-mean-square norm of every query and key head */
    GFWA_ROPE_PAIRED = 2  /* rotate dimensions (2j, 2j+1) together; otherwise (j, j + rot/2) */
};

/*
 * Norm and rotation of queries and keys (paper Sec. 3.3: the layer's queries and keys are normed per head; rotation as
 * usual), and the layout gfwa_forward_gqa reads.  For every row x (one head of one token) of q and k:
 *
 *   y = weight * x / sqrt(mean(x^2) + eps)      with GFWA_HEAD_NORM (weight NULL: ones), else y = x
 *   (y_i, y_j) -> (y_i cos a - y_j sin a, y_i sin a + y_j cos a),    a = p * freq[m],  m = 0 .. rot/2 - 1
 *
 * where p is the token's position and (i, j) is (m, m + rot/2), or (2m, 2m + 1) with GFWA_ROPE_PAIRED; dimensions from rot
 * on are not rotated.  Rows of v change their place alone.  fp32 arithmetic, rounded once; the angle is formed and
 * reduced in fp64.  Squares are fp32 numbers too: a row whose squares add up to more than 3.4e38 comes out as zeros, and with eps = 0 one
 * whose squares are all below 2^-149 as infinities or NaN.
 *
 * q: [B,N,H,d], k, v: [B,N,Hkv,d] of dtype `dt`, strided;  v may be NULL (V is then ignored).
 * wq, wk: [d] fp32 or NULL.  freq: [rot/2] fp64 in device memory, 8-byte aligned, in radians for each position; rot: a multiple of
 * 16 up to d, 0: no rotation, freq ignored.  pos: [B,N] int32 in device memory, any values; NULL: token n stands at position n.
 * Q: [B,H,N,d], K, V: [B,Hkv,N,d] of dtype `dt`, dense, out.
 * d in {64, 128}; Hkv divides H.
 */
int gfwa_qk_norm_rope(gfwa_dtype_t dt, const gfwa_heads_t *q, const gfwa_heads_t *k, const gfwa_heads_t *v, const float *wq,
                      const float *wk, float eps, const double *freq, int rot, const int *pos, int flags, void *Q, void *K,
                      void *V, int B, int H, int Hkv, int N, int d, gfwa_stream_t stream);

/* Bytes of device scratch gfwa_qk_norm_rope_backward needs for the sums of the weights' gradients (0 on invalid sizes). */
size_t gfwa_qk_norm_rope_backward_workspace_bytes(int B, int H, int Hkv, int N, int d);

/*
 * Its derivative.  With g the rows of dQ (dK) rotated back, r = 1 / sqrt(mean(x^2) + eps) and u = r x:
 *
 *   dx = r (weight g - u mean(weight g u)),    dweight = sum over all rows of g u       (without the norm: dx = g)
 *
 * q, k, wq, wk, eps, freq, rot, pos, flags: as given to gfwa_qk_norm_rope; q and k are read with GFWA_HEAD_NORM only and may be
 * NULL without it.  dQ: [B,H,N,d], dK, dV: [B,Hkv,N,d] of dtype `dt`, dense, as gfwa_backward_gqa writes them.
 * dq: [B,N,H,d], dk, dv: [B,N,Hkv,d] of dtype `dt`, strided, out (views of one packed gradient, say: their rows may interleave, but
 * share no element); dV and dv are both NULL or both given.  dwq, dwk: [d] fp32, out; each may be NULL; with GFWA_HEAD_NORM only
 * (without it they have to be NULL).  They are summed in an order that the sizes and the device alone decide.  workspace: device scratch of
 * at least gfwa_qk_norm_rope_backward_workspace_bytes(...) bytes, 16-byte aligned, contents undefined before and after; may
 * be NULL where dwq and dwk are.
 */
int gfwa_qk_norm_rope_backward(gfwa_dtype_t dt, const gfwa_heads_t *q, const gfwa_heads_t *k, const float *wq, const float *wk,
                               float eps, const double *freq, int rot, const int *pos, int flags, const void *dQ, const void *dK,
                               const void *dV, const gfwa_heads_t *dq, const gfwa_heads_t *dk, const gfwa_heads_t *dv, float *dwq,
                               float *dwk, void *workspace, size_t workspace_bytes, int B, int H, int Hkv, int N, int d,
                               gfwa_stream_t stream);

/*
 * The paged cache.  Kp, Vp: [pages,Hkv,page,d] of dtype `dt`;  cp: [pages,H,page] fp32, the gate prefix.  page: tokens of a page, a
 * multiple of 16.  table: [B,max_pages] int32 in device memory; position p of sequence b stands in row p % page of page
 * table[b, p / page].  Sequences may share pages that nothing appends to.  A table entry outside 0 .. pages-1 says that the
 * page is not there (a window has left it behind, or it was never given): nothing is read from it or written to it.
 * pages * heads * page * d may pass 2^31; max_pages * page (positions) may not, nor B * H 2^22.
 */

/*
 * Appends new tokens to the paged cache: norm and rotation of queries and keys as in gfwa_qk_norm_rope, on the way.
 * Row n of the new tokens belongs to the sequence b with start[b] <= n < start[b+1] and stands at position
 * p = cached[b] + n - start[b], by which it is rotated.  Keys and values go to the cache; queries to Q; and the prefix is
 * carried on,
 *
 *   c_p = c_{cached-1} + sum of alpha over the new tokens up to p     (fp64 sums, rounded once; c_{-1} = 0, and 0 where the
 *                                                                    page of position cached-1 is not there)
 *
 * k, v: [rows,Hkv,d], q: [rows,H,d] of dtype `dt`, strided (`batch` is ignored);  q NULL: no queries, Q is ignored.
 * alpha: fp32, gate of head h of row n at alpha[n * alpha_token + h * alpha_head] (strides of at least 0, offsets below 2^40);  NULL: cp is left
 * alone and may be NULL.
 * start: [B+1], cached: [B] int32 in device memory, start not decreasing, cached >= 0 (a sequence may have no new token).
 * Rows 0 .. rows-1 alone are there: where start begins in front of row 0 or ends behind the last row, the others' tokens are passed over.
 * Rows that belong to no sequence (in front of start[0], from start[B] on) are left out: their rows of Q stay as they were.  Of rows whose
 * position lies outside the table, or in a page that is not there, the query alone is written.
 * Q: [rows,H,d] of dtype `dt`, dense, out.  Two sequences must not append to one page, and what cached counts is in the cache before the call: none
 * of it may be a new token of another sequence of the same call (a prompt in two pieces takes two calls).
 *
 * What reads Q: gfwa_decode_paged, a query for each of its rows.  In a decoding step these are the batch's; of several new tokens every one
 * can be a row there, with its sequence's row of the table and its own position, which reads each one's window.  gfwa_forward_gqa reads no
 * pages: a prompt goes through gfwa_qk_norm_rope and the attention, and is appended without queries, from the projection's k and v (the
 * same bits as K and V have; rows of padding between sequences of a padded batch count as tokens and are written over by those that follow,
 * cached being the lengths without them) or, a sequence a call, from K and V themselves without norm and rotation.
 */
int gfwa_append_paged(gfwa_dtype_t dt, const gfwa_heads_t *q, const gfwa_heads_t *k, const gfwa_heads_t *v, const float *wq,
                      const float *wk, float eps, const double *freq, int rot, int flags, const float *alpha, long long alpha_token,
                      long long alpha_head, const int *start, const int *cached, const int *table, void *Q, void *Kp, void *Vp,
                      float *cp, int rows, int B, int H, int Hkv, int d, int pages, int page, int max_pages,
                      gfwa_stream_t stream);

/*
 * The decoding step of gfwa_decode against the paged cache: for every sequence b with position p = pos[b] (appended already) and
 * every query head h,
 *
 *   S_i = scale * <q, k_i> + (c_i - c_p)        for  max(0, p-w+1) <= i <= p  whose page is there
 *   o   = sum_i softmax_i(S_i) v_i              L = log sum_i exp(S_i)
 *
 * q: [B,H,d] of dtype `dt`, dense.  pos: [B] int32 in device memory; a position past the table is taken as its last one.  pos[b] < 0,
 * or a page of position p that is not there: the sequence has no token, o = 0 and L = -inf; so it is where every score is minus
 * infinity (scores below -2e38 count as that).
 * An infinite v_i whose weight softmax_i is not below 2^-126 of the largest is the result of its column, as the definition has it; below that its
 * weight is zero, and the column NaN.  Weights stand up to 2^16 above one on the way: finite values beyond about 2^100 may come out as infinities.
 * o: [B,H,d] of dtype `dt`, out.  L: [B,H] fp32 out, may be NULL.  workspace: device scratch of at least
 * gfwa_decode_paged_workspace_bytes(...) bytes, 16-byte aligned, contents undefined before and after.
 * Only the window is read: 2 * min(w, p+1) * d cache elements per key/value head, once for up to 16 query heads.
 */
/* (the query: 0 on invalid sizes) */
size_t gfwa_decode_paged_workspace_bytes(int B, int H, int Hkv, int d, int page, int max_pages, int w);
int gfwa_decode_paged(gfwa_dtype_t dt, const void *q, const void *Kp, const void *Vp, const float *cp, const int *table,
                      const int *pos, void *o, float *L, void *workspace, size_t workspace_bytes, int B, int H, int Hkv, int d,
                      int pages, int page, int max_pages, int w, float scale, gfwa_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* GFWA_LAYER_H */
