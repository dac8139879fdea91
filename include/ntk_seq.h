/*
 * ntk_seq.h -- C ABI of the operators of a sequence model's block on MI355X (gfx950): root-mean-square
 * norm, rotary positions and attention, forward, backward and for single tokens.
 *
 * They compute what stands in front of the networks of ntk.h when these read the features of a sequence
 * trunk: the trunk's pass (its output is the X of ntk_compute), the trunk's gradients, and its answer token
 * by token over a cache.
 *
 * Conventions, as in ntk.h: the caller owns every pointer and the workspace; a call checks its
 * arguments on the host, enqueues on `hip_stream` (NULL = the default stream) and returns before the work is
 * done; nothing is allocated, and nothing is kept between calls.  NTK_OK or a negative NTK_E_* code comes back, the
 * message is read with ntk_last_error(NULL), and on NTK_E_ARG / NTK_E_SHAPE / NTK_E_UNSUPPORTED nothing is
 * enqueued.  No C++ exception crosses this interface.  Every result is deterministic (no atomics), and
 * the calls can be captured in a HIP graph.
 *
 * Arrays hold fp32, bf16 or fp16 (`dtype`); sums, softmax statistics and norms are fp32.  Rows and heads
 * may lie at any stride, and pointers at any multiple of the element size: 16-byte accesses are used where every array of a
 * call allows them (addresses, strides and the head or row length in whole 16 bytes), single
 * elements otherwise.  Values that are not finite spread as the formulas say; what a mask hides does not
 * spread.
 */
#ifndef NTK_SEQ_H_
#define NTK_SEQ_H_

#include "ntk.h"

#ifdef __cplusplus
extern "C" {
#endif

#define NTK_F32  0
#define NTK_BF16 1
#define NTK_F16  2

/* ---- root-mean-square norm -----------------------------------------------------------------------
 * h = x + residual (residual NULL: h = x),  r = (mean(h^2) + eps)^(-1/2) over each row,  y = h r weight.
 *   x, residual   [rows, width], `*_stride` elements between rows (>= width).
 *   weight        [width] of type wtype: dtype, or NTK_F32.
 *   y             [rows, width] contiguous, of dtype; or, with `scale` not NULL, 8-bit e4m3 values q with
 *                 q[row] scale[row] = y: scale = max|y| / 448 (at least 2^-126), 1 for a row of zeros.
 *   h             [rows, width] contiguous, of dtype: the sum, for the next block and the backward pass; may
 *                 be NULL, and may be x or residual itself where that is contiguous.
 *   scale         [rows] fp32, or NULL.
 * y follows from h before h is rounded to dtype.  Rows of any size keep their bits: where squares would leave fp32's range
 * the row is taken times a power of two.  1 <= width <= 32768; rows may be 0.
 *
 * ntk_rms_norm_bwd: with g = dy weight,  dx = r (g - h r^2 mean(g h)) + dh  (the gradient of x and of the residual),
 * dweight = sum over rows of dy h r, all at the h that is given: the one that the forward pass rounded to dtype.
 *   dh            the gradient that reaches h otherwise, or NULL.
 *   dx            [rows, width] contiguous, of dtype; may be dy or dh where that is contiguous.
 *   dweight       [width] of wtype.
 *   workspace     ntk_rms_norm_workspace(rows, width) bytes, 16-byte aligned (dweight's partial sums). */
int ntk_rms_norm(int dtype, int wtype, long long rows, int width, const void* x, long long x_stride, const void* residual,
                 long long residual_stride, const void* weight, float eps, void* y, void* h, float* scale,
                 void* hip_stream);
long long ntk_rms_norm_workspace(long long rows, int width);
int ntk_rms_norm_bwd(int dtype, int wtype, long long rows, int width, const void* dy, long long dy_stride, const void* h,
                     long long h_stride, const void* weight, const void* dh, long long dh_stride, float eps, void* dx,
                     void* dweight, void* workspace, long long workspace_bytes, void* hip_stream);

/* An array [batch, position, head, dim] in device memory: dim contiguous, the other strides in elements
 * (>= 0).  Inputs may be broadcast (a stride of 0); an output whose stride is below the head size, or that starts where another
 * array of its call does (but for rotary in place), is refused.  Other overlaps are the caller's to avoid. */
typedef struct ntk_view {
    void* data;
    long long stride_batch, stride_position, stride_head;
} ntk_view;

/* ---- rotary positions ------------------------------------------------------------------------------
 * ntk_rotary_table -- table[p][j] = mag (cos(p f_j), sin(p f_j)) for p < max_pos, j < rot / 2, angles in 64 bits,
 * f_j = base^(-2 j / rot), changed for contexts longer than the trained one by
 *   NTK_ROTARY_PLAIN   nothing;
 *   NTK_ROTARY_LINEAR  f_j / factor (positions are interpolated);
 *   NTK_ROTARY_BASE    base factor^(rot / (rot - 2)) in place of base (the slowest pair is interpolated by
 *                      factor, the fastest kept);
 *   NTK_ROTARY_RAMP    f_j (k_j + (1 - k_j) / factor), where k_j grows from 0 to 1 as the pair's turns over
 *                      `original` positions grow from `low` to `high`; mag = 0.1 log(factor) + 1 (else 1).
 *   table              [max_pos, rot / 2, 2] fp32.  base > 1; factor >= 1; original >= 1; 0 <= low < high.
 *
 * ntk_rotary -- turns the first `rot` elements of every head of q (and of k, unless NULL) at its position:
 * (u, v) -> (u c - v s, v c + u s), and copies the others.  The pairs are (x[j], x[j + rot / 2]), or with `interleaved`
 * (x[2 j], x[2 j + 1]).  `inverse`: by -s, which carries gradients back, and undoes the turn where mag is 1 (with
 * NTK_ROTARY_RAMP it gives mag^2 times what was turned).
 *   positions   [batch, length] int32, or NULL: first_position + index.  A position outside the table gives NaN.
 *   q_out       may be q itself (in place), and k_out k; no other overlap.
 * rot is even, 2 <= rot <= dim.  batch, length and head counts may be 0. */
#define NTK_ROTARY_PLAIN  0
#define NTK_ROTARY_LINEAR 1
#define NTK_ROTARY_BASE   2
#define NTK_ROTARY_RAMP   3
typedef struct ntk_rotary_scaling {
    int kind;                       /* NTK_ROTARY_* */
    double factor, original, low, high;
} ntk_rotary_scaling;
int ntk_rotary_table(int max_pos, int rot, double base, const ntk_rotary_scaling* scaling, float* table,
                     void* hip_stream);
int ntk_rotary(int dtype, int batch, int length, int q_heads, int k_heads, int dim, int rot, int interleaved, int inverse,
               const ntk_view* q, const ntk_view* k, const float* table, int max_pos, const int* positions,
               int first_position, const ntk_view* q_out, const ntk_view* k_out, void* hip_stream);

/* ---- attention ---------------------------------------------------------------------------------------
 * o[i] = sum_j P[i, j] v[j] for every query head, P = softmax over the keys j that query i sees of
 *
 *     s[i, j] = softcap tanh(scale q[i].k[j] / softcap) - slope |p_i - j|      (no cap with softcap = 0).
 *
 * Query head h reads key/value head h / (heads / kv_heads).  A batch entry has n = k_lens[b] keys (k_len without
 * k_lens) and its q_len queries are the last q_len positions: p_i = n - q_len + i.  So q_len = k_len is a whole
 * sequence, and q_len = 1 over a cache of k_len places, n of them filled, is the next token.  Query i sees key j if
 *   j < n,  p_i >= 0,  (not causal) or j <= p_i or j < prefix[b],  and docs[b, j] = docs[b, p_i] >= 0
 * as far as each applies.  A query that sees no key has o = 0, lse = -inf and no gradient.  What a query does
 * not see has no effect on it, whatever the values there.
 *   dtype                    of q, k, v, o and their gradients.
 *   heads, kv_heads          heads a multiple of kv_heads.  1 <= head_dim <= 128.
 *   scale > 0; softcap >= 0.
 *   k_lens, prefix           [batch] int32 or NULL (values are clamped to 0 .. k_len).
 *   docs                     [batch, k_len] int32 or NULL: a document number a position, negative for padding.
 *   slopes                   [heads] fp32 or NULL.
 *   lse                      [batch, heads, q_len] fp32 or NULL: log of the softmax's sum (natural).
 *   o                        must not overlap q, k or v.
 *   workspace                ntk_attention_workspace(desc, 0) bytes, 16-byte aligned: partial results of the ranges that
 *                            the keys are cut into where there are few rows, and flags (it may be 0).
 *
 * ntk_attention_bwd -- dq, dk and dv from dout, with o and lse of the forward call.  softcap, slopes and masks as
 * there; the slopes get no gradient.  Keys past k_lens get zeros.  dq, dk, dv must not overlap the inputs.
 *   workspace                ntk_attention_workspace(desc, 1) bytes.
 * The p and ds factors of the products over the keys (rows), forward and backward, are rounded to dtype, in fp16 under powers of
 * two that keep them in its range, and the backward pass goes by the o that was rounded to dtype.  With a cap, scores of bf16 and fp16
 * have an absolute error of about 2^-22 softcap.  fp32 products are formed from three bf16 parts of each operand and are
 * good to 2^-22; where one meets an infinity or a NaN, on the fp32 matrix instructions. */
typedef struct ntk_attention_desc {
    int dtype, batch, q_len, k_len, heads, kv_heads, head_dim, causal;
    float scale, softcap;
    const int* k_lens;
    const int* prefix;
    const int* docs;
    const float* slopes;
} ntk_attention_desc;

/* Bytes, or a negative NTK_E_* code. */
long long ntk_attention_workspace(const ntk_attention_desc* desc, int backward);
int ntk_attention(const ntk_attention_desc* desc, const ntk_view* q, const ntk_view* k, const ntk_view* v, const ntk_view* o,
                  float* lse, void* workspace, long long workspace_bytes, void* hip_stream);
int ntk_attention_bwd(const ntk_attention_desc* desc, const ntk_view* dout, const ntk_view* q, const ntk_view* k,
                      const ntk_view* v, const ntk_view* o, const float* lse, const ntk_view* dq, const ntk_view* dk,
                      const ntk_view* dv, void* workspace, long long workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* NTK_SEQ_H_ */
