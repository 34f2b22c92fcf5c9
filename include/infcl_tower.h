/*
 * infcl_tower.h -- C ABI of the text tower's operators on AMD Instinct MI355X
 * (gfx950): what an encoder beside the tiled contrastive loss (infcl.h) runs.
 *
 *   token embedding        out_t = scale * table[token_t], and the table's
 *                          gradient by sorted tokens
 *   packed attention       grouped heads over sequences of different lengths,
 *                          packed row after row; forward and backward, and
 *                          few query tokens over many keys
 *   8-bit checkpoints      activations kept for the backward pass in 8 bits,
 *                          and the backward's uses of them
 *
 * Conventions (those of infcl.h): device pointers, 16-byte aligned unless
 * stated; element types INFCL_BF16, INFCL_F32, INFCL_F16; work is enqueued on
 * `stream` and nothing is allocated, cleared with memset nodes or waited for,
 * so the calls may be captured into a HIP graph; arguments are checked on the
 * host before anything is enqueued.  Workspaces are device memory, 256-byte
 * aligned, free to use again once the stream has passed the call.  No atomic
 * additions of floats: results are bitwise reproducible for given arguments.
 */
#ifndef INFCL_TOWER_H
#define INFCL_TOWER_H

#include <stddef.h>
#include <stdint.h>

#include "infcl.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Token embedding.
 * tokens [n]: int32 (token_bytes 4, 4-byte aligned) or int64 (8, 8-byte
 * aligned).  table [vocab, d] and out [n, d] of dtype, contiguous rows of whole
 * 16-byte units (d a multiple of 8, or 4 with fp32).  A token outside
 * [0, vocab) stands for nothing: its row of out is zero and it has no
 * gradient (padding may be marked by -1).
 * out_t = scale * table[token_t], one fp32 product rounded once to dtype. */
infcl_status infcl_embed_fwd(const void* tokens, int token_bytes, int64_t n, const void* table, int64_t vocab,
                             int64_t d, int dtype, float scale, void* out, void* stream);

/* dtable [vocab, d] of grad_dtype (INFCL_F32, or dtype):
 *   dtable_v = scale * sum over t with token_t = v of dout_t,
 * every row written (rows of absent tokens with zeros).  dout [n, d] of dtype.
 * The tokens are sorted (stable), the rows of one token summed in fp32 in order
 * of t, in parts of 32 or 64 where there are more.  n <= 2^26,
 * vocab < 2^31 - 1. */
infcl_status infcl_embed_bwd_workspace(int64_t n, int64_t vocab, int64_t d, size_t* bytes);
infcl_status infcl_embed_bwd(const void* tokens, int token_bytes, int64_t n, const void* dout, int64_t vocab,
                             int64_t d, int dtype, float scale, void* dtable, int grad_dtype, void* workspace,
                             size_t ws_bytes, void* stream);

/* ---- Packed attention.
 * Sequence z of nseq has the queries cu_q[z] .. cu_q[z+1] and the keys
 * cu_k[z] .. cu_k[z+1] (device, int32, nseq + 1 entries from 0 on, not
 * descending), m and n of them.  Query i sees key j where j < n and, with
 * causal, j <= i + n - m (the last query sees the last key).  heads is a multiple
 * of kv_heads; query head a reads key head a / (heads / kv_heads).
 *   s_ij = scale <q_i, k_j>, lse_i = log sum_j e^{s_ij}, out_i = sum_j e^{s_ij - lse_i} v_j
 * A query that sees no key has out = 0, lse = -infinity and no gradient.  Rows
 * from cu_q[nseq] (cu_k[nseq]) to the end of the arrays count as such queries
 * (keys that no one sees): their outputs and gradients are zeros.  What a masked
 * key, value, query or dout row holds reaches no one, infinities and NaN included;
 * those that are seen propagate (a query whose scores are all -infinity has no
 * weights: out and lse are NaN).
 * dtype is INFCL_BF16 or INFCL_F16 (MFMA products accumulated in fp32, softmax in
 * fp32, its weights rounded to dtype for the products with v, dout, q and k);
 * head_dim is a multiple of 8 up to 128 (built for 64 and 128), scale > 0.
 * max_q and max_k: upper bounds of m and n.  They set the grid only: results do
 * not depend on them beyond rounding, and smaller ones than the true lengths cost
 * time, not rows.
 * Views: entry (token t, head a, feature f) at data[t token_stride + a head_stride
 * + f], both strides multiples of 8, token_stride <= 2^23: q, k and v may be views
 * of one projection, and dq, dk, dv of its gradient. */
typedef struct {
  int64_t total_q, total_k; /* tokens of q, out, dq and of k, v */
  int32_t nseq, heads, kv_heads, head_dim, dtype, causal;
  int64_t max_q, max_k;
  float scale;
} infcl_attn_shape;

typedef struct {
  void* data;
  int64_t token_stride, head_stride; /* elements */
} infcl_attn_view;

/* Bytes of workspace of the two calls (either pointer may be NULL). */
infcl_status infcl_attn_workspace(const infcl_attn_shape* shape, size_t* fwd_bytes, size_t* bwd_bytes);

/* lse [heads][total_q] float (may be NULL): what the backward needs.
 * len_k [nseq] int32 (device, may be NULL): how many of a sequence's keys, from
 * its first on, there are, where its rows of k and v are room for more (a cache
 * that grows); n above is then the lesser of the two. */
infcl_status infcl_attn_fwd(const infcl_attn_shape* shape, infcl_attn_view q, infcl_attn_view k, infcl_attn_view v,
                            const int32_t* cu_q, const int32_t* cu_k, const int32_t* len_k, infcl_attn_view out,
                            float* lse, void* workspace, size_t ws_bytes, void* stream);

/* dq, dk, dv of dtype; out and lse as infcl_attn_fwd left them without len_k: the
 * backward pass is that of all keys cu_k[z] .. cu_k[z+1] (after a call with len_k it
 * would count the unused rows as seen). */
infcl_status infcl_attn_bwd(const infcl_attn_shape* shape, infcl_attn_view q, infcl_attn_view k, infcl_attn_view v,
                            const int32_t* cu_q, const int32_t* cu_k, infcl_attn_view out, const float* lse,
                            infcl_attn_view dout, infcl_attn_view dq, infcl_attn_view dk, infcl_attn_view dv,
                            void* workspace, size_t ws_bytes, void* stream);

/* ---- Activation checkpoints in 8 bits.
 * x [n, d] is kept as q [n, d] (int8, 16-byte aligned) and exps [n, ceil(d/32)]
 * (one byte): 32 consecutive features of a row share the least e >= -126 with
 * rint(max|x| 2^-e) <= 127, q = rint(x 2^-e) (ties to even), exps = e + 127, and
 * x^ = q 2^e stands for x: within 2^(e-1) of it, which is at most max|x| / 127 for
 * e > -126 (groups below 2^-119 or so are kept with e = -126, to 2^-127).  A maximum
 * that would round to 2^128 is kept as 127 2^121, entries of its group within 2^121.
 * A group that holds an infinity or a NaN has exponent byte 255 and reads back as
 * NaN.  d a multiple of 8; x_stride, dy_stride: elements from row to row (a multiple
 * of 8, >= d); the other arrays are contiguous.  In fp16, x^ and f(x^) are limited to
 * 65504 (an entry next to it rounds to 65536 in 8 bits); dx is not, as no product is.
 */
typedef enum {
  INFCL_ACT_NONE = 0,
  INFCL_ACT_GELU = 1,       /* x Phi(x), Phi by erf        */
  INFCL_ACT_QUICK_GELU = 2  /* x / (1 + e^(-1.702 x))      */
} infcl_act;

infcl_status infcl_ckpt8_pack(const void* x, int64_t x_stride, int64_t n, int64_t d, int dtype, void* q, void* exps,
                              void* stream);
infcl_status infcl_ckpt8_unpack(const void* q, const void* exps, int64_t n, int64_t d, int dtype, void* out,
                                void* stream);

/* out = f(x) and the checkpoint of x, in one pass; dx = dy f'(x^) from it.
 * act is GELU or QUICK_GELU; x, out, dy, dx of dtype, computed in fp32. */
infcl_status infcl_ckpt8_act_fwd(const void* x, int64_t x_stride, int64_t n, int64_t d, int dtype, int act, void* out,
                                 void* q, void* exps, void* stream);
infcl_status infcl_ckpt8_act_bwd(const void* dy, int64_t dy_stride, const void* q, const void* exps, int64_t n,
                                 int64_t d, int dtype, int act, void* dx, void* stream);

/* Weight gradient of a layer y = f(x) W^T from the checkpoint of x:
 *   dw [m, d] = dy^T f(x^),  dy [n, m] of dtype (INFCL_BF16 or INFCL_F16),
 * dw of grad_dtype (INFCL_F32 or dtype).  x^ enters the products in dtype: exactly
 * in bf16, and in fp16 down to its subnormal step; f(x^) is rounded to dtype.
 * Products are accumulated in fp32, and the result rounded once. */
infcl_status infcl_ckpt8_wgrad_workspace(int64_t n, int64_t d, int64_t m, size_t* bytes);
infcl_status infcl_ckpt8_wgrad(const void* dy, int64_t dy_stride, const void* q, const void* exps, int64_t n, int64_t d,
                               int64_t m, int dtype, int act, void* dw, int grad_dtype, void* workspace,
                               size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* INFCL_TOWER_H */
