// C ABI of packed attention: argument checks, plans and launches.
#include "attn.hpp"

namespace infcl {
AttnFwdPlan attn_fwd_plan(const AttnArgs& a, int64_t max_q, int64_t max_k);
int launch_attn_fwd(const AttnArgs& a, const AttnFwdPlan& p, int dtype, uint16_t* out, int64_t os, int64_t oh,
                    float* lse, char* ws, hipStream_t st);
AttnBwdPlan attn_bwd_plan(const AttnArgs& a, int64_t max_q, int64_t max_k);
int launch_attn_bwd(const AttnArgs& a, const AttnBwdPlan& p, int dtype, int64_t max_q, int64_t max_k,
                    const uint16_t* out, int64_t os, int64_t oh, const float* lse, const uint16_t* dout, int64_t dos,
                    int64_t doh, uint16_t* dq, int64_t dqs, int64_t dqh, uint16_t* dk, int64_t dks, int64_t dkh,
                    uint16_t* dv, int64_t dvs, int64_t dvh, char* ws, hipStream_t st);
}  // namespace infcl

using namespace infcl;

namespace {

constexpr int64_t kMaxTokens = ((int64_t)1 << 31) - 65536;
constexpr int64_t kMaxStride = (int64_t)1 << 23;  // elements: 64 rows fit a 31-bit offset in bytes

bool aligned(const void* p, size_t a) { return p != nullptr && ((uintptr_t)p % a) == 0; }

// INFCL_OK, or what is wrong with the call's sizes.
infcl_status shape_status(const infcl_attn_shape* s) {
  if (!s || s->total_q < 0 || s->total_k < 0 || s->nseq < 0 || s->heads < 1 || s->kv_heads < 1 || s->head_dim < 1 ||
      s->heads % s->kv_heads != 0 || s->max_q < 0 || s->max_k < 0 || (s->causal != 0 && s->causal != 1) ||
      !(s->scale > 0.f) || s->scale > 3e38f ||
      (s->dtype != INFCL_BF16 && s->dtype != INFCL_F16 && s->dtype != INFCL_F32))
    return INFCL_ERR_INVALID;
  if (s->dtype == INFCL_F32 || s->head_dim % 8 != 0 || s->head_dim > 128 || s->total_q > kMaxTokens ||
      s->total_k > kMaxTokens || s->heads > 4096 || s->nseq > (1 << 24))
    return INFCL_ERR_UNSUPPORTED;
  // rows of a sequence in 31 bits; a wave for each sequence and key head in one launch
  const int64_t group = s->heads / s->kv_heads, mq = s->max_q < s->total_q ? s->max_q : s->total_q;
  if (mq * group > kMaxTokens || ((int64_t)s->nseq + 1) * s->kv_heads > kAttnItems / 64) return INFCL_ERR_UNSUPPORTED;
  return INFCL_OK;
}

bool view_ok(const infcl_attn_view& v, int64_t tokens, int64_t hd) {
  return tokens == 0 || (aligned(v.data, 16) && v.token_stride >= hd && v.head_stride >= 0);
}
bool view_supported(const infcl_attn_view& v) {
  return v.token_stride % 8 == 0 && v.head_stride % 8 == 0 && v.token_stride <= kMaxStride &&
         v.head_stride <= ((int64_t)1 << 40);
}

AttnArgs args_of(const infcl_attn_shape* s, const infcl_attn_view& q, const infcl_attn_view& k,
                 const infcl_attn_view& v, const int32_t* cu_q, const int32_t* cu_k, const int32_t* len_k) {
  AttnArgs a;
  a.q = (const uint16_t*)q.data, a.k = (const uint16_t*)k.data, a.v = (const uint16_t*)v.data;
  a.qs = q.token_stride, a.qh = q.head_stride, a.ks = k.token_stride, a.kh = k.head_stride;
  a.vs = v.token_stride, a.vh = v.head_stride;
  a.cu_q = cu_q, a.cu_k = cu_k, a.len_k = len_k;
  a.tq = s->total_q, a.tk = s->total_k;
  a.nseq = s->nseq, a.heads = s->heads, a.kvh = s->kv_heads, a.group = s->heads / s->kv_heads;
  a.hd = s->head_dim, a.causal = s->causal;
  a.scale = s->scale, a.sl2 = s->scale * kLog2e;
  return a;
}

int64_t least(int64_t a, int64_t b) { return a < b ? a : b; }

}  // namespace

extern "C" infcl_status infcl_attn_workspace(const infcl_attn_shape* s, size_t* fwd_bytes, size_t* bwd_bytes) {
  const infcl_status st = shape_status(s);
  if (st != INFCL_OK) return st;
  const infcl_attn_view none = {nullptr, 0, 0};
  const AttnArgs a = args_of(s, none, none, none, nullptr, nullptr, nullptr);
  if (fwd_bytes) *fwd_bytes = attn_fwd_plan(a, least(s->max_q, s->total_q), least(s->max_k, s->total_k)).total;
  if (bwd_bytes) *bwd_bytes = attn_bwd_plan(a, least(s->max_q, s->total_q), least(s->max_k, s->total_k)).total;
  return fwd_bytes || bwd_bytes ? INFCL_OK : INFCL_ERR_INVALID;
}

extern "C" infcl_status infcl_attn_fwd(const infcl_attn_shape* s, infcl_attn_view q, infcl_attn_view k,
                                       infcl_attn_view v, const int32_t* cu_q, const int32_t* cu_k,
                                       const int32_t* len_k, infcl_attn_view out, float* lse, void* workspace,
                                       size_t ws_bytes, void* stream) {
  const infcl_status st = shape_status(s);
  if (st != INFCL_OK) return st;
  if (s->total_q == 0) return INFCL_OK;
  const int64_t hd = s->head_dim;
  if (!view_ok(q, s->total_q, hd) || !view_ok(k, s->total_k, hd) || !view_ok(v, s->total_k, hd) ||
      !view_ok(out, s->total_q, hd) || !aligned(cu_q, 4) || !aligned(cu_k, 4) ||
      (len_k && !aligned(len_k, 4)) || (lse && !aligned(lse, 4)))
    return INFCL_ERR_INVALID;
  if (!view_supported(q) || !view_supported(k) || !view_supported(v) || !view_supported(out))
    return INFCL_ERR_UNSUPPORTED;
  const AttnArgs a = args_of(s, q, k, v, cu_q, cu_k, len_k);
  const AttnFwdPlan p = attn_fwd_plan(a, least(s->max_q, s->total_q), least(s->max_k, s->total_k));
  if (p.total > 0 && !aligned(workspace, 256)) return INFCL_ERR_INVALID;
  if (ws_bytes < p.total) return INFCL_ERR_WORKSPACE;
  return (infcl_status)launch_attn_fwd(a, p, s->dtype, (uint16_t*)out.data, out.token_stride, out.head_stride, lse,
                                       (char*)workspace, (hipStream_t)stream);
}

extern "C" infcl_status infcl_attn_bwd(const infcl_attn_shape* s, infcl_attn_view q, infcl_attn_view k,
                                       infcl_attn_view v, const int32_t* cu_q, const int32_t* cu_k, infcl_attn_view out,
                                       const float* lse, infcl_attn_view dout, infcl_attn_view dq, infcl_attn_view dk,
                                       infcl_attn_view dv, void* workspace, size_t ws_bytes, void* stream) {
  const infcl_status st = shape_status(s);
  if (st != INFCL_OK) return st;
  if (s->total_q == 0 && s->total_k == 0) return INFCL_OK;
  const int64_t hd = s->head_dim;
  if (!view_ok(q, s->total_q, hd) || !view_ok(k, s->total_k, hd) || !view_ok(v, s->total_k, hd) ||
      !view_ok(out, s->total_q, hd) || !view_ok(dout, s->total_q, hd) || !view_ok(dq, s->total_q, hd) ||
      !view_ok(dk, s->total_k, hd) || !view_ok(dv, s->total_k, hd) || !aligned(cu_q, 4) || !aligned(cu_k, 4) ||
      (s->total_q > 0 && !aligned(lse, 4)) || !aligned(workspace, 256))
    return INFCL_ERR_INVALID;
  if (!view_supported(q) || !view_supported(k) || !view_supported(v) || !view_supported(out) ||
      !view_supported(dout) || !view_supported(dq) || !view_supported(dk) || !view_supported(dv))
    return INFCL_ERR_UNSUPPORTED;
  const AttnArgs a = args_of(s, q, k, v, cu_q, cu_k, nullptr);
  const int64_t mq = least(s->max_q, s->total_q), mk = least(s->max_k, s->total_k);
  const AttnBwdPlan p = attn_bwd_plan(a, mq, mk);
  if (ws_bytes < p.total) return INFCL_ERR_WORKSPACE;
  return (infcl_status)launch_attn_bwd(
      a, p, s->dtype, mq, mk, (const uint16_t*)out.data,
      out.token_stride, out.head_stride, lse, (const uint16_t*)dout.data, dout.token_stride, dout.head_stride,
      (uint16_t*)dq.data, dq.token_stride, dq.head_stride, (uint16_t*)dk.data, dk.token_stride, dk.head_stride,
      (uint16_t*)dv.data, dv.token_stride, dv.head_stride, (char*)workspace, (hipStream_t)stream);
}
