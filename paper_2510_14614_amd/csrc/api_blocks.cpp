// Entry points of the C ABI that take no context, continued: the parts of a
// gated block (head norms with rotated positions) declared in include/fal.h.
// Argument checks, then one call of the launchers.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>

#include "../../include/fal.h"
#include "api_checks.h"
#include "kernels.h"

using namespace fal;

namespace {

DType type_of(int32_t dtype) { return dtype == FAL_BF16 ? BF16 : F32; }

// ------------------------------------------------------------ head norms --
int64_t packed_width(const fal_qk_norm_rope_t* p) {
  const int64_t kv = p->n_kv_head ? p->n_kv_head : p->n_head;
  return (p->n_head + 2 * kv) * p->head_dim;
}

// A row stride of packed rows (name: the message's subject).
Refusal check_stride(const fal_qk_norm_rope_t* p, int64_t ld) {
  if (ld < packed_width(p)) return {FAL_ERR_INVALID_ARG, "a row stride is smaller than a row"};
  if (ld % (p->dtype == FAL_BF16 ? 8 : 4)) return {FAL_ERR_INVALID_ARG, "row strides must be multiples of 16 bytes"};
  if (ld > kMaxStride || ld > kMaxExtent / ((int64_t)p->batch * p->seq_len))
    return {FAL_ERR_INVALID_ARG, "batch * seq_len rows at this stride exceed the address space"};
  return kFine;
}

Refusal check_norm(const fal_qk_norm_rope_t* p) {
  if (!p) return {FAL_ERR_INVALID_ARG, "NULL shape"};
  if (p->dtype != FAL_F32 && p->dtype != FAL_BF16) return {FAL_ERR_INVALID_ARG, "unknown dtype"};
  if (p->batch < 1 || p->seq_len < 1) return {FAL_ERR_INVALID_ARG, "batch and seq_len must be >= 1"};
  if ((int64_t)p->batch * p->seq_len > 0x7fffffff) return {FAL_ERR_INVALID_ARG, "batch * seq_len must be below 2^31"};
  if (p->n_head < 1 || p->n_head > 65535) return {FAL_ERR_INVALID_ARG, "n_head must lie in [1, 65535]"};
  if (p->n_kv_head < 0 || (p->n_kv_head > 0 && p->n_head % p->n_kv_head))
    return {FAL_ERR_INVALID_ARG, "n_kv_head must be 0 or divide n_head"};
  if (p->head_dim != 16 && p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128)
    return {FAL_ERR_UNSUPPORTED, "head_dim must be 16, 32, 64 or 128 (not supported otherwise)"};
  if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim)
    return {FAL_ERR_INVALID_ARG, "rotary_dim must lie in [0, head_dim]"};
  if (p->rotary_dim % 8) return {FAL_ERR_UNSUPPORTED, "rotary_dim must be a multiple of 8 (not supported otherwise)"};
  if (p->interleaved != 0 && p->interleaved != 1) return {FAL_ERR_INVALID_ARG, "interleaved must be 0 or 1"};
  if (!std::isfinite(p->theta) || !(p->theta > 1.f)) return {FAL_ERR_INVALID_ARG, "theta must be finite and > 1"};
  if (!std::isfinite(p->eps) || !(p->eps > 0.f)) return {FAL_ERR_INVALID_ARG, "eps must be finite and > 0"};
  const Refusal no = check_stride(p, p->ld_qkv);
  return no.why ? no : check_stride(p, p->ld_out);
}

HeadNorm norm_args(const fal_qk_norm_rope_t* p, const void* wq, const void* wk, const int32_t* positions,
                   const int32_t* lens) {
  HeadNorm a;
  memset(&a, 0, sizeof(a));
  a.tokens = (int64_t)p->batch * p->seq_len;
  a.T = p->seq_len; a.H = p->n_head; a.Hkv = p->n_kv_head ? p->n_kv_head : p->n_head; a.hd = p->head_dim;
  a.rotary = p->rotary_dim; a.interleaved = p->interleaved; a.eps = p->eps;
  a.log2_theta_step = p->rotary_dim ? std::log2((double)p->theta) * 2.0 / p->rotary_dim : 0.0;
  a.wq = wq; a.wk = wk; a.positions = positions; a.lens = lens;
  a.ldx = a.lddx = p->ld_qkv;
  a.ldy = p->ld_out;
  return a;
}

}  // namespace

extern "C" {

fal_status_t fal_qk_norm_rope_workspace_bytes(const fal_qk_norm_rope_t* shape, size_t* bytes) {
  return guarded([&] {
    const Refusal no = check_norm(shape);
    if (no.why) return fail(no.st, no.why);
    if (!bytes) return fail(FAL_ERR_INVALID_ARG, "NULL bytes");
    *bytes = (size_t)head_norm_rope_scratch(norm_args(shape, nullptr, nullptr, nullptr, nullptr)) * 4;
    return FAL_OK;
  });
}

fal_status_t fal_qk_norm_rope_fwd(const fal_qk_norm_rope_t* shape, const void* qkv, const void* q_weight,
                                  const void* k_weight, const int32_t* positions, const int32_t* lens, void* out,
                                  void* stream) {
  return guarded([&] {
    const Refusal no = check_norm(shape);
    if (no.why) return fail(no.st, no.why);
    if (!qkv || !out) return fail(FAL_ERR_INVALID_ARG, "NULL qkv or out");
    const int64_t es = element_bytes(shape->dtype), w = shape->head_dim * es;
    if (!aligned(qkv, 16) || !aligned(out, 16)) return fail(FAL_ERR_INVALID_ARG, "qkv and out must be 16-byte aligned");
    if (!aligned(q_weight, es) || !aligned(k_weight, es) || !aligned(positions, 4) || !aligned(lens, 4))
      return fail(FAL_ERR_INVALID_ARG, "weights, positions or lens misaligned");
    const HeadNorm a = norm_args(shape, q_weight, k_weight, positions, lens);
    const Extent x = rows_of(qkv, a.tokens, a.ldx, packed_width(shape), es),
                 o = rows_of(out, a.tokens, a.ldy, packed_width(shape), es);
    if (!(out == qkv && a.ldx == a.ldy) && meets(o, {x}))
      return fail(FAL_ERR_INVALID_ARG, "out overlaps qkv (it may only be qkv itself, with its row stride)");
    if (meets(o, {{q_weight, w}, {k_weight, w}, {positions, a.tokens * 4}, {lens, (int64_t)shape->batch * 4}}))
      return fail(FAL_ERR_INVALID_ARG, "out overlaps another argument");
    return launched(head_norm_rope_fwd(type_of(shape->dtype), a, qkv, out, static_cast<hipStream_t>(stream)),
                    "fal_qk_norm_rope_fwd");
  });
}

fal_status_t fal_qk_norm_rope_bwd(const fal_qk_norm_rope_t* shape, const void* qkv, const void* q_weight,
                                  const void* k_weight, const int32_t* positions, const int32_t* lens,
                                  const void* d_out, void* d_qkv, int64_t ld_d_qkv, float* d_q_weight,
                                  float* d_k_weight, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&] {
    Refusal no = check_norm(shape);
    if (!no.why) no = check_stride(shape, ld_d_qkv);
    if (no.why) return fail(no.st, no.why);
    if (!qkv || !d_out || !d_qkv) return fail(FAL_ERR_INVALID_ARG, "NULL qkv, d_out or d_qkv");
    const int64_t es = element_bytes(shape->dtype), w = shape->head_dim * es, w4 = shape->head_dim * 4;
    if (!aligned(qkv, 16) || !aligned(d_out, 16) || !aligned(d_qkv, 16))
      return fail(FAL_ERR_INVALID_ARG, "qkv, d_out and d_qkv must be 16-byte aligned");
    if (!aligned(q_weight, es) || !aligned(k_weight, es) || !aligned(positions, 4) || !aligned(lens, 4) ||
        !aligned(d_q_weight, 4) || !aligned(d_k_weight, 4))
      return fail(FAL_ERR_INVALID_ARG, "weights, their gradients, positions or lens misaligned");
    HeadNorm a = norm_args(shape, q_weight, k_weight, positions, lens);
    a.lddx = ld_d_qkv;
    const int64_t need = head_norm_rope_scratch(a) * 4;
    if (!workspace || ws_bytes < (size_t)need || !aligned(workspace, kWorkspaceAlign))
      return fail(FAL_ERR_WORKSPACE, "workspace NULL, too small or not 256-byte aligned");
    const Extent x = rows_of(qkv, a.tokens, a.ldx, packed_width(shape), es),
                 g = rows_of(d_out, a.tokens, a.ldy, packed_width(shape), es),
                 d = rows_of(d_qkv, a.tokens, a.lddx, packed_width(shape), es), q = {q_weight, w}, k = {k_weight, w},
                 at = {positions, a.tokens * 4}, n = {lens, (int64_t)shape->batch * 4}, ws = {workspace, need};
    if (!(d_qkv == d_out && a.lddx == a.ldy) && meets(d, {g}))
      return fail(FAL_ERR_INVALID_ARG, "d_qkv overlaps d_out (it may only be d_out itself, with its row stride)");
    if (meets(d, {x, q, k, at, n, ws}) || meets(ws, {x, g, q, k, at, n}) ||
        outputs_meet({{d_q_weight, w4}, {d_k_weight, w4}}, {x, g, d, q, k, at, n, ws}))
      return fail(FAL_ERR_INVALID_ARG, "an output or the workspace overlaps another argument");
    return launched(head_norm_rope_bwd(type_of(shape->dtype), a, qkv, d_out, d_qkv, d_q_weight, d_k_weight,
                                       static_cast<float*>(workspace), static_cast<hipStream_t>(stream)),
                    "fal_qk_norm_rope_bwd");
  });
}

}  // extern "C"
