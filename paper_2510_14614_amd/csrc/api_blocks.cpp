// Entry points of the C ABI that take no context, continued: the parts of a
// gated block (head norms with rotated positions, the gated feed-forward
// block) and orthogonal updates of its matrices, declared in include/fal.h.
// Argument checks, then one call of the launchers.
#include <hip/hip_runtime.h>

#include <algorithm>
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

// Whether packed rows may lie `ld` elements apart.
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

// ----------------------------------------------------- gated feed-forward --
constexpr int64_t kMaxProduct = (int64_t)1 << 33;  // elements of a product
// Rows of fp32: tiles of 64 of them, two products of 256 threads a tile in one launch,
// are fewer than 2^32 threads.
constexpr int32_t kMaxRows = (1 << 29) - 64;

Refusal check_gated(const fal_gated_ffn_t* p) {
  if (!p) return {FAL_ERR_INVALID_ARG, "NULL shape"};
  if (p->dtype != FAL_F32 && p->dtype != FAL_BF16) return {FAL_ERR_INVALID_ARG, "unknown dtype"};
  if (p->grad_dtype != p->dtype && p->grad_dtype != FAL_F32)
    return {FAL_ERR_INVALID_ARG, "grad_dtype must be dtype or FAL_F32"};
  if (p->activation < FAL_GATE_SILU || p->activation > FAL_GATE_GELU_ERF)
    return {FAL_ERR_INVALID_ARG, "unknown activation"};
  if (p->rows < 1) return {FAL_ERR_INVALID_ARG, "rows must be >= 1"};
  const int32_t most = 1 << 20;
  if (p->d_model < 1 || p->d_model > most || p->d_ff < 1 || p->d_ff > most)
    return {FAL_ERR_INVALID_ARG, "d_model and d_ff must lie in [1, 2^20]"};
  const int64_t d = p->d_model, f = p->d_ff;
  if (p->ld_x < d || p->ld_y < d || p->ld_gate < f || p->ld_up < f || p->ld_down < d)
    return {FAL_ERR_INVALID_ARG, "a row stride is smaller than a row"};
  if ((p->ld_dx && p->ld_dx < d) || (p->ld_dgate && p->ld_dgate < f) || (p->ld_dup && p->ld_dup < f) ||
      (p->ld_ddown && p->ld_ddown < d))
    return {FAL_ERR_INVALID_ARG, "a gradient's row stride is smaller than a row"};
  for (int64_t ld : {p->ld_x, p->ld_y, p->ld_gate, p->ld_up, p->ld_down, p->ld_dx, p->ld_dgate, p->ld_dup, p->ld_ddown})
    if (ld > kMaxStride) return {FAL_ERR_INVALID_ARG, "row stride above 2^40 elements"};
  for (int64_t ld : {p->ld_x, p->ld_y, p->ld_dx})
    if (ld > kMaxExtent / p->rows) return {FAL_ERR_INVALID_ARG, "rows at this stride exceed the address space"};
  // (a launch's tiles of up to four products are counted in 32 bits)
  if (p->rows * std::max(d, f) > kMaxProduct || d * f > kMaxProduct)
    return {FAL_ERR_UNSUPPORTED, "rows * d_ff, rows * d_model or d_model * d_ff above 2^33 is not supported"};
  if (p->rows > kMaxRows) return {FAL_ERR_UNSUPPORTED, "more than 2^29 - 64 rows are not supported"};
  if (p->dtype == FAL_F32) return kFine;
  if (d % 8 || f % 8) return {FAL_ERR_UNSUPPORTED, "bf16 d_model and d_ff must be multiples of 8 (not supported otherwise)"};
  if (p->ld_x % 8 || p->ld_y % 8 || p->ld_gate % 8 || p->ld_up % 8 || p->ld_down % 8 || p->ld_dx % 8 ||
      p->ld_dgate % 8 || p->ld_dup % 8 || p->ld_ddown % 8)
    return {FAL_ERR_INVALID_ARG, "bf16 row strides must be multiples of 8"};
  // 32-bit byte offsets inside an operand, whose last slices of k run up to 256
  // rows past its end
  auto fits = [](int64_t rows, int64_t ld) { return (rows + 256) * ld * 2 < ((int64_t)1 << 31) - (1 << 20); };
  if (!fits(p->rows, p->ld_x) || !fits(p->rows, p->ld_y) || !fits(p->rows, f) || !fits(d, p->ld_gate) ||
      !fits(d, p->ld_up) || !fits(f, p->ld_down))
    return {FAL_ERR_UNSUPPORTED, "bf16 operands of 2 GiB or more are not supported"};
  return kFine;
}

GatedFfn gated_args(const fal_gated_ffn_t* p) {
  GatedFfn a;
  a.M = p->rows; a.d = p->d_model; a.f = p->d_ff;
  a.act = p->activation == FAL_GATE_SILU ? GATE_SILU : p->activation == FAL_GATE_GELU_TANH ? GATE_GELU_TANH
                                                                                          : GATE_GELU_ERF;
  a.ldx = p->ld_x; a.ldy = p->ld_y; a.ldg = p->ld_gate; a.ldu = p->ld_up; a.ldd = p->ld_down;
  a.lddx = p->ld_dx ? p->ld_dx : p->ld_x;
  a.lddg = p->ld_dgate ? p->ld_dgate : p->ld_gate;
  a.lddu = p->ld_dup ? p->ld_dup : p->ld_up;
  a.lddd = p->ld_ddown ? p->ld_ddown : p->ld_down;
  a.grads_f32 = p->grad_dtype == FAL_F32;
  return a;
}

// Whether two [rows, width] matrices share no element: apart, or of one row stride
// with their columns beside each other, as the halves of one matrix are.
bool interleave_free(const void* a, const void* b, int64_t rows, int64_t ld_a, int64_t ld_b, int64_t width,
                     int64_t es) {
  if (!meets(rows_of(a, rows, ld_a, width, es), {rows_of(b, rows, ld_b, width, es)})) return true;
  if (ld_a != ld_b) return false;
  const int64_t apart = static_cast<const char*>(b) - static_cast<const char*>(a), step = ld_a * es;
  const int64_t in = ((apart % step) + step) % step;
  return in >= width * es && in + width * es <= step;
}

// ---------------------------------------------------- orthogonal updates --
NewtonSchulz schulz_args(const fal_newton_schulz_t* p) {
  return {type_of(p->dtype), p->count, p->rows, p->cols, p->steps, p->a, p->b, p->c, p->stride,
          p->out_stride ? p->out_stride : p->stride};
}

Refusal check_schulz(const fal_newton_schulz_t* p) {
  if (!p) return {FAL_ERR_INVALID_ARG, "NULL shape"};
  if (p->dtype != FAL_F32 && p->dtype != FAL_BF16) return {FAL_ERR_INVALID_ARG, "unknown dtype"};
  if (p->count < 1 || p->rows < 1 || p->cols < 1) return {FAL_ERR_INVALID_ARG, "count, rows and cols must be >= 1"};
  // (one workgroup a matrix where they are small)
  if (p->count > 1 << 22) return {FAL_ERR_UNSUPPORTED, "more than 2^22 matrices are not supported"};
  if (p->steps < 1 || p->steps > kMaxNewtonSteps) return {FAL_ERR_INVALID_ARG, "steps must lie in [1, 32]"};
  if (!std::isfinite(p->a) || !std::isfinite(p->b) || !std::isfinite(p->c))
    return {FAL_ERR_INVALID_ARG, "coefficients must be finite"};
  // 32-bit byte offsets inside a 16-bit copy of a matrix
  const int64_t r = ((int64_t)p->rows + 127) / 128 * 128, c = ((int64_t)p->cols + 127) / 128 * 128;
  if (r * c > ((int64_t)1 << 30) - (1 << 20))
    return {FAL_ERR_UNSUPPORTED, "matrices of more than 2^30 - 2^20 elements (sides rounded up to 128) are not supported"};
  const int64_t one = (int64_t)p->rows * p->cols;
  if (p->stride < one || (p->out_stride && p->out_stride < one))
    return {FAL_ERR_INVALID_ARG, "stride or out_stride is smaller than a matrix"};
  if (p->stride > kMaxExtent / p->count || p->out_stride > kMaxExtent / p->count)
    return {FAL_ERR_INVALID_ARG, "count matrices at this stride exceed the address space"};
  double sigma[kMaxNewtonSteps + 1];
  if (!newton_schulz_bounds(schulz_args(p), sigma))
    return {FAL_ERR_INVALID_ARG, "coefficients let singular values grow past 2^20"};
  return kFine;
}

Extent matrices_of(const void* p, const fal_newton_schulz_t* s, int64_t stride, int64_t es) {
  return {p, ((s->count - 1) * stride + (int64_t)s->rows * s->cols) * es};
}

}  // namespace

extern "C" {

fal_status_t fal_newton_schulz_workspace_bytes(const fal_newton_schulz_t* shape, size_t* bytes) {
  return guarded([&] {
    const Refusal no = check_schulz(shape);
    if (no.why) return fail(no.st, no.why);
    if (!bytes) return fail(FAL_ERR_INVALID_ARG, "NULL bytes");
    *bytes = (size_t)newton_schulz_scratch(schulz_args(shape));
    return FAL_OK;
  });
}

fal_status_t fal_newton_schulz(const fal_newton_schulz_t* shape, const void* x, void* out, void* workspace,
                               size_t ws_bytes, void* stream) {
  return guarded([&] {
    const Refusal no = check_schulz(shape);
    if (no.why) return fail(no.st, no.why);
    if (!x || !out) return fail(FAL_ERR_INVALID_ARG, "NULL x or out");
    const int64_t es = element_bytes(shape->dtype);
    if (!aligned(x, es) || !aligned(out, es)) return fail(FAL_ERR_INVALID_ARG, "x or out misaligned");
    const int64_t need = newton_schulz_scratch(schulz_args(shape));
    if (!workspace || ws_bytes < (size_t)need || !aligned(workspace, kWorkspaceAlign))
      return fail(FAL_ERR_WORKSPACE, "workspace NULL, too small or not 256-byte aligned");
    const NewtonSchulz n = schulz_args(shape);
    const Extent a = matrices_of(x, shape, n.stride, es), o = matrices_of(out, shape, n.out_stride, es),
                 ws = {workspace, need};
    if ((!(out == x && n.out_stride == n.stride) && meets(o, {a})) || meets(ws, {a, o}))
      return fail(FAL_ERR_INVALID_ARG, "out or the workspace overlaps another argument (out may only be x itself, with its stride)");
    return launched(newton_schulz(n, nullptr, x, out, workspace, static_cast<hipStream_t>(stream)),
                    "fal_newton_schulz");
  });
}

fal_status_t fal_muon_step(const fal_newton_schulz_t* shape, const fal_muon_t* hp, float* master, void* params,
                           const float* grads, float* momentum, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&] {
    const Refusal no = check_schulz(shape);
    if (no.why) return fail(no.st, no.why);
    if (!hp) return fail(FAL_ERR_INVALID_ARG, "NULL hyper-parameters");
    for (float v : {hp->lr, hp->beta, hp->weight_decay, hp->scale})
      if (!std::isfinite(v) || v < 0.f)
        return fail(FAL_ERR_INVALID_ARG, "lr, beta, weight_decay and scale must be finite and >= 0");
    if (hp->beta >= 1.f) return fail(FAL_ERR_INVALID_ARG, "beta must lie in [0, 1)");
    if (shape->out_stride) return fail(FAL_ERR_INVALID_ARG, "out_stride must be 0 in an update");
    if (hp->nesterov != 0 && hp->nesterov != 1) return fail(FAL_ERR_INVALID_ARG, "nesterov must be 0 or 1");
    if (!master || !grads || !momentum) return fail(FAL_ERR_INVALID_ARG, "NULL master, grads or momentum");
    if (params == master && shape->dtype == FAL_F32) params = nullptr;
    const int64_t es = element_bytes(shape->dtype);
    if (!aligned(master, 4) || !aligned(grads, 4) || !aligned(momentum, 4) || !aligned(params, es))
      return fail(FAL_ERR_INVALID_ARG, "master, params, grads or momentum misaligned");
    const int64_t need = newton_schulz_scratch(schulz_args(shape));
    if (!workspace || ws_bytes < (size_t)need || !aligned(workspace, kWorkspaceAlign))
      return fail(FAL_ERR_WORKSPACE, "workspace NULL, too small or not 256-byte aligned");
    if (outputs_meet({matrices_of(master, shape, shape->stride, 4), matrices_of(params, shape, shape->stride, es),
                      matrices_of(momentum, shape, shape->stride, 4), {workspace, need}},
                     {matrices_of(grads, shape, shape->stride, 4)}))
      return fail(FAL_ERR_INVALID_ARG, "master, params, momentum or the workspace overlaps another argument");
    MuonArgs u;
    u.grads = grads; u.momentum = momentum; u.master = master;
    u.beta = hp->beta;
    u.decay = (float)(1.0 - (double)hp->lr * hp->weight_decay);
    u.step = (float)((double)hp->lr * hp->scale);
    u.nesterov = hp->nesterov;
    return launched(newton_schulz(schulz_args(shape), &u, nullptr, params, workspace, static_cast<hipStream_t>(stream)),
                    "fal_muon_step");
  });
}

fal_status_t fal_gated_ffn_workspace_bytes(const fal_gated_ffn_t* shape, size_t* forward, size_t* backward) {
  return guarded([&] {
    const Refusal no = check_gated(shape);
    if (no.why) return fail(no.st, no.why);
    if (forward) *forward = (size_t)gated_ffn_scratch(type_of(shape->dtype), gated_args(shape), 0);
    if (backward) *backward = (size_t)gated_ffn_scratch(type_of(shape->dtype), gated_args(shape), 1);
    return FAL_OK;
  });
}

fal_status_t fal_gated_ffn_fwd(const fal_gated_ffn_t* shape, const void* x, const void* w_gate, const void* w_up,
                               const void* w_down, void* y, float* saved, void* workspace, size_t ws_bytes,
                               void* stream) {
  return guarded([&] {
    const Refusal no = check_gated(shape);
    if (no.why) return fail(no.st, no.why);
    if (!x || !w_gate || !w_up || !w_down || !y) return fail(FAL_ERR_INVALID_ARG, "NULL x, y or weight");
    const GatedFfn a = gated_args(shape);
    const int64_t es = element_bytes(shape->dtype), to = shape->dtype == FAL_BF16 ? 16 : 4;
    if (!aligned(x, to) || !aligned(w_gate, to) || !aligned(w_up, to) || !aligned(w_down, to) || !aligned(y, to) ||
        !aligned(saved, 16))
      return fail(FAL_ERR_INVALID_ARG, "an array is misaligned (bf16 and saved: 16 bytes, fp32: 4)");
    const int64_t need = gated_ffn_scratch(type_of(shape->dtype), a, 0);
    if (!workspace || ws_bytes < (size_t)need || !aligned(workspace, kWorkspaceAlign))
      return fail(FAL_ERR_WORKSPACE, "workspace NULL, too small or not 256-byte aligned");
    if (outputs_meet({rows_of(y, a.M, a.ldy, a.d, es), {saved, (int64_t)a.M * a.f * 8}, {workspace, need}},
                     {rows_of(x, a.M, a.ldx, a.d, es), rows_of(w_gate, a.d, a.ldg, a.f, es),
                      rows_of(w_up, a.d, a.ldu, a.f, es), rows_of(w_down, a.f, a.ldd, a.d, es)}))
      return fail(FAL_ERR_INVALID_ARG, "y, saved or the workspace overlaps another argument");
    return launched(gated_ffn_fwd(type_of(shape->dtype), a, x, w_gate, w_up, w_down, y, saved, workspace,
                                  static_cast<hipStream_t>(stream)),
                    "fal_gated_ffn_fwd");
  });
}

fal_status_t fal_gated_ffn_bwd(const fal_gated_ffn_t* shape, const void* x, const void* w_gate, const void* w_up,
                               const void* w_down, const float* saved, const void* dy, void* dx, void* dw_gate,
                               void* dw_up, void* dw_down, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&] {
    const Refusal no = check_gated(shape);
    if (no.why) return fail(no.st, no.why);
    if (!x || !w_gate || !w_up || !w_down || !saved || !dy)
      return fail(FAL_ERR_INVALID_ARG, "NULL x, weight, saved or dy");
    if (!dw_gate != !dw_up || !dw_gate != !dw_down)
      return fail(FAL_ERR_INVALID_ARG, "dw_gate, dw_up and dw_down must all be given or all be NULL");
    const GatedFfn a = gated_args(shape);
    const int64_t es = element_bytes(shape->dtype), eg = element_bytes(shape->grad_dtype);
    const int64_t to = shape->dtype == FAL_BF16 ? 16 : 4;
    if (!aligned(x, to) || !aligned(w_gate, to) || !aligned(w_up, to) || !aligned(w_down, to) || !aligned(dy, to) ||
        !aligned(saved, 16) || !aligned(dx, to) || !aligned(dw_gate, to) || !aligned(dw_up, to) ||
        !aligned(dw_down, to))
      return fail(FAL_ERR_INVALID_ARG, "an array is misaligned (bf16 and saved: 16 bytes, fp32: 4)");
    const int64_t need = gated_ffn_scratch(type_of(shape->dtype), a, 1);
    if (!workspace || ws_bytes < (size_t)need || !aligned(workspace, kWorkspaceAlign))
      return fail(FAL_ERR_WORKSPACE, "workspace NULL, too small or not 256-byte aligned");
    const Extent in[] = {rows_of(x, a.M, a.ldx, a.d, es), rows_of(w_gate, a.d, a.ldg, a.f, es),
                         rows_of(w_up, a.d, a.ldu, a.f, es), rows_of(w_down, a.f, a.ldd, a.d, es),
                         {saved, (int64_t)a.M * a.f * 8}, rows_of(dy, a.M, a.ldy, a.d, es)};
    const Extent g = rows_of(dw_gate, a.d, a.lddg, a.f, eg), u = rows_of(dw_up, a.d, a.lddu, a.f, eg),
                 d = rows_of(dw_down, a.f, a.lddd, a.d, eg), ox = rows_of(dx, a.M, a.lddx, a.d, es),
                 ws = {workspace, need};
    bool bad = meets(ws, {in[0], in[1], in[2], in[3], in[4], in[5]});
    // dw_gate and dw_up may be the halves of one matrix
    for (const Extent& o : {g, u, d, ox}) bad = bad || (o.p && meets(o, {in[0], in[1], in[2], in[3], in[4], in[5], ws}));
    if (dw_gate)
      bad = bad || meets(d, {g, u}) || !interleave_free(dw_gate, dw_up, a.d, a.lddg, a.lddu, a.f, eg) ||
            (dx && meets(ox, {g, u, d}));
    if (bad) return fail(FAL_ERR_INVALID_ARG, "an output or the workspace overlaps another argument");
    return launched(gated_ffn_bwd(type_of(shape->dtype), a, x, w_gate, w_up, w_down, saved, dy, dx, dw_gate, dw_up,
                                  dw_down, workspace, static_cast<hipStream_t>(stream)),
                    "fal_gated_ffn_bwd");
  });
}

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
