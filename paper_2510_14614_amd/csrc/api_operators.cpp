// Entry points of the C ABI that take no context: windowed attention, token
// log-probabilities and the policy and preference losses (declared in
// include/fal.h).  Argument checks, then one call of the launchers.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>

#include "../../include/fal.h"
#include "api_checks.h"
#include "kernels.h"

using namespace fal;

namespace {

constexpr uintptr_t kWorkspaceAlign = 256;
constexpr int64_t kMaxStride = (int64_t)1 << 40;  // elements between rows
constexpr int64_t kMaxExtent = (int64_t)1 << 47;  // elements from a matrix's first row to its last: the address space

fal_status_t fail(fal_status_t st, const char* why) {
  noctx_error() = why;
  return st;
}

fal_status_t launched(hipError_t e, const char* call) {
  if (e == hipSuccess) return FAL_OK;
  noctx_error() = std::string(call) + ": " + hipGetErrorString(e);
  return FAL_ERR_HIP;
}

// No C++ exception (the message string may fail to allocate) leaves a C entry.
template <typename F>
fal_status_t guarded(F f) {
  try {
    noctx_error().clear();
    return f();
  } catch (...) {
    return FAL_ERR_HIP;
  }
}

struct Refusal {
  fal_status_t st;
  const char* why;
};
const Refusal kFine = {FAL_OK, nullptr};

// ------------------------------------------------------- window attention --
// Whether a shape's rows at a stride of ld elements stay within kMaxExtent.
bool fits(const fal_window_attention_t* p, int64_t ld) {
  return ld <= kMaxExtent / ((int64_t)p->batch * p->seq_len);
}

Refusal check_shape(const fal_window_attention_t* p) {
  if (!p) return {FAL_ERR_INVALID_ARG, "NULL shape"};
  if (p->dtype != FAL_F32 && p->dtype != FAL_BF16) return {FAL_ERR_INVALID_ARG, "unknown dtype"};
  if (p->batch < 1 || p->batch > 65535) return {FAL_ERR_INVALID_ARG, "batch must lie in [1, 65535]"};
  if (p->seq_len < 1 || p->seq_len > kMaxWindowSeq) return {FAL_ERR_INVALID_ARG, "seq_len must lie in [1, 2^22]"};
  if (p->n_head < 1 || p->n_head > 65535) return {FAL_ERR_INVALID_ARG, "n_head must lie in [1, 65535]"};
  if (p->n_kv_head < 0 || (p->n_kv_head > 0 && p->n_head % p->n_kv_head))
    return {FAL_ERR_INVALID_ARG, "n_kv_head must be 0 or divide n_head"};
  if (p->window < 1) return {FAL_ERR_INVALID_ARG, "window must be >= 1"};
  if (p->sinks < 0) return {FAL_ERR_INVALID_ARG, "sinks must be >= 0"};
  if (p->sinks > kMaxSinks) return {FAL_ERR_UNSUPPORTED, "more than 128 sinks are not supported"};
  if (p->head_dim != 16 && p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128)
    return {FAL_ERR_UNSUPPORTED, "head_dim must be 16, 32, 64 or 128 (not supported otherwise)"};
  const int64_t kv = p->n_kv_head ? p->n_kv_head : p->n_head;
  const int64_t chunk = p->dtype == FAL_BF16 ? 8 : 4;  // elements of 16 bytes
  if (p->ld_qkv < (p->n_head + 2 * kv) * p->head_dim) return {FAL_ERR_INVALID_ARG, "ld_qkv is smaller than a row"};
  if (p->ld_out < (int64_t)p->n_head * p->head_dim) return {FAL_ERR_INVALID_ARG, "ld_out is smaller than a row"};
  if (p->ld_qkv % chunk || p->ld_out % chunk)
    return {FAL_ERR_INVALID_ARG, "row strides must be multiples of 16 bytes"};
  if (p->ld_qkv > kMaxStride || p->ld_out > kMaxStride) return {FAL_ERR_INVALID_ARG, "row stride above 2^40 elements"};
  if (!fits(p, p->ld_qkv) || !fits(p, p->ld_out))
    return {FAL_ERR_INVALID_ARG, "batch * seq_len rows at this stride exceed the address space"};
  return kFine;
}

WindowAttn window_args(const fal_window_attention_t* p, const int32_t* lens) {
  WindowAttn a;
  memset(&a, 0, sizeof(a));
  a.B = p->batch; a.T = p->seq_len; a.H = p->n_head; a.Hkv = p->n_kv_head ? p->n_kv_head : p->n_head;
  a.hd = p->head_dim; a.window = std::min(p->window, p->seq_len); a.sinks = p->sinks;
  a.lens = lens;
  a.ldq = a.lddq = p->ld_qkv;
  a.ldo = a.lddo = p->ld_out;
  return a;
}

// A row matrix's bytes from its first element to its last.
Extent rows_of(const void* p, int64_t rows, int64_t ld, int64_t width, int64_t es) {
  return {p, ((rows - 1) * ld + width) * es};
}

int64_t window_scratch_bytes(int32_t dtype, const WindowAttn& a, int64_t* part_off) {
  int64_t n = (int64_t)a.B * a.H * a.T * 4;
  n = (n + kWorkspaceAlign - 1) / kWorkspaceAlign * kWorkspaceAlign;
  *part_off = n;
  return n + window_attention_scratch(dtype == FAL_BF16 ? BF16 : F32, a) * 4;
}

// ------------------------------------------------------------ logit rows --
Refusal check_rows(const fal_logit_rows_t* r, bool gradient) {
  if (!r) return {FAL_ERR_INVALID_ARG, "NULL rows"};
  if (r->dtype != FAL_F32 && r->dtype != FAL_BF16) return {FAL_ERR_INVALID_ARG, "unknown dtype"};
  if (r->batch < 1 || r->seq_len < 1) return {FAL_ERR_INVALID_ARG, "batch and seq_len must be >= 1"};
  if ((int64_t)r->batch * r->seq_len > (1 << 24)) return {FAL_ERR_INVALID_ARG, "batch*seq_len too large"};
  if (r->vocab < 1 || r->vocab > (1 << 20)) return {FAL_ERR_INVALID_ARG, "vocab must lie in [1, 2^20]"};
  const int64_t most = (int64_t)1 << 32;
  if (r->ld_logits < r->vocab || r->ld_logits > most)
    return {FAL_ERR_INVALID_ARG, "ld_logits must lie in [vocab, 2^32]"};
  if (r->ld_targets < r->seq_len || r->ld_targets > most)
    return {FAL_ERR_INVALID_ARG, "ld_targets must lie in [seq_len, 2^32]"};
  if (gradient && (r->dlogits_cols < r->vocab || r->ld_dlogits < r->dlogits_cols || r->ld_dlogits > most))
    return {FAL_ERR_INVALID_ARG, "dlogits_cols must lie in [vocab, ld_dlogits], ld_dlogits be at most 2^32"};
  // (the kernels count columns in 32 bits, a workgroup's stride past the last one included)
  if (gradient && r->dlogits_cols > (1 << 30)) return {FAL_ERR_INVALID_ARG, "dlogits_cols must be at most 2^30"};
  if (const char* why = check_temperature(r->temperature)) return {FAL_ERR_INVALID_ARG, why};
  return kFine;
}

LogitRows row_args(const fal_logit_rows_t* r, const void* logits, const int32_t* targets, const uint8_t* mask) {
  LogitRows a;
  memset(&a, 0, sizeof(a));
  a.logits = logits; a.targets = targets; a.mask = mask;
  a.B = r->batch; a.T = r->seq_len; a.V = r->vocab; a.width = r->dlogits_cols;
  a.ldl = r->ld_logits; a.ldt = r->ld_targets; a.ldd = r->ld_dlogits;
  a.set_temperature(r->temperature);
  return a;
}

int64_t element_bytes(int32_t dtype) { return dtype == FAL_BF16 ? 2 : 4; }

// The checks that both losses share: dlogits may be the logits, and meets
// nothing else; the small outputs meet nothing.
Refusal check_loss(const fal_logit_rows_t* r, const void* logits, const int32_t* targets, const uint8_t* mask,
                   const void* dlogits, const void* workspace, size_t ws_bytes, std::initializer_list<Extent> in,
                   std::initializer_list<Extent> out) {
  const int64_t es = element_bytes(r->dtype), N = (int64_t)r->batch * r->seq_len;
  if (!aligned(logits, es) || !aligned(dlogits, es)) return {FAL_ERR_INVALID_ARG, "logits or dlogits misaligned"};
  if (!aligned(targets, 4)) return {FAL_ERR_INVALID_ARG, "targets must be 4-byte aligned"};
  if (!all_aligned(in, 4) || !all_aligned(out, 4)) return {FAL_ERR_INVALID_ARG, "fp32 arrays must be 4-byte aligned"};
  const int64_t need = logit_loss_scratch(r->batch, r->seq_len) * 4;
  if (!workspace || ws_bytes < (size_t)need || !aligned(workspace, kWorkspaceAlign))
    return {FAL_ERR_WORKSPACE, "workspace NULL, too small or not 256-byte aligned"};
  const Extent x = rows_of(logits, N, r->ld_logits, r->vocab, es),
               dx = rows_of(dlogits, N, r->ld_dlogits, r->dlogits_cols, es),
               tg = rows_of(targets, r->batch, r->ld_targets, r->seq_len, 4), mk = {mask, N}, ws = {workspace, need};
  const bool in_place = dlogits == logits && r->ld_dlogits == r->ld_logits;
  if ((!in_place && meets(dx, {x})) || meets(dx, {tg, mk, ws}) || meets(ws, {x, tg, mk}))
    return {FAL_ERR_INVALID_ARG, "dlogits or workspace overlaps an input (dlogits may only be the logits themselves)"};
  for (const Extent& e : in)
    if (meets(dx, {e}) || meets(ws, {e})) return {FAL_ERR_INVALID_ARG, "dlogits or workspace overlaps an input"};
  if (outputs_meet(out, {x, dx, tg, mk, ws}) || outputs_meet(out, in))
    return {FAL_ERR_INVALID_ARG, "an output overlaps another argument"};
  return kFine;
}

}  // namespace

extern "C" {

fal_status_t fal_window_attention_workspace_bytes(const fal_window_attention_t* shape, size_t* bytes) {
  return guarded([&] {
    const Refusal no = check_shape(shape);
    if (no.why) return fail(no.st, no.why);
    if (!bytes) return fail(FAL_ERR_INVALID_ARG, "NULL bytes");
    int64_t off;
    *bytes = (size_t)window_scratch_bytes(shape->dtype, window_args(shape, nullptr), &off);
    return FAL_OK;
  });
}

fal_status_t fal_window_attention_fwd(const fal_window_attention_t* shape, const void* qkv, const int32_t* lens,
                                      void* out, float* lse, void* stream) {
  return guarded([&] {
    const Refusal no = check_shape(shape);
    if (no.why) return fail(no.st, no.why);
    if (!qkv || !out || !lse) return fail(FAL_ERR_INVALID_ARG, "NULL qkv, out or lse");
    if (!aligned(qkv, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(lens, 4))
      return fail(FAL_ERR_INVALID_ARG, "qkv and out must be 16-byte aligned, lse and lens 4-byte");
    const WindowAttn a = window_args(shape, lens);
    const int64_t es = element_bytes(shape->dtype), M = (int64_t)a.B * a.T;
    const Extent x = rows_of(qkv, M, a.ldq, (int64_t)(a.H + 2 * a.Hkv) * a.hd, es),
                 o = rows_of(out, M, a.ldo, (int64_t)a.H * a.hd, es), l = {lse, M * a.H * 4},
                 n = {lens, (int64_t)a.B * 4};
    if (meets(o, {x, l, n}) || meets(l, {x, n}))
      return fail(FAL_ERR_INVALID_ARG, "out or lse overlaps another argument");
    return launched(window_attention_fwd(shape->dtype == FAL_BF16 ? BF16 : F32, a, qkv, out, lse,
                                         static_cast<hipStream_t>(stream)),
                    "fal_window_attention_fwd");
  });
}

fal_status_t fal_window_attention_bwd(const fal_window_attention_t* shape, const void* qkv, const int32_t* lens,
                                      const void* out, const void* d_out, const float* lse, void* d_qkv,
                                      int64_t ld_d_qkv, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&] {
    const Refusal no = check_shape(shape);
    if (no.why) return fail(no.st, no.why);
    if (!qkv || !out || !d_out || !lse || !d_qkv)
      return fail(FAL_ERR_INVALID_ARG, "NULL qkv, out, d_out, lse or d_qkv");
    if (!aligned(qkv, 16) || !aligned(out, 16) || !aligned(d_out, 16) || !aligned(d_qkv, 16) || !aligned(lse, 4) ||
        !aligned(lens, 4))
      return fail(FAL_ERR_INVALID_ARG, "qkv, out, d_out and d_qkv must be 16-byte aligned, lse and lens 4-byte");
    const int64_t kv = shape->n_kv_head ? shape->n_kv_head : shape->n_head;
    const int64_t width = (shape->n_head + 2 * kv) * shape->head_dim;
    if (ld_d_qkv < width || ld_d_qkv > kMaxStride || ld_d_qkv % (shape->dtype == FAL_BF16 ? 8 : 4))
      return fail(FAL_ERR_INVALID_ARG,
                  "ld_d_qkv must be a multiple of 16 bytes, at least a row and at most 2^40 elements");
    if (!fits(shape, ld_d_qkv))
      return fail(FAL_ERR_INVALID_ARG, "batch * seq_len rows of d_qkv at this stride exceed the address space");
    WindowAttn a = window_args(shape, lens);
    a.lddq = ld_d_qkv;
    int64_t part_off;
    const int64_t need = window_scratch_bytes(shape->dtype, a, &part_off);
    if (!workspace || ws_bytes < (size_t)need || !aligned(workspace, kWorkspaceAlign))
      return fail(FAL_ERR_WORKSPACE, "workspace NULL, too small or not 256-byte aligned");
    const int64_t es = element_bytes(shape->dtype), M = (int64_t)a.B * a.T;
    const int64_t dA = (int64_t)a.H * a.hd;
    const Extent x = rows_of(qkv, M, a.ldq, width, es), dx = rows_of(d_qkv, M, a.lddq, width, es),
                 o = rows_of(out, M, a.ldo, dA, es), g = rows_of(d_out, M, a.lddo, dA, es), l = {lse, M * a.H * 4},
                 n = {lens, (int64_t)a.B * 4}, ws = {workspace, need};
    if (meets(dx, {x, o, g, l, n, ws}) || meets(ws, {x, o, g, l, n}))
      return fail(FAL_ERR_INVALID_ARG, "d_qkv or workspace overlaps another argument");
    float* D = static_cast<float*>(workspace);
    float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + part_off);
    return launched(window_attention_bwd(shape->dtype == FAL_BF16 ? BF16 : F32, a, qkv, out, d_out, lse, D, part,
                                         d_qkv, static_cast<hipStream_t>(stream)),
                    "fal_window_attention_bwd");
  });
}

fal_status_t fal_token_logprobs(const fal_logit_rows_t* rows, const void* logits, const int32_t* targets,
                                const uint8_t* mask, float* logp, float* entropy, void* stream) {
  return guarded([&] {
    const Refusal no = check_rows(rows, false);
    if (no.why) return fail(no.st, no.why);
    if (!logits || !targets || !logp) return fail(FAL_ERR_INVALID_ARG, "NULL logits, targets or logp");
    if (!aligned(logits, element_bytes(rows->dtype)) || !aligned(targets, 4) || !aligned(logp, 4) ||
        !aligned(entropy, 4))
      return fail(FAL_ERR_INVALID_ARG, "logits, targets, logp or entropy misaligned");
    const int64_t N = (int64_t)rows->batch * rows->seq_len;
    const Extent x = rows_of(logits, N, rows->ld_logits, rows->vocab, element_bytes(rows->dtype)),
                 tg = rows_of(targets, rows->batch, rows->ld_targets, rows->seq_len, 4), mk = {mask, N},
                 lp = {logp, 4 * N}, en = {entropy, 4 * N};
    if (meets(lp, {x, tg, mk, en}) || (entropy && meets(en, {x, tg, mk})))
      return fail(FAL_ERR_INVALID_ARG, "logp or entropy overlaps another argument");
    return launched(token_logprobs(rows->dtype == FAL_BF16 ? BF16 : F32, row_args(rows, logits, targets, mask), logp,
                                   entropy, static_cast<hipStream_t>(stream)),
                    "fal_token_logprobs");
  });
}

fal_status_t fal_logit_loss_workspace_bytes(const fal_logit_rows_t* rows, size_t* bytes) {
  return guarded([&] {
    const Refusal no = check_rows(rows, true);
    if (no.why) return fail(no.st, no.why);
    if (!bytes) return fail(FAL_ERR_INVALID_ARG, "NULL bytes");
    *bytes = (size_t)(logit_loss_scratch(rows->batch, rows->seq_len) * 4);
    return FAL_OK;
  });
}

fal_status_t fal_policy_loss(const fal_logit_rows_t* rows, const fal_policy_t* hp, const void* logits,
                             const int32_t* targets, const uint8_t* mask, const float* old_logp,
                             const float* ref_logp, const float* advantages, float* stats, float* logp,
                             void* dlogits, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&] {
    const Refusal no = check_rows(rows, true);
    if (no.why) return fail(no.st, no.why);
    if (const char* why = check_policy(hp)) return fail(FAL_ERR_INVALID_ARG, why);
    if (!logits || !targets || !old_logp || !advantages || !stats || !dlogits)
      return fail(FAL_ERR_INVALID_ARG, "NULL logits, targets, old_logp, advantages, stats or dlogits");
    const int64_t N4 = (int64_t)rows->batch * rows->seq_len * 4;
    const Refusal bad = check_loss(rows, logits, targets, mask, dlogits, workspace, ws_bytes,
                                   {{old_logp, N4}, {ref_logp, N4}, {advantages, N4}}, {{stats, 16}, {logp, N4}});
    if (bad.why) return fail(bad.st, bad.why);
    const PolicyArgs p{old_logp, ref_logp, advantages, hp->clip_low, hp->clip_high, hp->kl_coef, hp->sequence_mean,
                       stats, logp};
    return launched(policy_loss(rows->dtype == FAL_BF16 ? BF16 : F32, row_args(rows, logits, targets, mask), p,
                                dlogits, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)),
                    "fal_policy_loss");
  });
}

fal_status_t fal_preference_loss(const fal_logit_rows_t* rows, const fal_preference_t* hp, const void* logits,
                                 const int32_t* targets, const uint8_t* mask, const float* ref_logp, float* loss,
                                 float* seq_logp, void* dlogits, void* workspace, size_t ws_bytes, void* stream) {
  return guarded([&] {
    const Refusal no = check_rows(rows, true);
    if (no.why) return fail(no.st, no.why);
    if (rows->batch % 2) return fail(FAL_ERR_INVALID_ARG, "preference pairs need an even batch");
    if (const char* why = check_preference(hp)) return fail(FAL_ERR_INVALID_ARG, why);
    if (!logits || !targets || !ref_logp || !loss || !dlogits)
      return fail(FAL_ERR_INVALID_ARG, "NULL logits, targets, ref_logp, loss or dlogits");
    const int64_t B4 = (int64_t)rows->batch * 4;
    const Refusal bad = check_loss(rows, logits, targets, mask, dlogits, workspace, ws_bytes, {{ref_logp, B4}},
                                   {{loss, 4}, {seq_logp, B4}});
    if (bad.why) return fail(bad.st, bad.why);
    const PreferenceArgs p{ref_logp, hp->beta, hp->label_smoothing, hp->ipo, hp->length_mean, loss, seq_logp};
    return launched(preference_loss(rows->dtype == FAL_BF16 ? BF16 : F32, row_args(rows, logits, targets, mask), p,
                                    dlogits, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)),
                    "fal_preference_loss");
  });
}

}  // extern "C"
