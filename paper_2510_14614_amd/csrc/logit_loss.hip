// Log-probabilities of given tokens under rows of logits, and the two losses
// built on them with their gradients: the clipped policy loss with a KL term
// and the preference loss.  For a row x (logits / temperature) with target y
//   logp = x_y - lse(x),   d logp / d logits_v = (1[v = y] - p_v) / temperature
// with p = softmax(x), so a row's gradient is one coefficient
// c = d loss / d logp times (onehot - p) / temperature.  Everything is fp32
// but the sums over rows and sequences, which are fp64: a sequence's
// log-probability is large (hundreds of terms) and the losses see a small
// difference of two.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace fal {

namespace {

constexpr int kRowThreads = 256;

__device__ __forceinline__ bool counted(const LogitRows& r, int64_t m) { return !r.mask || r.mask[m] != 0; }
__device__ __forceinline__ int target_of(const LogitRows& r, int b, int t) {
  return min(max(r.targets[(int64_t)b * r.ldt + t], 0), r.V - 1);
}

template <typename T>
__device__ __forceinline__ T block_total(T v, T* red) {
  __syncthreads();
  red[threadIdx.x] = v;
  __syncthreads();
  for (int w = blockDim.x / 2; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
    __syncthreads();
  }
  return red[0];
}

// Row statistics: maximum, sum of exp(x - maximum), and sum of x exp(x - maximum).
struct RowStat {
  float top, sum, dot;
};
template <typename S>
__device__ RowStat row_stat(const S* l, int V, float inv_temp, float* red) {
  float top = -INFINITY;
  for (int v = threadIdx.x; v < V; v += kRowThreads) top = fmaxf(top, to_f(l[v]) * inv_temp);
  __syncthreads();
  red[threadIdx.x] = top;
  __syncthreads();
  for (int w = kRowThreads / 2; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) red[threadIdx.x] = fmaxf(red[threadIdx.x], red[threadIdx.x + w]);
    __syncthreads();
  }
  RowStat st;
  st.top = red[0];
  float sum = 0.f, dot = 0.f;
  for (int v = threadIdx.x; v < V; v += kRowThreads) {
    const float x = to_f(l[v]) * inv_temp, e = expf(x - st.top);
    sum += e;
    if (e > 0.f) dot = fmaf(x - st.top, e, dot);  // a column of -inf adds nothing
  }
  st.sum = block_total(sum, red);
  st.dot = block_total(dot, red);
  return st;
}

// drow = c (onehot - p) inv_temp over the row's width, zeros past V
template <typename S>
__device__ void row_gradient(const S* l, S* drow, const LogitRows& r, int tgt, const RowStat& st, float c) {
  const float k = c * r.inv_temp, norm = k / st.sum;
  for (int v = threadIdx.x; v < r.width; v += kRowThreads) {
    float d = 0.f;
    if (v < r.V) d = (v == tgt ? k : 0.f) - norm * expf(to_f(l[v]) * r.inv_temp - st.top);
    drow[v] = from_f<S>(d);
  }
}
template <typename S>
__device__ void row_zero(S* drow, int width) {
  for (int v = threadIdx.x; v < width; v += kRowThreads) drow[v] = from_f<S>(0.f);
}

// Counted rows of each sequence.
__global__ __launch_bounds__(kRowThreads) void mask_counts(const uint8_t* mask, int T, int32_t* count) {
  __shared__ int red[kRowThreads];
  int n = 0;
  for (int t = threadIdx.x; t < T; t += kRowThreads) n += !mask || mask[(int64_t)blockIdx.x * T + t] != 0;
  n = block_total(n, red);
  if (threadIdx.x == 0) count[blockIdx.x] = n;
}

template <typename S>
__global__ __launch_bounds__(kRowThreads) void logprob_rows(LogitRows r, float* logp, float* entropy) {
  __shared__ float red[kRowThreads];
  const int64_t m = blockIdx.x;
  const int b = (int)(m / r.T), t = (int)(m % r.T);
  float lp = 0.f, en = 0.f;
  if (counted(r, m)) {
    const S* l = static_cast<const S*>(r.logits) + m * r.ldl;
    const RowStat st = row_stat(l, r.V, r.inv_temp, red);
    const float ls = logf(st.sum);
    lp = to_f(l[target_of(r, b, t)]) * r.inv_temp - st.top - ls;
    en = ls - st.dot / st.sum;  // lse - sum p x
  }
  if (threadIdx.x == 0) {
    logp[m] = lp;
    if (entropy) entropy[m] = en;
  }
}

// ---------------------------------------------------------------- policy --
// e^d - d - 1 without its cancellation at small d
__device__ __forceinline__ float kl_term(float d) {
  if (fabsf(d) > 0.5f) return expf(d) - d - 1.f;
  // d^2 (1/2 + d/6 + d^2/24 + ...), the next term under 2^-24 of the first
  float s = 1.f / 362880.f;
  s = fmaf(s, d, 1.f / 40320.f);
  s = fmaf(s, d, 1.f / 5040.f);
  s = fmaf(s, d, 1.f / 720.f);
  s = fmaf(s, d, 1.f / 120.f);
  s = fmaf(s, d, 1.f / 24.f);
  s = fmaf(s, d, 1.f / 6.f);
  s = fmaf(s, d, 0.5f);
  return d * d * s;
}

template <typename S>
__global__ __launch_bounds__(kRowThreads) void policy_rows(LogitRows r, PolicyArgs p, const int32_t* count, S* dl,
                                                           float* terms) {
  __shared__ float red[kRowThreads];
  __shared__ int ired[kRowThreads];
  const int64_t m = blockIdx.x, N = (int64_t)r.B * r.T;
  const int b = (int)(m / r.T), t = (int)(m % r.T);
  S* drow = dl + m * r.ldd;
  if (!counted(r, m)) {
    row_zero(drow, r.width);
    if (threadIdx.x == 0) {
      if (p.logp) p.logp[m] = 0.f;
      for (int k = 0; k < 3; ++k) terms[k * N + m] = 0.f;
    }
    return;
  }
  float w;
  if (p.sequence_mean) {
    w = 1.f / ((float)r.B * (float)count[b]);
  } else {
    int n = 0;
    for (int k = threadIdx.x; k < r.B; k += kRowThreads) n += count[k];
    w = 1.f / (float)block_total(n, ired);
  }
  const S* l = static_cast<const S*>(r.logits) + m * r.ldl;
  const int tgt = target_of(r, b, t);
  const float xt = to_f(l[tgt]) * r.inv_temp;
  const RowStat st = row_stat(l, r.V, r.inv_temp, red);
  const float lp = xt - st.top - logf(st.sum);
  const float A = p.adv[m], ratio = expf(lp - p.old_logp[m]);
  const bool clipped = (A > 0.f && ratio > 1.f + p.high) || (A < 0.f && ratio < 1.f - p.low);
  const float held = fminf(fmaxf(ratio, 1.f - p.low), 1.f + p.high);
  // a zero advantage adds nothing, whatever the ratio
  const float pg = A == 0.f ? 0.f : -fminf(ratio * A, held * A);
  float c = clipped || A == 0.f ? 0.f : -ratio * A;
  float kl = 0.f;
  if (p.ref_logp) {
    const float d = p.ref_logp[m] - lp;
    kl = kl_term(d);
    c -= p.kl * expm1f(d);
  }
  __syncthreads();  // dl may be the logits: every read of the target's is done
  row_gradient(l, drow, r, tgt, st, c * w);
  if (threadIdx.x == 0) {
    if (p.logp) p.logp[m] = lp;
    terms[m] = w * pg;
    terms[N + m] = w * kl;
    terms[2 * N + m] = clipped ? w : 0.f;
  }
}

__global__ __launch_bounds__(1024) void policy_total(const float* terms, int64_t N, float kl_coef, float* stats) {
  __shared__ double red[1024];
  double tot[3];
  for (int k = 0; k < 3; ++k) {
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < N; i += 1024) s += terms[k * N + i];
    tot[k] = block_total(s, red);
  }
  if (threadIdx.x == 0) {
    stats[0] = (float)(tot[0] + (double)kl_coef * tot[1]);
    for (int k = 0; k < 3; ++k) stats[1 + k] = (float)tot[k];
  }
}

// ------------------------------------------------------------ preference --
// A pair's loss and each of its sequences' coefficient of a counted row.
__global__ __launch_bounds__(kRowThreads) void preference_pairs(LogitRows r, PreferenceArgs p, const float* logp,
                                                                float* coef, double* pair_loss) {
  __shared__ double red[kRowThreads];
  __shared__ int ired[kRowThreads];
  const int P = r.B / 2, b0 = blockIdx.x;
  double gain[2];
  double share[2];
  for (int k = 0; k < 2; ++k) {
    const int64_t m0 = (int64_t)(b0 + k * P) * r.T;
    double s = 0.0;
    int n = 0;
    for (int t = threadIdx.x; t < r.T; t += kRowThreads)
      if (counted(r, m0 + t)) {
        s += logp[m0 + t];
        ++n;
      }
    s = block_total(s, red);
    n = block_total(n, ired);
    share[k] = p.length_mean ? 1.0 / max(n, 1) : 1.0;
    s *= share[k];
    if (threadIdx.x == 0 && p.seq_logp) p.seq_logp[b0 + k * P] = (float)s;
    gain[k] = s - p.ref_logp[b0 + k * P];
  }
  if (threadIdx.x != 0) return;
  const double h = gain[0] - gain[1], beta = p.beta, sm = p.smoothing;
  double loss, dh;
  if (p.ipo) {
    const double u = h - 0.5 / beta;
    loss = u * u;
    dh = 2.0 * u;
  } else {
    const double z = beta * h, tail = log1p(exp(-fabs(z)));
    loss = (1.0 - sm) * (tail + fmax(-z, 0.0)) + sm * (tail + fmax(z, 0.0));
    dh = beta * (1.0 / (1.0 + exp(-z)) - (1.0 - sm));
  }
  pair_loss[b0] = loss;
  coef[b0] = (float)(dh / P * share[0]);
  coef[b0 + P] = (float)(-dh / P * share[1]);
}

template <typename S>
__global__ __launch_bounds__(kRowThreads) void preference_rows(LogitRows r, const float* coef, S* dl) {
  __shared__ float red[kRowThreads];
  const int64_t m = blockIdx.x;
  const int b = (int)(m / r.T), t = (int)(m % r.T);
  S* drow = dl + m * r.ldd;
  if (!counted(r, m)) {
    row_zero(drow, r.width);
    return;
  }
  const S* l = static_cast<const S*>(r.logits) + m * r.ldl;
  const RowStat st = row_stat(l, r.V, r.inv_temp, red);
  row_gradient(l, drow, r, target_of(r, b, t), st, coef[b]);
}

__global__ __launch_bounds__(kRowThreads) void preference_total(const double* pair_loss, int P, float* loss) {
  __shared__ double red[kRowThreads];
  double s = 0.0;
  for (int i = threadIdx.x; i < P; i += kRowThreads) s += pair_loss[i];
  s = block_total(s, red);
  if (threadIdx.x == 0) *loss = (float)(s / P);
}

}  // namespace

int64_t logit_loss_scratch(int B, int T) { return 3 * (int64_t)B * T + 4 * (int64_t)B; }

hipError_t token_logprobs(DType dt, const LogitRows& r, float* logp, float* entropy, hipStream_t s) {
  const dim3 grid((unsigned)((int64_t)r.B * r.T)), block(kRowThreads);
  if (dt == BF16)
    hipLaunchKernelGGL(logprob_rows<bf16>, grid, block, 0, s, r, logp, entropy);
  else
    hipLaunchKernelGGL(logprob_rows<float>, grid, block, 0, s, r, logp, entropy);
  return hipGetLastError();
}

hipError_t policy_loss(DType dt, const LogitRows& r, const PolicyArgs& p, void* dlogits, float* scratch,
                       hipStream_t s) {
  const int64_t N = (int64_t)r.B * r.T;
  int32_t* count = reinterpret_cast<int32_t*>(scratch + 3 * N);
  hipLaunchKernelGGL(mask_counts, dim3(r.B), dim3(kRowThreads), 0, s, r.mask, r.T, count);
  const dim3 grid((unsigned)N), block(kRowThreads);
  if (dt == BF16)
    hipLaunchKernelGGL(policy_rows<bf16>, grid, block, 0, s, r, p, count, static_cast<bf16*>(dlogits), scratch);
  else
    hipLaunchKernelGGL(policy_rows<float>, grid, block, 0, s, r, p, count, static_cast<float*>(dlogits), scratch);
  hipLaunchKernelGGL(policy_total, dim3(1), dim3(1024), 0, s, scratch, N, p.kl, p.stats);
  return hipGetLastError();
}

hipError_t preference_loss(DType dt, const LogitRows& r, const PreferenceArgs& p, void* dlogits, float* scratch,
                           hipStream_t s) {
  const int64_t N = (int64_t)r.B * r.T;
  double* pair_loss = reinterpret_cast<double*>(scratch);  // [B / 2]
  float* coef = scratch + r.B;                             // [B]
  float* logp = coef + r.B;                                // [B, T]
  hipError_t e = token_logprobs(dt, r, logp, nullptr, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(preference_pairs, dim3(r.B / 2), dim3(kRowThreads), 0, s, r, p, logp, coef, pair_loss);
  const dim3 grid((unsigned)N), block(kRowThreads);
  if (dt == BF16)
    hipLaunchKernelGGL(preference_rows<bf16>, grid, block, 0, s, r, coef, static_cast<bf16*>(dlogits));
  else
    hipLaunchKernelGGL(preference_rows<float>, grid, block, 0, s, r, coef, static_cast<float*>(dlogits));
  hipLaunchKernelGGL(preference_total, dim3(1), dim3(kRowThreads), 0, s, pair_loss, r.B / 2, p.loss);
  return hipGetLastError();
}

}  // namespace fal
