// Log-probabilities of given tokens under rows of logits, and the two losses
// built on them with their gradients: the clipped policy loss with a KL term
// and the preference loss.  For a row x (logits / temperature) with target y
//   logp = x_y - lse(x),   d logp / d logits_v = (1[v = y] - p_v) / temperature
// with p = softmax(x), so a row's gradient is one coefficient
// c = d loss / d logp times (onehot - p) / temperature.
//
// All of it is bound by HBM: a row is read in 16-byte chunks and, while the
// registers of its threads hold it, read once: each thread reduces its chunks
// to (maximum, sum of exponentials), one exchange joins the threads, and the
// gradient is written from the registers.  A longer row is read twice.  Rows
// need no alignment: a chunk that a row's edge crosses is read and written
// element by element (two of a row's chunks), columns outside the row read as
// -inf.  Exponentials are exp2 of (x - maximum) log2(e) / temperature, sums
// fp32 within a row; sums over rows and sequences are fp64, since a sequence's
// log-probability is large (hundreds of terms) and the losses see a small
// difference of two.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace fal {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// ---- chunks of a row --------------------------------------------------------
template <typename S>
struct Chunk;
template <>
struct Chunk<bf16> {
  static constexpr int E = 8;
  static __device__ __forceinline__ float at(const uint4& u, int e) {
    const uint32_t w = e < 2 ? u.x : e < 4 ? u.y : e < 6 ? u.z : u.w;
    return __uint_as_float((e & 1) ? w & 0xFFFF0000u : w << 16);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    return (uint32_t)__builtin_bit_cast(uint16_t, from_f<bf16>(a)) |
           ((uint32_t)__builtin_bit_cast(uint16_t, from_f<bf16>(b)) << 16);
  }
  static __device__ __forceinline__ uint4 of(const float (&v)[8]) {
    return make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]), pack(v[6], v[7]));
  }
};
template <>
struct Chunk<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ float at(const uint4& u, int e) {
    return __uint_as_float(e == 0 ? u.x : e == 1 ? u.y : e == 2 ? u.z : u.w);
  }
  static __device__ __forceinline__ uint4 of(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};

// A row of `cols` elements seen through aligned chunks: element 0 is element
// `shift` of chunk 0.
template <typename S, typename P>
struct Row {
  static constexpr int E = Chunk<S>::E;
  P* base;
  int shift, cols;
  __device__ __forceinline__ Row(P* row, int cols_) : cols(cols_) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(row);
    shift = (int)(a % 16) / (int)sizeof(S);
    base = reinterpret_cast<P*>(a - a % 16);
  }
  __device__ __forceinline__ int chunks() const { return (shift + cols + E - 1) / E; }
  __device__ __forceinline__ int column(int c) const { return c * E - shift; }
  __device__ __forceinline__ bool inside(int c) const { return column(c) >= 0 && column(c) + E <= cols; }
  __device__ __forceinline__ uint4 load(int c) const {
    if (inside(c)) return *reinterpret_cast<const uint4*>(base + (int64_t)c * E);
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int col = column(c) + e;
      v[e] = col >= 0 && col < cols ? to_f(base[(int64_t)c * E + e]) : -INFINITY;
    }
    return Chunk<S>::of(v);
  }
  __device__ __forceinline__ void store(int c, const float (&v)[E]) const {
    if (inside(c)) {
      *reinterpret_cast<uint4*>(base + (int64_t)c * E) = Chunk<S>::of(v);
      return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int col = column(c) + e;
      if (col >= 0 && col < cols) base[(int64_t)c * E + e] = from_f<S>(v[e]);
    }
  }
};

// ---- a row's statistics -----------------------------------------------------
// With m the maximum, in units of log2: top = m k (k = log2(e) / temperature),
// sum of 2^(x k - top), and dot = sum of (x k - top) 2^(x k - top).
struct Stat {
  float m, sum, dot;
};
__device__ __forceinline__ void join(Stat& a, const Stat& b, float k) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return;
  const float da = (a.m - m) * k, db = (b.m - m) * k;  // <= 0, -inf for a side without a column
  const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
  const float la = fa > 0.f ? fmaf(da, a.sum, a.dot) * fa : 0.f, lb = fb > 0.f ? fmaf(db, b.sum, b.dot) * fb : 0.f;
  a.sum = a.sum * fa + b.sum * fb;
  a.dot = la + lb;
  a.m = m;
}

template <typename S>
__device__ __forceinline__ float chunk_max(const uint4& u, float m) {
#pragma unroll
  for (int e = 0; e < Chunk<S>::E; ++e) m = fmaxf(m, Chunk<S>::at(u, e));
  return m;
}
// adds a chunk to sums relative to st.m (not -inf)
template <typename S, bool DOT>
__device__ __forceinline__ void chunk_add(const uint4& u, Stat& st, float k) {
  constexpr int E = Chunk<S>::E;
  float e2[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float a = (Chunk<S>::at(u, e) - st.m) * k;
    e2[e] = __builtin_amdgcn_exp2f(a);
    if (DOT && e2[e] > 0.f) st.dot = fmaf(a, e2[e], st.dot);
  }
#pragma unroll
  for (int w = E / 2; w > 0; w >>= 1)
#pragma unroll
    for (int e = 0; e < w; ++e) e2[e] += e2[e + w];
  st.sum += e2[0];
}

// What a row's threads share after the exchange.
struct Shared {
  Stat st;
  float target;  // the target's logit
  int count;     // counted rows of the whole batch (policy, mean over rows)
};

// Joins the statistics of the G threads of a row (and sums their counts);
// the thread that holds the target's logit is t == 0.
template <int G>
__device__ __forceinline__ Shared exchange(Stat st, float target, int count, float k) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    const Stat b{__shfl_xor(st.m, o, FAL_WAVE), __shfl_xor(st.sum, o, FAL_WAVE), __shfl_xor(st.dot, o, FAL_WAVE)};
    join(st, b, k);
    count += __shfl_xor(count, o, FAL_WAVE);
  }
  if (G == FAL_WAVE) return {st, __shfl(target, 0, FAL_WAVE), count};
  constexpr int W = G / FAL_WAVE;
  __shared__ Stat rs[W];
  __shared__ int rn[W];
  __shared__ float rt;
  const int w = threadIdx.x / FAL_WAVE;
  if (threadIdx.x % FAL_WAVE == 0) {
    rs[w] = st;
    rn[w] = count;
  }
  if (threadIdx.x == 0) rt = target;
  __syncthreads();
  Shared sh{rs[0], rt, rn[0]};
#pragma unroll
  for (int i = 1; i < W; ++i) {
    join(sh.st, rs[i], k);
    sh.count += rn[i];
  }
  return sh;
}

__device__ __forceinline__ bool counted(const LogitRows& r, int64_t m) { return !r.mask || r.mask[m] != 0; }
__device__ __forceinline__ int target_of(const LogitRows& r, int b, int t) {
  return min(max(r.targets[(int64_t)b * r.ldt + t], 0), r.V - 1);
}

// ---- a row's gradient -------------------------------------------------------
// out chunk c from logits chunk c of the same shift: zero past V.
template <typename S>
__device__ __forceinline__ void grad_chunk(const uint4& u, int col0, int V, int tgt, float k, float top, float log2sum,
                                           float scale, const Row<S, S>& out, int c) {
  constexpr int E = Chunk<S>::E;
  float v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    // p from x - maximum, not x - lse: the log-sum-exp alone, rounded, is off
    // by more than all else here
    v[e] = -scale * __builtin_amdgcn_exp2f(fmaf(Chunk<S>::at(u, e) - top, k, -log2sum));
    if (col0 + e == tgt) v[e] += scale;
    if (col0 + e >= V) v[e] = 0.f;
  }
  if (out.shift == c * E - col0) {
    out.store(c, v);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (col0 + e >= 0 && col0 + e < V) out.base[out.shift + col0 + e] = from_f<S>(v[e]);
  }
}

template <typename S, int G>
__device__ __forceinline__ void zero_row(const Row<S, S>& out, int t) {
  const float z[Chunk<S>::E] = {};
  for (int c = t; c < out.chunks(); c += G) out.store(c, z);
}
// columns from V on of a gradient row whose shift differs from its logits'
template <typename S, int G>
__device__ __forceinline__ void zero_tail(const Row<S, S>& out, int V, int t) {
  for (int col = V + t; col < out.cols; col += G) out.base[out.shift + col] = from_f<S>(0.f);
}

// ---------------------------------------------------------------- policy --
// e^d - d - 1, and e^d - 1, without their cancellation at small d
__device__ __forceinline__ float kl_term(float d, float* em1) {
  float kl;
  if (fabsf(d) > 0.5f) {
    const float e = expf(d);
    *em1 = e - 1.f;
    kl = *em1 - d;
  } else {
    // d^2 (1/2 + d/6 + d^2/24 + ...): the first term left out is under
    // 2^-24 of the sum
    float s = 1.f / 362880.f;
    s = fmaf(s, d, 1.f / 40320.f);
    s = fmaf(s, d, 1.f / 5040.f);
    s = fmaf(s, d, 1.f / 720.f);
    s = fmaf(s, d, 1.f / 120.f);
    s = fmaf(s, d, 1.f / 24.f);
    s = fmaf(s, d, 1.f / 6.f);
    s = fmaf(s, d, 0.5f);
    kl = d * d * s;
    *em1 = kl + d;
  }
  return kl;
}

struct PolicyRow {
  float c, pg, kl, clipped;
};
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& p, int64_t m, float lp) {
  PolicyRow o;
  const float A = p.adv[m], ratio = expf(lp - p.old_logp[m]);
  const bool held = (A > 0.f && ratio > 1.f + p.high) || (A < 0.f && ratio < 1.f - p.low);
  const float clip = fminf(fmaxf(ratio, 1.f - p.low), 1.f + p.high);
  // a zero advantage adds nothing, whatever the ratio
  o.pg = A == 0.f ? 0.f : -fminf(ratio * A, clip * A);
  o.c = held || A == 0.f ? 0.f : -ratio * A;
  o.kl = 0.f;
  if (p.ref_logp) {
    float em1;
    o.kl = kl_term(p.ref_logp[m] - lp, &em1);
    o.c -= p.kl * em1;
  }
  o.clipped = held ? 1.f : 0.f;
  return o;
}

// Counted rows of each sequence.
__global__ __launch_bounds__(256) void mask_counts(const uint8_t* mask, int T, int32_t* count) {
  __shared__ int red[4];
  int n = 0;
  for (int t = threadIdx.x; t < T; t += 256) n += mask[(int64_t)blockIdx.x * T + t] != 0;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, FAL_WAVE);
  if (threadIdx.x % FAL_WAVE == 0) red[threadIdx.x / FAL_WAVE] = n;
  __syncthreads();
  if (threadIdx.x == 0) count[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// ------------------------------------------------------------ row kernels --
enum Mode { LOGP, LOGP_ENTROPY, POLICY };
struct RowOut {
  float *logp, *entropy;  // [B, T], each may be NULL
  float *top, *log2sum;   // [B, T] or NULL: a row's largest logit, and log2 of its sum relative to it
  PolicyArgs p;
  const int32_t* count;  // counted rows of each sequence (NULL: T)
  float* terms;          // [3][B * T]
  void* dlogits;
};

// G threads a row, NPT chunks each held in registers; NPT = 0: the row is
// read again for its gradient.
template <typename S, int G, int NPT, Mode MODE>
__global__ __launch_bounds__(G < 256 ? 256 : G) void logit_rows(LogitRows r, RowOut o) {
  constexpr int RPW = (G < 256 ? 256 : G) / G;
  const int64_t N = (int64_t)r.B * r.T, m = (int64_t)blockIdx.x * RPW + threadIdx.x / G;
  if (RPW > 1 && m >= N) return;  // a whole wavefront: no barrier follows
  const int t = threadIdx.x % G;
  const bool on = counted(r, m);
  const Row<S, S> out(MODE == POLICY ? static_cast<S*>(o.dlogits) + m * r.ldd : nullptr, r.width);
  if (!on) {
    if (MODE == POLICY) zero_row<S, G>(out, t);
    if (t == 0) {
      if (o.logp) o.logp[m] = 0.f;
      if (o.entropy) o.entropy[m] = 0.f;
      if (MODE == POLICY)
        for (int k = 0; k < 3; ++k) o.terms[k * N + m] = 0.f;
    }
    return;  // the whole row's threads
  }
  const S* l = static_cast<const S*>(r.logits) + m * r.ldl;
  const Row<S, const S> in(l, r.V);
  const int nc = in.chunks(), b = (int)(m / r.T), tgt = target_of(r, b, (int)(m % r.T));
  const float k = r.inv_temp * kLog2e;
  const float xt = t == 0 ? to_f(l[tgt]) : 0.f;
  int n = 0;
  if (MODE == POLICY && o.count && !o.p.sequence_mean)
    for (int i = t; i < r.B; i += G) n += o.count[i];

  uint4 raw[NPT ? NPT : 1];
  Stat st{-INFINITY, 0.f, 0.f};
  if (NPT) {
#pragma unroll
    for (int i = 0; i < NPT; ++i) {
      const int c = t + G * i;
      if (c < nc) raw[i] = in.load(c);
    }
#pragma unroll
    for (int i = 0; i < NPT; ++i)
      if (t + G * i < nc) st.m = chunk_max<S>(raw[i], st.m);
    if (st.m != -INFINITY) {
#pragma unroll
      for (int i = 0; i < NPT; ++i)
        if (t + G * i < nc) chunk_add<S, MODE == LOGP_ENTROPY>(raw[i], st, k);
    }
  } else {
    for (int c = t; c < nc; c += G) {
      const uint4 u = in.load(c);
      const float top = chunk_max<S>(u, -INFINITY);
      if (top > st.m) {
        const Stat none{top, 0.f, 0.f};
        join(st, none, k);
      }
      if (st.m != -INFINITY) chunk_add<S, MODE == LOGP_ENTROPY>(u, st, k);
    }
  }
  const Shared sh = exchange<G>(st, xt, n, k);
  const float log2sum = log2f(sh.st.sum);
  const float lp = ((sh.target - sh.st.m) * k - log2sum) * kLn2;
  if (t == 0) {
    if (o.logp) o.logp[m] = lp;
    if (MODE == LOGP && o.top) {
      o.top[m] = sh.st.m;
      o.log2sum[m] = log2sum;
    }
    if (MODE == LOGP_ENTROPY) o.entropy[m] = (log2sum - sh.st.dot / sh.st.sum) * kLn2;
  }
  if (MODE != POLICY) return;
  const float rows = o.p.sequence_mean ? (float)r.B * (float)(o.count ? o.count[b] : r.T)
                                       : (float)(o.count ? (int64_t)sh.count : N);
  const float w = 1.f / rows;
  const PolicyRow pr = policy_row(o.p, m, lp);
  if (t == 0) {
    o.terms[m] = w * pr.pg;
    o.terms[N + m] = w * pr.kl;
    o.terms[2 * N + m] = w * pr.clipped;
  }
  const float scale = pr.c * w * r.inv_temp;
  const bool same = in.shift == out.shift;
  const int end = same ? out.chunks() : nc;
  const uint4 none = [] {
    float v[Chunk<S>::E];
#pragma unroll
    for (int e = 0; e < Chunk<S>::E; ++e) v[e] = -INFINITY;
    return Chunk<S>::of(v);
  }();
  if (NPT) {
#pragma unroll
    for (int i = 0; i < NPT; ++i) {
      const int c = t + G * i;
      if (c < end) grad_chunk<S>(c < nc ? raw[i] : none, in.column(c), r.V, tgt, k, sh.st.m, log2sum, scale, out, c);
    }
  } else {
    for (int c = t; c < end; c += G)
      grad_chunk<S>(c < nc ? in.load(c) : none, in.column(c), r.V, tgt, k, sh.st.m, log2sum, scale, out, c);
  }
  if (!same) zero_tail<S, G>(out, r.V, t);
}

__device__ __forceinline__ double block_total(double v, double* red) {
  __syncthreads();
  red[threadIdx.x] = v;
  __syncthreads();
  for (int w = blockDim.x / 2; w > 0; w >>= 1) {
    if ((int)threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
    __syncthreads();
  }
  return red[0];
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
__global__ __launch_bounds__(256) void preference_pairs(LogitRows r, PreferenceArgs p, const float* logp, float* coef,
                                                        double* pair_loss) {
  __shared__ double red[256];
  const int P = r.B / 2, b0 = blockIdx.x;
  double gain[2], share[2];
  for (int k = 0; k < 2; ++k) {
    const int64_t m0 = (int64_t)(b0 + k * P) * r.T;
    double s = 0.0, n = 0.0;
    for (int t = threadIdx.x; t < r.T; t += 256)
      if (counted(r, m0 + t)) {
        s += logp[m0 + t];
        n += 1.0;
      }
    s = block_total(s, red);
    n = block_total(n, red);
    share[k] = p.length_mean ? 1.0 / fmax(n, 1.0) : 1.0;
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

template <typename S, int G>
__global__ __launch_bounds__(G < 256 ? 256 : G) void preference_rows(LogitRows r, const float* coef, const float* top,
                                                                     const float* log2sum, S* dl) {
  constexpr int RPW = (G < 256 ? 256 : G) / G;
  const int64_t N = (int64_t)r.B * r.T, m = (int64_t)blockIdx.x * RPW + threadIdx.x / G;
  if (RPW > 1 && m >= N) return;
  const int t = threadIdx.x % G;
  const Row<S, S> out(dl + m * r.ldd, r.width);
  if (!counted(r, m)) {
    zero_row<S, G>(out, t);
    return;
  }
  const Row<S, const S> in(static_cast<const S*>(r.logits) + m * r.ldl, r.V);
  const int b = (int)(m / r.T), tgt = target_of(r, b, (int)(m % r.T)), nc = in.chunks();
  const float k = r.inv_temp * kLog2e, scale = coef[b] * r.inv_temp, mx = top[m], ls = log2sum[m];
  const bool same = in.shift == out.shift;
  const int end = same ? out.chunks() : nc;
  for (int c = t; c < end; c += G) {
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (c < nc) u = in.load(c);
    grad_chunk<S>(u, in.column(c), r.V, tgt, k, mx, ls, scale, out, c);
  }
  if (!same) zero_tail<S, G>(out, r.V, t);
}

__global__ __launch_bounds__(256) void preference_total(const double* pair_loss, int P, float* loss) {
  __shared__ double red[256];
  double s = 0.0;
  for (int i = threadIdx.x; i < P; i += 256) s += pair_loss[i];
  s = block_total(s, red);
  if (threadIdx.x == 0) *loss = (float)(s / P);
}

// ------------------------------------------------------------- launching --
template <typename S, int G, int NPT, Mode MODE>
hipError_t launch(const LogitRows& r, const RowOut& o, hipStream_t s) {
  constexpr int WG = G < 256 ? 256 : G;
  const int64_t N = (int64_t)r.B * r.T;
  hipLaunchKernelGGL((logit_rows<S, G, NPT, MODE>), dim3((unsigned)((N + WG / G - 1) / (WG / G))), dim3(WG), 0, s, r, o);
  return hipGetLastError();
}

// The threads of a row: enough that none holds more than eight chunks, up to
// a workgroup of 1024 that holds sixteen each; longer rows are read twice.
template <typename S, Mode MODE>
hipError_t rows(const LogitRows& r, const RowOut& o, hipStream_t s) {
  constexpr int E = Chunk<S>::E;
  const int cols = MODE == POLICY ? r.width : r.V;
  const int n = (cols + 2 * (E - 1)) / E;  // chunks of a row at any alignment
  if (n <= 64) return launch<S, 64, 1, MODE>(r, o, s);
  if (n <= 128) return launch<S, 64, 2, MODE>(r, o, s);
  if (n <= 256) return launch<S, 64, 4, MODE>(r, o, s);
  if (n <= 512) return launch<S, 64, 8, MODE>(r, o, s);
  if (n <= 1024) return launch<S, 256, 4, MODE>(r, o, s);
  if (n <= 2048) return launch<S, 256, 8, MODE>(r, o, s);
  if (n <= 4096) return launch<S, 1024, 4, MODE>(r, o, s);
  if (n <= 7168) return launch<S, 1024, 7, MODE>(r, o, s);
  if (n <= 13312) return launch<S, 1024, 13, MODE>(r, o, s);
  if (n <= 16384) return launch<S, 1024, 16, MODE>(r, o, s);
  return launch<S, 1024, 0, MODE>(r, o, s);
}

template <typename S>
hipError_t preference_grad(const LogitRows& r, const float* coef, const RowOut& o, S* dl, hipStream_t s) {
  const int64_t N = (int64_t)r.B * r.T;
  if (r.width <= 8192)
    hipLaunchKernelGGL((preference_rows<S, 64>), dim3((unsigned)((N + 3) / 4)), dim3(256), 0, s, r, coef, o.top,
                       o.log2sum, dl);
  else
    hipLaunchKernelGGL((preference_rows<S, 1024>), dim3((unsigned)N), dim3(1024), 0, s, r, coef, o.top,
                       o.log2sum, dl);
  return hipGetLastError();
}

}  // namespace

int64_t logit_loss_scratch(int B, int T) { return 3 * (int64_t)B * T + 4 * (int64_t)B; }

hipError_t token_logprobs(DType dt, const LogitRows& r, float* logp, float* entropy, hipStream_t s) {
  RowOut o{};
  o.logp = logp;
  o.entropy = entropy;
  if (dt == BF16) return entropy ? rows<bf16, LOGP_ENTROPY>(r, o, s) : rows<bf16, LOGP>(r, o, s);
  return entropy ? rows<float, LOGP_ENTROPY>(r, o, s) : rows<float, LOGP>(r, o, s);
}

hipError_t policy_loss(DType dt, const LogitRows& r, const PolicyArgs& p, void* dlogits, float* scratch,
                       hipStream_t s) {
  const int64_t N = (int64_t)r.B * r.T;
  RowOut o{};
  o.logp = p.logp;
  o.p = p;
  o.terms = scratch;
  o.dlogits = dlogits;
  if (r.mask) {
    int32_t* count = reinterpret_cast<int32_t*>(scratch + 3 * N);
    hipLaunchKernelGGL(mask_counts, dim3(r.B), dim3(256), 0, s, r.mask, r.T, count);
    o.count = count;
  }
  const hipError_t e = dt == BF16 ? rows<bf16, POLICY>(r, o, s) : rows<float, POLICY>(r, o, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(policy_total, dim3(1), dim3(1024), 0, s, scratch, N, p.kl, p.stats);
  return hipGetLastError();
}

hipError_t preference_loss(DType dt, const LogitRows& r, const PreferenceArgs& p, void* dlogits, float* scratch,
                           hipStream_t s) {
  const int64_t N = (int64_t)r.B * r.T;
  double* pair_loss = reinterpret_cast<double*>(scratch);  // [B / 2]
  float* coef = scratch + r.B;                             // [B]
  RowOut o{};
  o.logp = coef + r.B;  // [B, T], as the two that follow
  o.top = o.logp + N;
  o.log2sum = o.top + N;
  hipError_t e = dt == BF16 ? rows<bf16, LOGP>(r, o, s) : rows<float, LOGP>(r, o, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(preference_pairs, dim3(r.B / 2), dim3(256), 0, s, r, p, o.logp, coef, pair_loss);
  e = dt == BF16 ? preference_grad(r, coef, o, static_cast<bf16*>(dlogits), s)
                 : preference_grad(r, coef, o, static_cast<float*>(dlogits), s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(preference_total, dim3(1), dim3(256), 0, s, pair_loss, r.B / 2, p.loss);
  return hipGetLastError();
}

}  // namespace fal
