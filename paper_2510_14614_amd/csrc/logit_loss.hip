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
// gradient is written from the registers; what they cannot hold of a longer
// row is read twice.  Rows need no alignment: a chunk that a row's edge crosses
// is read and written element by element (two of a row's chunks), columns
// outside the row read as -inf.  Exponentials are exp2 of
// (x - maximum) log2(e) / temperature, sums fp32 within a row; sums over rows
// and sequences are fp64, since a sequence's log-probability is large (hundreds
// of terms) and the losses see a small difference of two.  So that a row's error
// is one of rounding, which such a sum averages out, the exponent's factor has
// two parts and the log-probability is taken in natural units: log2(e) and ln 2
// as fp32 constants would shift every row by 1e-8 of it.
//
// 4551 of 8192 rows of 50257 bf16 counted, after 300 ms of such calls:
// log-probabilities with entropy 80 us (5.7 TB/s of those rows), the policy
// gradient 255 (5.0 TB/s of those rows read and all of the gradient written, the
// rate of a copy); of 5002 counted, the preference loss's statistics 94 (5.3
// TB/s) and its gradient 201 (6.6).
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace fal {

namespace {

constexpr float kLn2 = 0.6931471805599453f;

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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

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
  // ONCE: nothing reads the chunk again, so it need not stay in a cache
  template <bool ONCE>
  __device__ __forceinline__ uint4 load(int c) const {
    if (inside(c)) {
      const u32x4* p = reinterpret_cast<const u32x4*>(base + (int64_t)c * E);
      const u32x4 q = ONCE ? __builtin_nontemporal_load(p) : *p;
      return make_uint4(q.x, q.y, q.z, q.w);
    }
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int col = column(c) + e;
      v[e] = col >= 0 && col < cols ? to_f(base[(int64_t)c * E + e]) : -INFINITY;
    }
    return Chunk<S>::of(v);
  }
  // stores pass by the caches: a gradient is larger than they are, and what
  // they hold of the logits is still to be read
  __device__ __forceinline__ void store(int c, const float (&v)[E]) const {
    if (inside(c)) {
      const uint4 q = Chunk<S>::of(v);
      __builtin_nontemporal_store(u32x4{q.x, q.y, q.z, q.w}, reinterpret_cast<u32x4*>(base + (int64_t)c * E));
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
// With m the maximum and k = log2(e) / temperature: sum of 2^((x - m) k), and
// dot = sum of (x - m) k 2^((x - m) k).
struct Stat {
  float m, sum, dot;
};
// k in two parts, both above 0: one fma more than a product by an fp32 k
struct Log2Scale {
  float hi, lo;
};
__device__ __forceinline__ float scaled(float d, const Log2Scale& k) { return fmaf(d, k.hi, d * k.lo); }

__device__ __forceinline__ void join(Stat& a, const Stat& b, const Log2Scale& k) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) {  // sums of 0, or of NaN
    a.sum += b.sum;
    return;
  }
  const float da = scaled(a.m - m, k), db = scaled(b.m - m, k);  // <= 0, -inf for a side without a column
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
__device__ __forceinline__ void chunk_add(const uint4& u, Stat& st, const Log2Scale& k) {
  constexpr int E = Chunk<S>::E;
  float e2[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float a = scaled(Chunk<S>::at(u, e) - st.m, k);
    e2[e] = __builtin_amdgcn_exp2f(a);
    if (DOT) st.dot = fmaf(fmaxf(a, -200.f), e2[e], st.dot);  // (2^-200 is 0, and -inf times it no term)
  }
#pragma unroll
  for (int w = E / 2; w > 0; w >>= 1)
#pragma unroll
    for (int e = 0; e < w; ++e) e2[e] += e2[e + w];
  st.sum += e2[0];
}

// log x of a sum of exponentials, to one rounding and 2^-25: with x = 2^e m, m
// in [sqrt 1/2, sqrt 2) and s = (m - 1) / (m + 1), the series
// log m = 2 s (1 + s^2/3 + s^4/5 + ...), whose first term left out is 2e-9 of
// it, and e ln 2 in two parts.  (logf came out 1e-7 too small on average.)
__device__ __forceinline__ float log_of_sum(float x) {
  float m = __builtin_amdgcn_frexp_mantf(x), e = (float)__builtin_amdgcn_frexp_expf(x);
  if (m < 0.70710678f) {
    m *= 2.f;
    e -= 1.f;
  }
  const float s = (m - 1.f) / (m + 1.f), z = s * s;
  const float tail = fmaf(z, fmaf(z, fmaf(z, 1.f / 9.f, 1.f / 7.f), 1.f / 5.f), 1.f / 3.f);
  const float log_m = fmaf(2.f * s * z, tail, 2.f * s);
  return fmaf(e, 0.693147182f, fmaf(e, -1.90465432e-9f, log_m));  // the fp32 ln 2, and what it lacks
}

// A chunk of a thread that has no maximum yet holds -inf, which adds nothing, or
// NaN, which no maximum shows.
template <typename S>
__device__ __forceinline__ void chunk_nan(const uint4& u, Stat& st) {
#pragma unroll
  for (int e = 0; e < Chunk<S>::E; ++e)
    if (Chunk<S>::at(u, e) != -INFINITY) st.sum = NAN;
}

// What a row's threads share after the exchange.
struct Shared {
  Stat st;
  float target;  // the target's logit
  int count;     // the sum of the threads' counts
};

// Joins the statistics of the G threads of a row (and sums their counts);
// the thread that holds the target's logit is t == 0.
template <int G>
__device__ __forceinline__ Shared exchange(Stat st, float target, int count, const Log2Scale& k) {
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

constexpr int kStream = 4;  // chunks in flight of a row that is not held

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
    // by more than all else here (an element's own error does not add up: the
    // factor's first part is enough)
    v[e] = -scale * __builtin_amdgcn_exp2f(fmaf(Chunk<S>::at(u, e) - top, k, -log2sum));
  }
  if ((unsigned)(tgt - col0) < (unsigned)E) {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (col0 + e == tgt) v[e] += scale;
  }
  if (col0 + E > V) {
#pragma unroll
    for (int e = 0; e < E; ++e)
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

// the chunks t, t + G, ... of a row's gradient, read from its logits
template <typename S, int G, bool ONCE>
__device__ __forceinline__ void row_grad(const Row<S, const S>& in, const Row<S, S>& out, int t, int end, int tgt,
                                         float k, float top, float log2sum, float scale) {
  const int nc = in.chunks();
  for (int c0 = t; c0 < end; c0 += kStream * G) {
    uint4 u[kStream];
#pragma unroll
    for (int i = 0; i < kStream; ++i) {
      u[i] = make_uint4(0u, 0u, 0u, 0u);
      if (c0 + G * i < nc) u[i] = in.template load<ONCE>(c0 + G * i);
    }
#pragma unroll
    for (int i = 0; i < kStream; ++i) {
      const int c = c0 + G * i;
      if (c < end) grad_chunk<S>(u[i], in.column(c), in.cols, tgt, k, top, log2sum, scale, out, c);
    }
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

// ---- rows of a launch -------------------------------------------------------
// A grid of more than 2^32 threads along x is not launched, which 2^22 rows of
// 1024 are: past kRowGrid workgroups the rest lie along y.
constexpr int64_t kRowGrid = 1 << 21;
template <int G>
constexpr int kRowThreads = G < 256 ? 256 : G;
template <int G>
dim3 row_grid(const LogitRows& r) {
  constexpr int per = kRowThreads<G> / G;
  const int64_t n = ((int64_t)r.B * r.T + per - 1) / per;
  return dim3((unsigned)std::min(n, kRowGrid), (unsigned)((n + kRowGrid - 1) / kRowGrid));
}
// this thread's row; rows from B T on are none
template <int G>
__device__ __forceinline__ int64_t row_of() {
  constexpr int per = kRowThreads<G> / G;
  return ((int64_t)blockIdx.y * kRowGrid + blockIdx.x) * per + threadIdx.x / G;
}

// ---------------------------------------------------------------- policy --
// e^d - d - 1, and e^d - 1, without their cancellation at small d
__device__ __forceinline__ float kl_term(float d, float* em1) {
  float kl;
  if (fabsf(d) > 0.5f) {
    const float e = expf(d);
    *em1 = e - 1.f;
    kl = e < INFINITY ? *em1 - d : e;  // (d = inf: the policy cannot give the token)
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
  // where the clip does not hold the ratio, the smaller product is the ratio's own
  // (compared, not fminf: that drops NaN); a zero advantage adds nothing,
  // whatever the ratio
  o.pg = A == 0.f ? 0.f : -(held ? (A > 0.f ? 1.f + p.high : 1.f - p.low) : ratio) * A;
  o.c = held || A == 0.f ? 0.f : -ratio * A;
  o.kl = 0.f;
  if (p.ref_logp) {
    float em1;
    o.kl = kl_term(p.ref_logp[m] - lp, &em1);
    if (p.kl > 0.f) o.c -= p.kl * em1;  // (0 times an infinite term is no term)
  }
  o.clipped = held ? 1.f : 0.f;
  return o;
}

// Counted rows of each `span` of the N rows' mask: of each sequence, or of
// slices of the batch.
__global__ __launch_bounds__(256) void mask_counts(const uint8_t* mask, int64_t N, int64_t span, int32_t* count) {
  __shared__ int red[4];
  int n = 0;
  const int64_t end = min((blockIdx.x + 1) * span, N);
  for (int64_t i = blockIdx.x * span + threadIdx.x; i < end; i += 256) n += mask[i] != 0;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, FAL_WAVE);
  if (threadIdx.x % FAL_WAVE == 0) red[threadIdx.x / FAL_WAVE] = n;
  __syncthreads();
  if (threadIdx.x == 0) count[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// ------------------------------------------------------------ row kernels --
// STATS: log-probabilities, with what preference_rows needs of each row.
enum Mode { LOGP, LOGP_ENTROPY, STATS, POLICY };
struct RowOut {
  float *logp, *entropy;  // [B, T], each may be NULL
  float *top, *log2sum;   // STATS, [B, T]: a row's largest logit, and log2 of its sum relative to it
  PolicyArgs p;
  const int32_t* count;  // POLICY: counted rows of each sequence, or of `slices` slices of the batch; NULL: each
  int slices;            // row's threads count the mask
  float* terms;          // [3][B * T]
  void* dlogits;
};

// G threads a row, NPT chunks each held in registers; what a longer row has past
// them is read again for its gradient.
template <typename S, int G, int NPT, Mode MODE>
__global__ __launch_bounds__(kRowThreads<G>) void logit_rows(LogitRows r, RowOut o) {
  const int64_t N = (int64_t)r.B * r.T, m = row_of<G>();
  if (m >= N) return;  // all of a row's threads, and barriers are among those only
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
  const Log2Scale k{r.log2_hi, r.log2_lo};
  const float xt = t == 0 ? to_f(l[tgt]) : 0.f;
  int n = 0;  // this thread's share of the counted rows that the mean is over
  if (MODE == POLICY && r.mask) {
    if (!o.count) {
      const uint8_t* mask = o.p.sequence_mean ? r.mask + (int64_t)b * r.T : r.mask;
      const int64_t len = o.p.sequence_mean ? r.T : N;
      for (int64_t i = t; i < len; i += G) n += mask[i] != 0;
    } else if (o.p.sequence_mean) {
      n = t == 0 ? o.count[b] : 0;
    } else {
      for (int i = t; i < o.slices; i += G) n += o.count[i];
    }
  }

  uint4 raw[NPT ? NPT : 1];
  Stat st{-INFINITY, 0.f, 0.f};
  if (NPT) {
#pragma unroll
    for (int i = 0; i < NPT; ++i) {
      const int c = t + G * i;
      if (c < nc) raw[i] = in.template load<true>(c);
    }
#pragma unroll
    for (int i = 0; i < NPT; ++i)
      if (t + G * i < nc) st.m = chunk_max<S>(raw[i], st.m);
    if (st.m != -INFINITY) {
#pragma unroll
      for (int i = 0; i < NPT; ++i)
        if (t + G * i < nc) chunk_add<S, MODE == LOGP_ENTROPY>(raw[i], st, k);
    } else {
#pragma unroll
      for (int i = 0; i < NPT; ++i)
        if (t + G * i < nc) chunk_nan<S>(raw[i], st);
    }
  }
  for (int c0 = t + NPT * G; c0 < nc; c0 += kStream * G) {
    uint4 u[kStream];
#pragma unroll
    for (int i = 0; i < kStream; ++i)
      if (c0 + G * i < nc) u[i] = in.template load<MODE == LOGP || MODE == LOGP_ENTROPY>(c0 + G * i);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kStream; ++i)
      if (c0 + G * i < nc) top = chunk_max<S>(u[i], top);
    if (top > st.m) {
      const Stat none{top, 0.f, 0.f};
      join(st, none, k);
    }
    if (st.m != -INFINITY) {
#pragma unroll
      for (int i = 0; i < kStream; ++i)
        if (c0 + G * i < nc) chunk_add<S, MODE == LOGP_ENTROPY>(u[i], st, k);
    } else {
#pragma unroll
      for (int i = 0; i < kStream; ++i)
        if (c0 + G * i < nc) chunk_nan<S>(u[i], st);
    }
  }
  const Shared sh = exchange<G>(st, xt, n, k);
  const float log2sum = log2f(sh.st.sum);
  const float lse = log_of_sum(sh.st.sum);  // less the maximum
  const float lp = (sh.target - sh.st.m) / r.temp - lse;
  if (t == 0) {
    if (o.logp) o.logp[m] = lp;
    if (MODE == STATS) {
      o.top[m] = sh.st.m;
      o.log2sum[m] = log2sum;
    }
    if (MODE == LOGP_ENTROPY) o.entropy[m] = lse - sh.st.dot / sh.st.sum * kLn2;
  }
  if (MODE != POLICY) return;
  const float rows = r.mask ? (float)sh.count : (float)(o.p.sequence_mean ? (int64_t)r.T : N);
  const float w = 1.f / (o.p.sequence_mean ? rows * (float)r.B : rows);
  const PolicyRow pr = policy_row(o.p, m, lp);
  if (t == 0) {
    o.terms[m] = w * pr.pg;
    o.terms[N + m] = w * pr.kl;
    o.terms[2 * N + m] = w * pr.clipped;
  }
  const float scale = pr.c * w * r.inv_temp;
  const bool same = in.shift == out.shift;
  const int end = same ? out.chunks() : nc;
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);  // columns past V: any value
#pragma unroll
  for (int i = 0; i < NPT; ++i) {
    const int c = t + G * i;
    if (c < end) grad_chunk<S>(c < nc ? raw[i] : none, in.column(c), r.V, tgt, k.hi, sh.st.m, log2sum, scale, out, c);
  }
  row_grad<S, G, false>(in, out, t + NPT * G, end, tgt, k.hi, sh.st.m, log2sum, scale);
  if (!same) zero_tail<S, G>(out, r.V, t);
}

// Sums K doubles over a workgroup of W wavefronts; every thread gets them.
template <int K, int W>
__device__ __forceinline__ void block_totals(double (&v)[K]) {
  __shared__ double red[W][K];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor(v[k], o, FAL_WAVE);
  if (threadIdx.x % FAL_WAVE == 0)
#pragma unroll
    for (int k = 0; k < K; ++k) red[threadIdx.x / FAL_WAVE][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = red[0][k];
#pragma unroll
    for (int w = 1; w < W; ++w) v[k] += red[w][k];
  }
}

__global__ __launch_bounds__(1024) void policy_total(const float* terms, int64_t N, float kl_coef, float* stats) {
  double tot[3] = {0.0, 0.0, 0.0};
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < N; i += 1024)
#pragma unroll
    for (int k = 0; k < 3; ++k) tot[k] += terms[k * N + i];
  block_totals<3, 16>(tot);
  if (threadIdx.x == 0) {
    stats[0] = (float)(kl_coef > 0.f ? tot[0] + (double)kl_coef * tot[1] : tot[0]);
    for (int k = 0; k < 3; ++k) stats[1 + k] = (float)tot[k];
  }
}

// ------------------------------------------------------------ preference --
// A pair's loss and each of its sequences' coefficient of a counted row.
__global__ __launch_bounds__(256) void preference_pairs(LogitRows r, PreferenceArgs p, const float* logp, float* coef,
                                                        double* pair_loss) {
  const int P = r.B / 2, b0 = blockIdx.x;
  double v[4] = {0.0, 0.0, 0.0, 0.0};  // sums and counted rows of both sequences
  for (int t = threadIdx.x; t < r.T; t += 256)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t m = (int64_t)(b0 + k * P) * r.T + t;
      v[k] += logp[m];  // 0 where the row does not count
      v[2 + k] += counted(r, m) ? 1.0 : 0.0;
    }
  block_totals<4, 4>(v);
  double gain[2], share[2];
  for (int k = 0; k < 2; ++k) {
    share[k] = p.length_mean ? 1.0 / fmax(v[2 + k], 1.0) : 1.0;
    gain[k] = v[k] * share[k];
    if (threadIdx.x == 0 && p.seq_logp) p.seq_logp[b0 + k * P] = (float)gain[k];
    gain[k] -= p.ref_logp[b0 + k * P];
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
    loss = (1.0 - sm) * (tail + fmax(-z, 0.0));
    if (sm > 0.0) loss += sm * (tail + fmax(z, 0.0));  // (0 times an infinite margin is no term)
    dh = beta * (sm - 1.0 / (1.0 + exp(z)));  // sigmoid(z) - 1 + sm without its cancellation at large z
  }
  pair_loss[b0] = loss;
  coef[b0] = (float)(dh / P * share[0]);
  coef[b0 + P] = (float)(-dh / P * share[1]);
}

template <typename S, int G>
__global__ __launch_bounds__(kRowThreads<G>) void preference_rows(LogitRows r, const double* pair_loss,
                                                                  const float* coef, const float* top,
                                                                  const float* log2sum, S* dl, float* loss) {
  const int64_t m = row_of<G>();
  if (blockIdx.x == gridDim.x - 1 && blockIdx.y == 0 && threadIdx.x < FAL_WAVE) {  // the mean over pairs
    double s = 0.0;
    for (int i = threadIdx.x; i < r.B / 2; i += FAL_WAVE) s += pair_loss[i];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, FAL_WAVE);
    if (threadIdx.x == 0) *loss = (float)(s / (r.B / 2));
  }
  if (m >= (int64_t)r.B * r.T) return;
  const int t = threadIdx.x % G;
  const Row<S, S> out(dl + m * r.ldd, r.width);
  if (!counted(r, m)) {
    zero_row<S, G>(out, t);
    return;
  }
  const Row<S, const S> in(static_cast<const S*>(r.logits) + m * r.ldl, r.V);
  const int b = (int)(m / r.T), tgt = target_of(r, b, (int)(m % r.T));
  const float k = r.log2_hi, scale = coef[b] * r.inv_temp, mx = top[m], ls = log2sum[m];
  const bool same = in.shift == out.shift;
  const int end = same ? out.chunks() : in.chunks();
  row_grad<S, G, true>(in, out, t, end, tgt, k, mx, ls, scale);
  if (!same) zero_tail<S, G>(out, r.V, t);
}

// ------------------------------------------------------------- launching --
template <typename S, int G, int NPT, Mode MODE>
hipError_t launch(const LogitRows& r, const RowOut& o, hipStream_t s) {
  hipLaunchKernelGGL((logit_rows<S, G, NPT, MODE>), row_grid<G>(r), dim3(kRowThreads<G>), 0, s, r, o);
  return hipGetLastError();
}

// Rows that are only scored are streamed: held or not, they are read once.
// 256 threads keep enough loads in flight and leave a compute unit several
// rows (8192 rows of 50257 bf16, half of them counted, with entropy: 80 us
// against 88 with 512 threads and 128 with 1024).  Of rows that leave the chip
// places, long ones are shortened by more threads, whose exchange then costs
// less than it gives (us with 256, 512 and 1024 threads: 270 rows of 2003
// chunks 5.1, 5.7, 8.9; 512 of 3750 8.3, 8.6, 11.4; 128 of 6283 9.2, 7.3, 8.6;
// 32 of 32064 21.4, 14.2, 12.7).
template <typename S, Mode MODE>
hipError_t scored_rows(const LogitRows& r, const RowOut& o, hipStream_t s) {
  const int n = r.V / Chunk<S>::E;
  if (n <= 512) return launch<S, 64, 0, MODE>(r, o, s);
  if (n <= 4096 || (int64_t)r.B * r.T >= 1024) return launch<S, 256, 0, MODE>(r, o, s);
  if (n <= 16384) return launch<S, 512, 0, MODE>(r, o, s);
  return launch<S, 1024, 0, MODE>(r, o, s);
}

// Rows with a gradient are held by as few threads as can (up to 26 chunks
// each, 13 in a workgroup of 1024, whose registers are half as many): several
// rows then share a compute unit and one's exchange and stores pass under
// another's loads (rows of 50257 bf16 as above: 264 us with 256 x 26, 307 with
// 512 x 13, 295 with 1024 x 7; 50257 fp32: 231 with 1024 x 13, 242 with
// 512 x 26).  The 1024 threads hold 13312 chunks and read the rest of a longer
// row twice (1028 rows of 128001 fp32, half of them counted: 170 us against
// 201 with none held and 185 with 24 chunks a thread).
template <typename S>
hipError_t policy_rows(const LogitRows& r, const RowOut& o, hipStream_t s) {
  constexpr int E = Chunk<S>::E;
  const int n = (r.width + 2 * (E - 1)) / E;  // chunks of a row at any alignment
  if (n <= 64) return launch<S, 64, 1, POLICY>(r, o, s);
  if (n <= 128) return launch<S, 64, 2, POLICY>(r, o, s);
  if (n <= 256) return launch<S, 64, 4, POLICY>(r, o, s);
  if (n <= 512) return launch<S, 64, 8, POLICY>(r, o, s);
  if (n <= 1024) return launch<S, 256, 4, POLICY>(r, o, s);
  if (n <= 2048) return launch<S, 256, 8, POLICY>(r, o, s);
  if (n <= 4096) return launch<S, 256, 16, POLICY>(r, o, s);
  if (n <= 6656) return launch<S, 256, 26, POLICY>(r, o, s);
  return launch<S, 1024, 13, POLICY>(r, o, s);
}

template <typename S, int G>
hipError_t preference_grad(const LogitRows& r, const double* pair_loss, const float* coef, const RowOut& o, void* dl,
                           float* loss, hipStream_t s) {
  hipLaunchKernelGGL((preference_rows<S, G>), row_grid<G>(r), dim3(kRowThreads<G>), 0, s, r, pair_loss, coef, o.top,
                     o.log2sum, static_cast<S*>(dl), loss);
  return hipGetLastError();
}
template <typename S>
hipError_t preference_grad(const LogitRows& r, const double* pair_loss, const float* coef, const RowOut& o, void* dl,
                           float* loss, hipStream_t s) {
  if (r.width <= 512 * Chunk<S>::E) return preference_grad<S, 64>(r, pair_loss, coef, o, dl, loss, s);
  if (r.width <= 2048 * Chunk<S>::E) return preference_grad<S, 256>(r, pair_loss, coef, o, dl, loss, s);
  return preference_grad<S, 1024>(r, pair_loss, coef, o, dl, loss, s);
}

}  // namespace

int64_t logit_loss_scratch(int B, int T) { return 3 * (int64_t)B * T + 4 * (int64_t)B; }

hipError_t token_logprobs(DType dt, const LogitRows& r, float* logp, float* entropy, hipStream_t s) {
  RowOut o{};
  o.logp = logp;
  o.entropy = entropy;
  if (dt == BF16) return entropy ? scored_rows<bf16, LOGP_ENTROPY>(r, o, s) : scored_rows<bf16, LOGP>(r, o, s);
  return entropy ? scored_rows<float, LOGP_ENTROPY>(r, o, s) : scored_rows<float, LOGP>(r, o, s);
}

hipError_t policy_loss(DType dt, const LogitRows& r, const PolicyArgs& p, void* dlogits, float* scratch,
                       hipStream_t s) {
  const int64_t N = (int64_t)r.B * r.T;
  RowOut o{};
  o.logp = p.logp;
  o.p = p;
  o.terms = scratch;
  o.dlogits = dlogits;
  // the rows' threads count the mask themselves while that is a few bytes
  // each, which saves a launch; past that a mean over the batch is counted in
  // slices, as many as a row's threads add up in a few reads and as the scratch
  // has place for, whatever the number of sequences (65536 sequences of 16 rows
  // of 256 fp32, half of them counted: 10.0 ms with a count each, 0.80 in slices)
  const int64_t span = p.sequence_mean ? r.T : N;
  if (r.mask && span > 16 * (r.width > 512 * (dt == BF16 ? 8 : 4) ? 256 : 64)) {
    int32_t* count = reinterpret_cast<int32_t*>(scratch + 3 * N);  // 4 B of them
    o.count = count;
    o.slices = (int)std::min({(int64_t)256, 4 * (int64_t)r.B, (N + 1023) / 1024});
    const int64_t of = p.sequence_mean ? r.T : (N + o.slices - 1) / o.slices;
    hipLaunchKernelGGL(mask_counts, dim3(p.sequence_mean ? r.B : o.slices), dim3(256), 0, s, r.mask, N, of, count);
  }
  const hipError_t e = dt == BF16 ? policy_rows<bf16>(r, o, s) : policy_rows<float>(r, o, s);
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
  hipError_t e = dt == BF16 ? scored_rows<bf16, STATS>(r, o, s) : scored_rows<float, STATS>(r, o, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(preference_pairs, dim3(r.B / 2), dim3(256), 0, s, r, p, o.logp, coef, pair_loss);
  return dt == BF16 ? preference_grad<bf16>(r, pair_loss, coef, o, dlogits, p.loss, s)
                    : preference_grad<float>(r, pair_loss, coef, o, dlogits, p.loss, s);
}

}  // namespace fal
