// Causal attention over a sliding window with a few first keys ("sinks") that
// stay visible: query t of a sequence of n tokens sees the keys
//   S(t) = { j <= t : t - j < W  or  j < sinks },   0 <= t < n,
// scores q . k / sqrt(hd), softmax over S(t), O = P V.  Backward, with
// D = rowsum(dO * O) and P recomputed from the saved log-sum-exp:
//   dS = P * (dO V^T - D),  dQ = dS K / sqrt(hd),  dK = dS^T Q / sqrt(hd),
//   dV = P^T dO,
// a shared key/value head summing over the query heads of its group.  Rows
// past n get O = 0, lse = -inf and zero gradients, whatever they hold.
//
// The work is proportional to T (W + sinks), so every kernel walks only the
// tiles that some row of its block sees; the tiles that an edge of the mask
// crosses test each element, the others none.  As in attention_mfma.hip a
// wavefront owns 32 rows of one sequence dimension (a workgroup 128) and the
// other streams through LDS in tiles of 64; scores sit in accumulator
// registers with the own row in the lane, which is the operand layout of the
// next product, so P and dS never leave registers:
//   bf16  v_mfma_f32_32x32x16_bf16, P and dS rounded to bf16 for their second
//         product (the rounding of every other operand of the matrix cores);
//   fp32  v_mfma_f32_32x32x2_f32, nothing rounded.  A register of the score
//         tile is the B operand of one such product (row 8 (r/4) + 4 g + r%4
//         for lane half g), its A operand one row of the LDS tile per half,
//         so fp32 needs no transposing read.
//
// Keys below `sinks` are seen by every later query: the first key block's
// column is T long where all others are W long.  The queries past the first
// block's own range form chunks (window_attn_sinks): each writes the fp32
// partial dK, dV of the sink keys, and the first key block adds the partials
// in a fixed order before it rounds.
#include <math.h>

#include <algorithm>

#include "attn_tiles.h"
#include "common.h"
#include "kernels.h"

namespace fal {

namespace {

// Kernels whose registers leave one or two wavefronts to a SIMD keep the LDS
// reads of the next four MFMAs in flight.
template <typename S, int HD>
constexpr bool kAhead = HD == 128 && sizeof(S) == 2;

template <int HD>
constexpr int n_tiles() { return HD < 32 ? 1 : HD / 32; }

// ---- 64-row LDS tiles -----------------------------------------------------
// bf16 tiles have the slot order of attn_tiles.h; fp32 rows follow each other
// at a stride of HD + 4 floats (an odd number of 16-byte chunks).
template <int HD>
__device__ __forceinline__ int row_off(const bf16*, int r) { return trow<HD>(r); }
template <int HD>
__device__ __forceinline__ int row_off(const float*, int r) { return (HD + 4) * r; }
template <typename S, int HD>
constexpr int tile_len() { return AT * (HD + 16 / (int)sizeof(S)); }

// Rows row0 .. row0 + 63 of a head, through registers; rows at or past n are
// zeros (a clamped row is read in their place).
template <typename S, int HD>
struct Stage {
  static constexpr int E = 16 / (int)sizeof(S), CH = HD / E, N = (AT * CH + 255) / 256;
  uint4 v[N];
  __device__ __forceinline__ void load(const S* src, int64_t ld, int row0, int n, int tid) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = tid + 256 * k;
      const int row = min(row0 + i / CH, n - 1);
      if (256 * (k + 1) <= AT * CH || i < AT * CH)
        v[k] = *reinterpret_cast<const uint4*>(src + (int64_t)row * ld + E * (i % CH));
    }
  }
  __device__ __forceinline__ void store(S* s, int row0, int n, int tid) {
    if (row0 + AT > n) {  // the sequence's last tile
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const uint32_t keep = row0 + (tid + 256 * k) / CH < n ? ~0u : 0u;
        v[k].x &= keep; v[k].y &= keep; v[k].z &= keep; v[k].w &= keep;
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = tid + 256 * k;
      if (256 * (k + 1) <= AT * CH || i < AT * CH)
        *reinterpret_cast<uint4*>(s + row_off<HD>(s, i / CH) + E * (i % CH)) = v[k];
    }
  }
};

// The window's mask over a 32x32 score tile whose tile rows are keys: row `off`
// (from the lane half's first) is hidden from the lane's query if it lies
// after it, or before its window and past the sinks.  No branches: the three
// comparisons join in the scalar unit.
struct KeyMask {
  int last, before, sink;
  __device__ __forceinline__ KeyMask(const WindowAttn& a, int kb, int g, int tq, int n) {
    const int key0 = kb + 4 * g;
    last = min(tq, n - 1) - key0;
    before = tq - a.window - key0;
    sink = a.sinks - key0;
  }
  __device__ __forceinline__ bool hides(int r) const {
    const int off = acc_row(r, 0);
    return (bool)((off > last) | ((off <= before) & (off >= sink)));
  }
};
// The same where tile rows are queries and the lane has the key.
struct QueryMask {
  int first, past;
  __device__ __forceinline__ QueryMask(const WindowAttn& a, int qs, int g, int key) {
    const int q0 = qs + 4 * g;
    first = key - q0;
    past = key < a.sinks ? 1 << 30 : key + a.window - q0;
  }
  __device__ __forceinline__ bool hides(int r) const {
    const int off = acc_row(r, 0);
    return (bool)((off < first) | (off >= past));
  }
};

// ---- operands -------------------------------------------------------------
// The lane's own row (row c of the wavefront's 32) as the B operand of the
// products that contract over head_dim.
template <typename S, int HD>
struct Own;
template <int HD>
struct Own<bf16, HD> {
  static constexpr int N = HD / 16, E = 8;
  bf16x8v f[N];
  __device__ __forceinline__ void load(const bf16* src, int64_t ld, int row, int n, int g) {
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = frag_global<HD>(src, ld, row, n, k, g);
  }
  __device__ __forceinline__ float dot(const Own& o) const {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(static_cast<float>(f[k][j]), static_cast<float>(o.f[k][j]), s);
    return s;
  }
};
typedef float f32x4v __attribute__((ext_vector_type(4)));
template <int HD>
struct Own<float, HD> {
  static constexpr int N = HD / 8, E = 4;
  f32x4v f[N];
  __device__ __forceinline__ void load(const float* src, int64_t ld, int row, int n, int g) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      f[k] = f32x4v{0.f, 0.f, 0.f, 0.f};
      if (row < n) f[k] = *reinterpret_cast<const f32x4v*>(src + (int64_t)row * ld + 8 * k + 4 * g);
    }
  }
  __device__ __forceinline__ float dot(const Own& o) const {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = fmaf(f[k][j], o.f[k][j], s);
    return s;
  }
};

// acc[tile row][own row] += sum over dims of tile row (rowbase + .) * own row
template <int HD>
__device__ __forceinline__ void dot_rows(const bf16* s, int rowbase, int c, int g, const Own<bf16, HD>& o, f32x16v& acc) {
#pragma unroll
  for (int k = 0; k < HD / 16; ++k) acc = mfma32(frag_rows<HD>(s, rowbase, c, k, g), o.f[k], acc);
}
template <int HD>
__device__ __forceinline__ void dot_rows(const float* s, int rowbase, int c, int g, const Own<float, HD>& o, f32x16v& acc) {
  const float* row = s + (HD + 4) * (rowbase + c) + 4 * g;
#pragma unroll
  for (int k = 0; k < HD / 8; ++k) {
    const f32x4v a = *reinterpret_cast<const f32x4v*>(row + 8 * k);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], o.f[k][j], acc, 0, 0, 0);
  }
}

// acc[t][dim 32 t + .][own row] += sum over the 32 tile rows from rowbase of
// tile[row][dim] * p[row][own row].  head_dim 16: dims 16..31 repeat 0..15
// and are not stored.
template <int HD>
__device__ __forceinline__ void add_rows(const bf16* s, int rowbase, int lane, const f32x16v& p,
                                         f32x16v (&acc)[n_tiles<HD>()]) {
  const bf16x8v p0 = pack8(p, 0), p1 = pack8(p, 8);
#pragma unroll
  for (int t = 0; t < n_tiles<HD>(); ++t) {
    acc[t] = mfma32(frag_tr<HD>(s, rowbase, 32 * t, lane), p0, acc[t]);
    acc[t] = mfma32(frag_tr<HD>(s, rowbase + 16, 32 * t, lane), p1, acc[t]);
  }
}
template <int HD>
__device__ __forceinline__ void add_rows(const float* s, int rowbase, int lane, const f32x16v& p,
                                         f32x16v (&acc)[n_tiles<HD>()]) {
  const int g = lane >> 5, c = HD < 32 ? lane & 15 : lane & 31;
  const float* col = s + (HD + 4) * (rowbase + 4 * g) + c;
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int t = 0; t < n_tiles<HD>(); ++t)
      acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(col[(HD + 4) * acc_row(r, 0) + 32 * t], p[r], acc[t], 0, 0, 0);
}

// Four consecutive dims of the lane's row, rounded to the storage type.
__device__ __forceinline__ void put4(bf16* p, float a, float b, float c, float d) {
  bf16x4v o;
  o[0] = static_cast<bf16>(a); o[1] = static_cast<bf16>(b); o[2] = static_cast<bf16>(c); o[3] = static_cast<bf16>(d);
  *reinterpret_cast<bf16x4v*>(p) = o;
}
__device__ __forceinline__ void put4(float* p, float a, float b, float c, float d) {
  *reinterpret_cast<f32x4v*>(p) = f32x4v{a, b, c, d};
}
// row[dim] = acc * mul, or zeros
template <typename S, int HD>
__device__ __forceinline__ void put_row(S* row, int g, const f32x16v (&acc)[n_tiles<HD>()], float mul, bool live) {
#pragma unroll
  for (int t = 0; t < n_tiles<HD>(); ++t)
#pragma unroll
    for (int r = 0; r < (HD < 32 ? 2 : 4); ++r) {
      S* p = row + 32 * t + 8 * r + 4 * g;
      if (live) put4(p, acc[t][4 * r] * mul, acc[t][4 * r + 1] * mul, acc[t][4 * r + 2] * mul, acc[t][4 * r + 3] * mul);
      else put4(p, 0.f, 0.f, 0.f, 0.f);
    }
}

template <int HD>
__device__ __forceinline__ void zero_acc(f32x16v (&acc)[n_tiles<HD>()]) {
#pragma unroll
  for (int t = 0; t < n_tiles<HD>(); ++t) acc[t] = zero16();
}

__device__ __forceinline__ int length_of(const WindowAttn& a, int b) {
  return a.lens ? min(max(a.lens[b], 0), a.T) : a.T;
}

// Key tiles of a block of 128 queries from qb on: `sink` tiles from key 0,
// then the window's tiles from `first` (a multiple of AT) up to `end`.
struct KeyTiles {
  int sink, first, end, count;
  __device__ __forceinline__ KeyTiles(const WindowAttn& a, int qb, int n) {
    end = min(n, qb + 128);
    first = max(0, qb - a.window + 1) / AT * AT;
    sink = (min(a.sinks, first) + AT - 1) / AT;
    count = sink + (end - first + AT - 1) / AT;
  }
  __device__ __forceinline__ int at(int i) const { return i < sink ? AT * i : first + AT * (i - sink); }
};

}  // namespace

// ------------------------------------------------------------- forward --
template <typename S, int HD>
__global__ __launch_bounds__(256, 2) void window_attn_fwd(WindowAttn a, const S* qkv, S* O, float* lse) {
  constexpr int NT = n_tiles<HD>();
  __shared__ __attribute__((aligned(16))) S sK[tile_len<S, HD>()];
  __shared__ __attribute__((aligned(16))) S sV[tile_len<S, HD>()];
  const int h = blockIdx.x, b = blockIdx.y, qb = 128 * blockIdx.z;
  const int kvh = h / (a.H / a.Hkv);
  const S* Qg = qkv + (int64_t)b * a.T * a.ldq + h * HD;
  const S* Kg = qkv + (int64_t)b * a.T * a.ldq + (a.H + kvh) * HD;
  const S* Vg = Kg + a.Hkv * HD;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, c = lane & 31;
  const int q0 = qb + wave * 32, tq = q0 + c;
  const int n = length_of(a, b);
  const float sl2 = kLog2e / sqrtf((float)HD);

  f32x16v acc[NT];
  zero_acc<HD>(acc);
  // Online softmax in log2 units against a reference maximum that moves only
  // when a row's maximum exceeds it by kSlack: acc and lsum share mref, so
  // O = acc / lsum does not depend on where it sits.  A row may see nothing
  // of the first tiles: mref stays -inf until it does.
  constexpr float kSlack = 8.f;
  float mref = -INFINITY, lsum = 0.f;
  if (qb < n) {
    Own<S, HD> q;
    q.load(Qg, a.ldq, tq, n, g);
    const KeyTiles kt(a, qb, n);
    Stage<S, HD> rk, rv;
    rk.load(Kg, a.ldq, kt.at(0), n, tid);
    rv.load(Vg, a.ldq, kt.at(0), n, tid);
    for (int i = 0; i < kt.count; ++i) {
      const int k0 = kt.at(i);
      __syncthreads();
      rk.store(sK, k0, n, tid);
      rv.store(sV, k0, n, tid);
      __syncthreads();
      if (i + 1 < kt.count) {
        rk.load(Kg, a.ldq, kt.at(i + 1), n, tid);
        rv.load(Vg, a.ldq, kt.at(i + 1), n, tid);
      }
#pragma unroll
      for (int sub = 0; sub < AT / 32; ++sub) {
        const int kb = k0 + 32 * sub;
        if (kb > q0 + 31 || kb >= n) break;
        if (kb >= a.sinks && q0 - (kb + 31) >= a.window) continue;  // before the window of every row
        f32x16v s = zero16();
        dot_rows<HD>(sK, 32 * sub, c, g, q, s);
        if (kb + 31 > q0 || kb + 31 >= n || q0 + 31 - kb >= a.window) {
          const KeyMask mask(a, kb, g, tq, n);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = mask.hides(r) ? -INFINITY : s[r];
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * sl2;
        if (__any(mx > mref + kSlack)) {
          if (mx > mref + kSlack) {
            const float alpha = __builtin_amdgcn_exp2f(mref - mx);
            lsum *= alpha;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[t][r] *= alpha;
            mref = mx;
          }
        }
        const float base = mref == -INFINITY ? 0.f : mref;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[r], sl2, -base));
          s[r] = p;
          lsum += p;
        }
        add_rows<HD>(sV, 32 * sub, lane, s, acc);
      }
    }
  }
  const float l = lsum + __shfl_xor(lsum, 32, 64);
  if (tq < a.T) {
    put_row<S, HD>(O + ((int64_t)b * a.T + tq) * a.ldo + h * HD, g, acc, 1.f / l, tq < n);
    if (g == 0)
      lse[((int64_t)b * a.H + h) * a.T + tq] = tq < n ? (mref + log2f(l)) * 0.6931471805599453f : -INFINITY;
  }
}

// ----------------------------------------------------------- backward: dQ --
// Also writes D = rowsum(dO * O) for the kernels that follow.
template <typename S, int HD>
__global__ __launch_bounds__(256, 2) void window_attn_dq(WindowAttn a, const S* qkv, const S* O, const S* dO,
                                                         const float* lse, float* Dvec, S* dqkv) {
  constexpr int NT = n_tiles<HD>();
  __shared__ __attribute__((aligned(16))) S sK[tile_len<S, HD>()];
  __shared__ __attribute__((aligned(16))) S sV[tile_len<S, HD>()];
  const int h = blockIdx.x, b = blockIdx.y, qb = 128 * blockIdx.z;
  const int kvh = h / (a.H / a.Hkv);
  const int64_t row0 = (int64_t)b * a.T;
  const S* Kg = qkv + row0 * a.ldq + (a.H + kvh) * HD;
  const S* Vg = Kg + a.Hkv * HD;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, c = lane & 31;
  const int q0 = qb + wave * 32, tq = q0 + c;
  const int n = length_of(a, b);
  const float sl2 = kLog2e / sqrtf((float)HD);

  f32x16v dq[NT];
  zero_acc<HD>(dq);
  if (qb < n) {
    Own<S, HD> q, d;
    q.load(qkv + row0 * a.ldq + h * HD, a.ldq, tq, n, g);
    d.load(dO + row0 * a.lddo + h * HD, a.lddo, tq, n, g);
    float D;
    {
      Own<S, HD> o;
      o.load(O + row0 * a.ldo + h * HD, a.ldo, tq, n, g);
      D = d.dot(o);
    }
    D += __shfl_xor(D, 32, 64);
    const int64_t stat = ((int64_t)b * a.H + h) * a.T + tq;
    const float L2 = tq < n ? lse[stat] * kLog2e : 0.f;
    if (g == 0 && tq < n) Dvec[stat] = D;
    const KeyTiles kt(a, qb, n);
    Stage<S, HD> rk, rv;
    rk.load(Kg, a.ldq, kt.at(0), n, tid);
    rv.load(Vg, a.ldq, kt.at(0), n, tid);
    for (int i = 0; i < kt.count; ++i) {
      const int k0 = kt.at(i);
      __syncthreads();
      rk.store(sK, k0, n, tid);
      rv.store(sV, k0, n, tid);
      __syncthreads();
      if (i + 1 < kt.count) {
        rk.load(Kg, a.ldq, kt.at(i + 1), n, tid);
        rv.load(Vg, a.ldq, kt.at(i + 1), n, tid);
      }
#pragma unroll
      for (int sub = 0; sub < AT / 32; ++sub) {
        const int kb = k0 + 32 * sub;
        if (kb > q0 + 31 || kb >= n) break;
        if (kb >= a.sinks && q0 - (kb + 31) >= a.window) continue;
        f32x16v s = zero16(), dp = zero16();
        dot_rows<HD>(sK, 32 * sub, c, g, q, s);
        dot_rows<HD>(sV, 32 * sub, c, g, d, dp);
        if (kAhead<S, HD>) lds_ahead<HD / 8, 1, 4>();
        if (kb + 31 > q0 || kb + 31 >= n || q0 + 31 - kb >= a.window) {
          const KeyMask mask(a, kb, g, tq, n);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = mask.hides(r) ? -INFINITY : s[r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[r], sl2, -L2));
          dp[r] = p * (dp[r] - D);
        }
        if (kAhead<S, HD>) __builtin_amdgcn_sched_barrier(0);
        add_rows<HD>(sK, 32 * sub, lane, dp, dq);
        if (kAhead<S, HD>) lds_ahead<HD / 16, 2, 4>();
      }
    }
  }
  if (tq < a.T)
    put_row<S, HD>(dqkv + (row0 + tq) * a.lddq + h * HD, g, dq, 1.f / sqrtf((float)HD), tq < n);
}

// ------------------------------------------- backward: dK, dV of the sinks --
// Queries from `far` on see of the first key block only the sink keys.  One
// workgroup takes a chunk of them for one query head and 32 sink keys, its
// wavefronts alternating over 32-query rows; the four sums are joined in LDS
// and written as fp32 partials [b][h][chunk][dK, dV][sinks][HD].
template <typename S, int HD>
__global__ __launch_bounds__(256, HD == 128 ? 1 : 2) void window_attn_sinks(WindowAttn a, const S* qkv, const S* dO,
                                                                            const float* lse, const float* Dvec,
                                                                            int far, int chunk, int nchunk,
                                                                            float* part) {
  constexpr int NT = n_tiles<HD>();
  __shared__ __attribute__((aligned(16))) S sQ[tile_len<S, HD>()];
  __shared__ __attribute__((aligned(16))) S sdO[tile_len<S, HD>()];
  __shared__ float sL[AT], sD[AT];
  const int h = blockIdx.x, b = blockIdx.y, ck = blockIdx.z % nchunk, kw = 32 * (blockIdx.z / nchunk);
  const int kvh = h / (a.H / a.Hkv);
  const int64_t row0 = (int64_t)b * a.T;
  const S* Qg = qkv + row0 * a.ldq + h * HD;
  const S* Kg = qkv + row0 * a.ldq + (a.H + kvh) * HD;
  const S* dOg = dO + row0 * a.lddo + h * HD;
  const float* Lg = lse + ((int64_t)b * a.H + h) * a.T;
  const float* Dg = Dvec + ((int64_t)b * a.H + h) * a.T;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, c = lane & 31;
  const int n = length_of(a, b), key = kw + c;
  const int qbeg = far + ck * chunk, qend = min(n, qbeg + chunk);
  const float sl2 = kLog2e / sqrtf((float)HD);

  f32x16v dk[NT], dv[NT];
  zero_acc<HD>(dk);
  zero_acc<HD>(dv);
  if (qbeg < qend) {
    Own<S, HD> k, v;
    k.load(Kg, a.ldq, key, n, g);
    v.load(Kg + a.Hkv * HD, a.ldq, key, n, g);
    Stage<S, HD> rq, ro;
    rq.load(Qg, a.ldq, qbeg, qend, tid);
    ro.load(dOg, a.lddo, qbeg, qend, tid);
    for (int q0 = qbeg; q0 < qend; q0 += AT) {
      __syncthreads();
      rq.store(sQ, q0, qend, tid);
      ro.store(sdO, q0, qend, tid);
      if (tid < AT) {
        const int tq = q0 + tid;
        sL[tid] = tq < qend ? Lg[tq] * kLog2e : 0.f;
        sD[tid] = tq < qend ? Dg[tq] : 0.f;
      }
      __syncthreads();
      if (q0 + AT < qend) {
        rq.load(Qg, a.ldq, q0 + AT, qend, tid);
        ro.load(dOg, a.lddo, q0 + AT, qend, tid);
      }
      // two wavefronts share a tile, the next tile's two the other pair
      const int sub = wave & 1;
      if ((((q0 - qbeg) / AT) & 1) != (wave >> 1)) continue;
      f32x16v s = zero16(), dp = zero16();
      dot_rows<HD>(sQ, 32 * sub, c, g, k, s);
      dot_rows<HD>(sdO, 32 * sub, c, g, v, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int qr = 32 * sub + acc_row(r, g);
        const float p = __builtin_amdgcn_exp2f(fmaf(s[r], sl2, -sL[qr]));
        s[r] = p;
        dp[r] = p * (dp[r] - sD[qr]);
      }
      add_rows<HD>(sdO, 32 * sub, lane, s, dv);
      add_rows<HD>(sQ, 32 * sub, lane, dp, dk);
    }
  }
  // join the wavefronts' sums in order, one at a time through LDS
  __shared__ __attribute__((aligned(16))) float sum[2][32][HD];
  for (int w = 0; w < 4; ++w) {
    __syncthreads();
    if (wave != w) continue;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < (HD < 32 ? 8 : 16); ++r) {
        const int dim = 32 * t + acc_row(r, g);
        sum[0][c][dim] = (w ? sum[0][c][dim] : 0.f) + dk[t][r];
        sum[1][c][dim] = (w ? sum[1][c][dim] : 0.f) + dv[t][r];
      }
  }
  __syncthreads();
  float* out = part + ((((int64_t)b * a.H + h) * nchunk + ck) * 2) * a.sinks * HD;
  const int rows = min(32, a.sinks - kw);
  for (int i = tid; i < rows * HD; i += 256) {
    out[kw * HD + i] = sum[0][i / HD][i % HD];
    out[(a.sinks + kw) * HD + i] = sum[1][i / HD][i % HD];
  }
}

// ------------------------------------------------------- backward: dK, dV --
template <typename S, int HD>
__global__ __launch_bounds__(256, HD == 128 ? 1 : 2) void window_attn_dkdv(WindowAttn a, const S* qkv, const S* dO,
                                                                           const float* lse, const float* Dvec,
                                                                           const float* part, int nchunk, S* dqkv) {
  constexpr int NT = n_tiles<HD>();
  __shared__ __attribute__((aligned(16))) S sQ[tile_len<S, HD>()];
  __shared__ __attribute__((aligned(16))) S sdO[tile_len<S, HD>()];
  __shared__ float sL[AT], sD[AT];
  const int kvh = blockIdx.x, b = blockIdx.y, kb0 = 128 * blockIdx.z, grp = a.H / a.Hkv;
  const int64_t row0 = (int64_t)b * a.T;
  const S* Kg = qkv + row0 * a.ldq + (a.H + kvh) * HD;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 5, c = lane & 31;
  const int kw = kb0 + wave * 32, key = kw + c;
  const int n = length_of(a, b);
  const float sl2 = kLog2e / sqrtf((float)HD);

  f32x16v dk[NT], dv[NT];
  zero_acc<HD>(dk);
  zero_acc<HD>(dv);
  if (kb0 < n) {
    Own<S, HD> k, v;
    k.load(Kg, a.ldq, key, n, g);
    v.load(Kg + a.Hkv * HD, a.ldq, key, n, g);
    // query tiles kb0 + 64 i that some key of the block has in its window
    const int nq = (min(n - kb0, 127 + a.window) + AT - 1) / AT;
    const int nit = grp * nq;
    Stage<S, HD> rq, ro;
    rq.load(qkv + row0 * a.ldq + kvh * grp * HD, a.ldq, kb0, n, tid);
    ro.load(dO + row0 * a.lddo + kvh * grp * HD, a.lddo, kb0, n, tid);
    int h = kvh * grp, qi = 0;
    for (int it = 0; it < nit; ++it) {
      const int q0 = kb0 + AT * qi;
      __syncthreads();
      rq.store(sQ, q0, n, tid);
      ro.store(sdO, q0, n, tid);
      if (tid < AT) {
        const int tq = q0 + tid;
        const int64_t stat = ((int64_t)b * a.H + h) * a.T + tq;
        sL[tid] = tq < n ? lse[stat] * kLog2e : 0.f;
        sD[tid] = tq < n ? Dvec[stat] : 0.f;
      }
      __syncthreads();
      if (++qi == nq) {
        qi = 0;
        ++h;
      }
      if (it + 1 < nit) {
        rq.load(qkv + row0 * a.ldq + h * HD, a.ldq, kb0 + AT * qi, n, tid);
        ro.load(dO + row0 * a.lddo + h * HD, a.lddo, kb0 + AT * qi, n, tid);
      }
#pragma unroll
      for (int sub = 0; sub < AT / 32; ++sub) {
        const int qs = q0 + 32 * sub;
        if (qs + 31 < kw || qs >= n) continue;                      // before this wavefront's keys, or past the end
        if (kw >= a.sinks && qs - (kw + 31) >= a.window) continue;  // past the window of all its keys
        f32x16v s = zero16(), dp = zero16();
        dot_rows<HD>(sQ, 32 * sub, c, g, k, s);
        dot_rows<HD>(sdO, 32 * sub, c, g, v, dp);
        if (kAhead<S, HD>) lds_ahead<HD / 8, 1, 4>();
        // queries past n have zero Q, dO, L and D: they add nothing
        if (qs < kw + 32 || qs + 31 - kw >= a.window) {
          const QueryMask mask(a, qs, g, key);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = mask.hides(r) ? -INFINITY : s[r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int qr = 32 * sub + acc_row(r, g);
          const float p = __builtin_amdgcn_exp2f(fmaf(s[r], sl2, -sL[qr]));
          s[r] = p;
          dp[r] = p * (dp[r] - sD[qr]);
        }
        if (kAhead<S, HD>) __builtin_amdgcn_sched_barrier(0);
        add_rows<HD>(sdO, 32 * sub, lane, s, dv);
        add_rows<HD>(sQ, 32 * sub, lane, dp, dk);
        if (kAhead<S, HD>) lds_ahead<HD / 8, 2, 4>();
      }
    }
    if (part && key < a.sinks) {
      for (int hh = kvh * grp; hh < (kvh + 1) * grp; ++hh)
        for (int ck = 0; ck < nchunk; ++ck) {
          const float* pk = part + ((((int64_t)b * a.H + hh) * nchunk + ck) * 2 * a.sinks + key) * HD;
          const float* pv = pk + a.sinks * HD;
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < (HD < 32 ? 8 : 16); ++r) {
              dk[t][r] += pk[32 * t + acc_row(r, g)];
              dv[t][r] += pv[32 * t + acc_row(r, g)];
            }
        }
    }
  }
  if (key < a.T) {
    S* row = dqkv + (row0 + key) * a.lddq + (a.H + kvh) * HD;
    put_row<S, HD>(row, g, dk, 1.f / sqrtf((float)HD), key < n);
    put_row<S, HD>(row + a.Hkv * HD, g, dv, 1.f, key < n);
  }
}

// ------------------------------------------------------------- launching --
namespace {

// Queries from here on reach the first key block through its sink keys only
// (the end of the last tile its own range walks).
int far_start(const WindowAttn& a) { return (int)(((int64_t)a.window + 127 + AT - 1) / AT * AT); }

// Chunks of the far queries: enough workgroups to fill the chip twice over,
// and no chunk under 128 queries.
int sink_chunks(const WindowAttn& a) {
  const int64_t far = a.sinks > 0 ? (int64_t)a.T - far_start(a) : 0;
  if (far <= 0) return 0;
  const int64_t want = (512 + (int64_t)a.B * a.H - 1) / ((int64_t)a.B * a.H);
  return (int)std::max<int64_t>(1, std::min<int64_t>(want, (far + 127) / 128));
}

template <typename S, int HD>
hipError_t fwd(const WindowAttn& a, const void* qkv, void* O, float* lse, hipStream_t s) {
  hipLaunchKernelGGL((window_attn_fwd<S, HD>), dim3(a.H, a.B, cdiv(a.T, 128)), dim3(256), 0, s, a,
                     static_cast<const S*>(qkv), static_cast<S*>(O), lse);
  return hipGetLastError();
}

template <typename S, int HD>
hipError_t bwd(const WindowAttn& a, const void* qkv, const void* O, const void* dO, const float* lse, float* Dvec,
               float* part, void* dqkv, hipStream_t s) {
  const S *x = static_cast<const S*>(qkv), *g = static_cast<const S*>(dO);
  S* dx = static_cast<S*>(dqkv);
  hipLaunchKernelGGL((window_attn_dq<S, HD>), dim3(a.H, a.B, cdiv(a.T, 128)), dim3(256), 0, s, a, x,
                     static_cast<const S*>(O), g, lse, Dvec, dx);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int nc = sink_chunks(a);
  if (nc > 0) {
    const int far = far_start(a), chunk = cdiv(cdiv(a.T - far, nc), AT) * AT;
    hipLaunchKernelGGL((window_attn_sinks<S, HD>), dim3(a.H, a.B, nc * cdiv(a.sinks, 32)), dim3(256), 0, s, a, x, g,
                       lse, Dvec, far, chunk, nc, part);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((window_attn_dkdv<S, HD>), dim3(a.Hkv, a.B, cdiv(a.T, 128)), dim3(256), 0, s, a, x, g, lse, Dvec,
                     nc > 0 ? part : nullptr, nc, dx);
  return hipGetLastError();
}

}  // namespace

int64_t window_attention_scratch(const WindowAttn& a) {
  return (int64_t)a.B * a.H * sink_chunks(a) * 2 * a.sinks * a.hd;
}

#define FAL_BY_HEAD(S, CALL)                                  \
  switch (a.hd) {                                             \
    case 16: return CALL(S, 16);                              \
    case 32: return CALL(S, 32);                              \
    case 64: return CALL(S, 64);                              \
    case 128: return CALL(S, 128);                            \
    default: return hipErrorInvalidValue;                     \
  }

hipError_t window_attention_fwd(DType dt, const WindowAttn& a, const void* qkv, void* O, float* lse, hipStream_t s) {
#define FAL_FWD(S, HD) (fwd<S, HD>(a, qkv, O, lse, s))
  if (dt == BF16) FAL_BY_HEAD(bf16, FAL_FWD)
  FAL_BY_HEAD(float, FAL_FWD)
#undef FAL_FWD
}

hipError_t window_attention_bwd(DType dt, const WindowAttn& a, const void* qkv, const void* O, const void* dO,
                                const float* lse, float* Dvec, float* part, void* dqkv, hipStream_t s) {
#define FAL_BWD(S, HD) (bwd<S, HD>(a, qkv, O, dO, lse, Dvec, part, dqkv, s))
  if (dt == BF16) FAL_BY_HEAD(bf16, FAL_BWD)
  FAL_BY_HEAD(float, FAL_BWD)
#undef FAL_BWD
}
#undef FAL_BY_HEAD

}  // namespace fal
