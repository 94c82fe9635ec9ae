// Matrices made orthogonal by Newton-Schulz products, and the update that takes
// its direction from them.
//
//   X_0 = U / |U|_F;   A = X X^T,  B = a I + b A + c A^2,  X <- B X   (steps times)
//
// on the smaller side p of a p x q matrix (a taller one is transposed on the way
// in and out), so every singular value s goes through the same odd polynomial
// a s + b s^3 + c s^5.  The update round it:
//   m <- beta m + g,  U = g + beta m  (or m),  W <- W (1 - lr decay) - lr scale X.
//
// Bound by the matrix cores.  The polynomial multiplies small singular values by
// a each step, 485 fold over five at the usual coefficients, and with them every
// rounding of X; one 16-bit operand is too coarse for that, and fp32 MFMA run at
// a sixteenth of the 16-bit rate.  So every matrix is kept as the sum of two fp16
// ones, 22 bits, and a product is three MFMA: hi hi + hi lo + lo hi, in fp32.
// fp16's narrow range is no matter here: the polynomial bounds each singular value,
// and with them every element of X, A and B, so each is stored times a power of
// two that takes its bound to fp16's largest values.
// A and B are symmetric: only tiles on and below the diagonal are computed, the
// others are written from them.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "common.h"
#include "gemm_pipe.h"
#include "kernels.h"

namespace fal {

namespace {

typedef _Float16 half_t;
typedef _Float16 halfx8_t __attribute__((ext_vector_type(8)));

constexpr int kTile = 128;      // tile sides; matrices are padded to it with zeros
constexpr int kNormParts = 1024;
constexpr int kOneRound = 256;  // tiles that have a compute unit each

// A matrix of a batch: hi and lo parts, [count][rows][ld] each.
struct Split {
  half_t *hi, *lo;
};

__device__ __forceinline__ void split4(const float (&v)[4], uint2& hi, uint2& lo) {
  union { half_t h[4]; uint2 w; } a, b;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    a.h[c] = static_cast<half_t>(v[c]);
    b.h[c] = static_cast<half_t>(v[c] - static_cast<float>(a.h[c]));
  }
  hi = a.w;
  lo = b.w;
}
__device__ __forceinline__ void join4(const uint2& hi, const uint2& lo, float (&v)[4]) {
  union { uint2 w; half_t h[4]; } a{hi}, b{lo};
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = static_cast<float>(a.h[c]) + static_cast<float>(b.h[c]);
}

enum Product : int { GRAM = 0, POLY = 1, APPLY = 2, LAST = 3 };

// What the last product writes: a dtype matrix, or the update of the weights.
struct Result {
  int rows, cols, flip;    // of the caller's matrices
  int64_t stride;          // elements between them
  void* out;               // dtype
  int bf16_out;
  float* master;           // update: out may be NULL
  float decay, step;       // 1 - lr weight_decay, lr scale
  int vec;                 // rows of whole 16-byte groups
};

struct NsArgs {
  Split a, b, c;           // operands and result
  Split d;                 // POLY: A, beside the product
  int lda, ldb, ldc, ldd;
  int64_t sa, sb, sc, sd;  // elements between the matrices of a batch
  int K, tiles_m, tiles_n, per_matrix, total;
  float scale;             // of the accumulators
  float ca, cb;            // POLY: a and b, at the result's scale
  int splits, per;         // ranges of K, slices of one
  float* part;             // the ranges' accumulators
  int M, N;                // sides, multiples of 128
  int tiles, whole;        // large tiles: in all, and those that are not cut
  Result r;
};

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, FAL_WAVE);
  return v;
}
__device__ __forceinline__ double block_sum_d(double v, double* red) {
  v = wave_sum_d(v);
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

// ---------------------------------------------------------------- input --
// What is made orthogonal: a dtype matrix, or momentum and gradient.
struct Source {
  const void* x;
  int bf16_in;
  const float* g;  // update: U = g + beta m, or m
  float* m;
  float beta;
  int nesterov;
  int rows, cols;
  int64_t stride;
};

__device__ __forceinline__ float element(const Source& s, int64_t i) {
  if (s.g) return s.nesterov ? fmaf(s.beta, s.m[i], s.g[i]) : s.m[i];
  return s.bf16_in ? to_f(static_cast<const bf16*>(s.x)[i]) : static_cast<const float*>(s.x)[i];
}

// The momentum's update, and a workgroup's part of each matrix's sum of squares
// in fp64.  VEC: matrices of whole 16-byte groups, taken four groups at a time so
// that their loads are under way together.
template <int VEC>
__global__ __launch_bounds__(256) void ns_norm(Source s, double* part) {
  __shared__ double red[4];
  const int64_t n = (int64_t)s.rows * s.cols, base = blockIdx.y * s.stride;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  double sum = 0.0;
  if (VEC && s.g) {
    const float4* g = reinterpret_cast<const float4*>(s.g + base);
    float4* m = reinterpret_cast<float4*>(s.m + base);
    constexpr int N = 4;
    for (int64_t i0 = at; i0 < n / 4; i0 += N * step) {
      float4 gv[N], mv[N];
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (i0 + k * step < n / 4) { gv[k] = g[i0 + k * step]; mv[k] = m[i0 + k * step]; }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (i0 + k * step >= n / 4) break;
        float4 v = mv[k];
        v.x = fmaf(s.beta, v.x, gv[k].x); v.y = fmaf(s.beta, v.y, gv[k].y);
        v.z = fmaf(s.beta, v.z, gv[k].z); v.w = fmaf(s.beta, v.w, gv[k].w);
        m[i0 + k * step] = v;
        if (s.nesterov) {
          v.x = fmaf(s.beta, v.x, gv[k].x); v.y = fmaf(s.beta, v.y, gv[k].y);
          v.z = fmaf(s.beta, v.z, gv[k].z); v.w = fmaf(s.beta, v.w, gv[k].w);
        }
        sum = fma((double)v.x, (double)v.x, fma((double)v.y, (double)v.y, sum));
        sum = fma((double)v.z, (double)v.z, fma((double)v.w, (double)v.w, sum));
      }
    }
  } else if (VEC) {
    // 16 bytes: four fp32 or eight bf16
    const uint4* x = static_cast<const uint4*>(s.x) + base / (s.bf16_in ? 8 : 4);
    const int64_t n16 = n / (s.bf16_in ? 8 : 4);
    constexpr int N = 4;
    for (int64_t i0 = at; i0 < n16; i0 += N * step) {
      uint4 q[N];
#pragma unroll
      for (int k = 0; k < N; ++k) q[k] = i0 + k * step < n16 ? x[i0 + k * step] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (s.bf16_in) {
            const double lo = __uint_as_float(w[e] << 16), hi = __uint_as_float(w[e] & 0xFFFF0000u);
            sum = fma(lo, lo, fma(hi, hi, sum));
          } else {
            const double v = __uint_as_float(w[e]);
            sum = fma(v, v, sum);
          }
        }
      }
    }
  } else {
    for (int64_t i = at; i < n; i += step) {
      if (s.g) s.m[base + i] = fmaf(s.beta, s.m[base + i], s.g[base + i]);
      const double v = element(s, base + i);
      sum = fma(v, v, sum);
    }
  }
  sum = block_sum_d(sum, red);
  if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = sum;
}

// A 64 x 64 tile of X_0: U / |U|, transposed if its columns are the smaller side,
// zeros in the padding.
__global__ __launch_bounds__(256) void ns_first(Source s, const double* part, int nparts, int flip, Split x, int P,
                                                int Q, float scale) {
  __shared__ double red[4];
  __shared__ float tile[64][65];
  const int mat = blockIdx.z;
  double sum = 0.0;
  for (int i = threadIdx.x; i < nparts; i += 256) sum += part[mat * nparts + i];
  const double norm2 = block_sum_d(sum, red);
  // (zeros for a matrix of zeros; NaN throughout where U is not finite)
  const double inv = norm2 == 0.0 ? 0.0 : norm2 <= 1.7e308 ? (double)scale / sqrt(norm2) : __builtin_nan("");
  const int64_t base = mat * s.stride;
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;  // of X
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  for (int i = w; i < 64; i += 4) {
    // element (r0 + i, c0 + lane) of U, or of X^T's tile
    const int r = (flip ? c0 : r0) + i, c = (flip ? r0 : c0) + lane;
    float v = 0.f;
    if (r < s.rows && c < s.cols) v = (float)((double)element(s, base + (int64_t)r * s.cols + c) * inv);
    if (flip) tile[lane][i] = v;
    else tile[i][lane] = v;
  }
  __syncthreads();
  for (int i = w * 4 + lane / 16; i < 64; i += 16) {
    const int c = lane % 16 * 4;
    const float v[4] = {tile[i][c], tile[i][c + 1], tile[i][c + 2], tile[i][c + 3]};
    uint2 hi, lo;
    split4(v, hi, lo);
    const int64_t o = (int64_t)mat * P * Q + (int64_t)(r0 + i) * Q + c0 + c;
    *reinterpret_cast<uint2*>(x.hi + o) = hi;
    *reinterpret_cast<uint2*>(x.lo + o) = lo;
  }
}

// ------------------------------------------------------------- products --
// Row and column of tile t of a lower triangle, row by row.
__device__ __forceinline__ void triangle(int t, int& r, int& c) {
  r = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
  while (r * (r + 1) / 2 > t) --r;
  while ((r + 1) * (r + 2) / 2 <= t) ++r;
  c = t - r * (r + 1) / 2;
}

// What the epilogue reads for four consecutive elements (r, c .. c + 3) of the
// result, asked for ahead of their use: POLY's A, or the update's weights.
struct Beside {
  uint2 hi, lo;
  float4 w;  // (single elements of four rows where rows are no whole 16-byte groups)
};
template <int MODE>
__device__ __forceinline__ void ask(const NsArgs& p, int mat, int r, int c, Beside& b) {
  if (MODE == POLY) {
    const int64_t o = mat * p.sd + (int64_t)r * p.ldd + c;
    b.hi = *reinterpret_cast<const uint2*>(p.d.hi + o);
    b.lo = *reinterpret_cast<const uint2*>(p.d.lo + o);
  } else if (MODE == LAST && p.r.master && r < p.r.rows) {
    if (c < p.r.cols)
      b.w = *reinterpret_cast<const float4*>(p.r.master + mat * p.r.stride + (int64_t)r * p.r.cols + c);
  }
}

// The result's element (r, c), of rows that are no whole 16-byte groups.
__device__ __forceinline__ float ask_one(const NsArgs& p, int mat, int r, int c) {
  return p.r.master && r < p.r.rows && c < p.r.cols ? p.r.master[mat * p.r.stride + (int64_t)r * p.r.cols + c] : 0.f;
}
__device__ __forceinline__ void put_one(const NsArgs& p, int mat, int r, int c, float v, float w) {
  if (r >= p.r.rows || c >= p.r.cols) return;
  const int64_t o = mat * p.r.stride + (int64_t)r * p.r.cols + c;
  v *= p.scale;
  if (p.r.master) {
    v = fmaf(w, p.r.decay, -p.r.step * v);
    p.r.master[o] = v;
    if (!p.r.out) return;
  }
  if (p.r.bf16_out) static_cast<bf16*>(p.r.out)[o] = from_f<bf16>(v);
  else static_cast<float*>(p.r.out)[o] = v;
}

// Four consecutive elements of the result.
template <int MODE>
__device__ __forceinline__ void put(const NsArgs& p, int mat, int r, int c, const float4& acc, const Beside& b) {
  float v[4] = {acc.x * p.scale, acc.y * p.scale, acc.z * p.scale, acc.w * p.scale};
  if (MODE == LAST) {
    if (r >= p.r.rows || c >= p.r.cols) return;
    const int64_t o = mat * p.r.stride + (int64_t)r * p.r.cols + c;
    if (p.r.master) {
      v[0] = fmaf(b.w.x, p.r.decay, -p.r.step * v[0]);
      v[1] = fmaf(b.w.y, p.r.decay, -p.r.step * v[1]);
      v[2] = fmaf(b.w.z, p.r.decay, -p.r.step * v[2]);
      v[3] = fmaf(b.w.w, p.r.decay, -p.r.step * v[3]);
      *reinterpret_cast<float4*>(p.r.master + o) = make_float4(v[0], v[1], v[2], v[3]);
      if (!p.r.out) return;
    }
    if (p.r.bf16_out) st4(static_cast<bf16*>(p.r.out) + o, v);
    else *reinterpret_cast<float4*>(static_cast<float*>(p.r.out) + o) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
  if (MODE == POLY) {
    float a[4];
    join4(b.hi, b.lo, a);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += fmaf(p.cb, a[e], r == c + e ? p.ca : 0.f);
  }
  uint2 hi, lo;
  split4(v, hi, lo);
  const int64_t o = mat * p.sc + (int64_t)r * p.ldc + c;
  *reinterpret_cast<uint2*>(p.c.hi + o) = hi;
  *reinterpret_cast<uint2*>(p.c.lo + o) = lo;
}

// The epilogue works on strips of 16 rows (COLS: columns) of a wavefront's W x W,
// passed through LDS so that consecutive lanes hold consecutive elements: lane 16g +
// c of block (i, j) holds row 16i + c, columns 16j + 4g .. +3.  A tile's columns are
// rows of the result where it is mirrored or transposed.
template <int MODE, bool COLS, int W = 64>
struct Strip {
  static constexpr int PITCH = W + 4;
  static constexpr int N = W / 16;          // blocks of a strip, and accesses of a lane
  static constexpr int LPR = W / 4;         // lanes of a row
  static constexpr int RPA = 64 / LPR;      // rows of an access
  static constexpr int ROWS = 16 * W / 64;  // rows of a lane that holds one column
  Beside beside[N];
  int r, c;  // this lane's first row and its columns
  // Strip q of the W x W at (mw, nw).
  __device__ __forceinline__ void ask_for(const NsArgs& p, int mat, int mw, int nw, int q) {
    const int lane = threadIdx.x & 63;
    r = (COLS ? nw : mw) + 16 * q;
    c = COLS ? mw : nw;
    if (MODE == LAST && !p.r.vec) {
      // a lane to a column
      r += lane / W * ROWS;
      c += lane % W;
#pragma unroll
      for (int k = 0; k < N; ++k)
        beside[k].w = make_float4(ask_one(p, mat, r + 4 * k, c), ask_one(p, mat, r + 4 * k + 1, c),
                                  ask_one(p, mat, r + 4 * k + 2, c), ask_one(p, mat, r + 4 * k + 3, c));
      return;
    }
    r += lane / LPR;
    c += 4 * (lane % LPR);
#pragma unroll
    for (int k = 0; k < N; ++k) ask<MODE>(p, mat, r + RPA * k, c, beside[k]);
  }
  // blocks: (q, 0 .. N - 1), COLS: (0 .. N - 1, q).
  __device__ __forceinline__ void emit(const NsArgs& p, int mat, const f32x4_t (&blocks)[N], float* strip) const {
    const int lane = threadIdx.x & 63, g = lane >> 4, cl = lane & 15;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (COLS) {
#pragma unroll
        for (int e = 0; e < 4; ++e) strip[(4 * g + e) * PITCH + 16 * j + cl] = blocks[j][e];
      } else {
        *reinterpret_cast<f32x4_t*>(strip + cl * PITCH + 16 * j + 4 * g) = blocks[j];
      }
    }
    wave_lds_order();
    if (MODE == LAST && !p.r.vec) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float* s = strip + (lane / W * ROWS + 4 * k) * PITCH + lane % W;
        put_one(p, mat, r + 4 * k, c, s[0], beside[k].w.x);
        put_one(p, mat, r + 4 * k + 1, c, s[PITCH], beside[k].w.y);
        put_one(p, mat, r + 4 * k + 2, c, s[2 * PITCH], beside[k].w.z);
        put_one(p, mat, r + 4 * k + 3, c, s[3 * PITCH], beside[k].w.w);
      }
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k)
        put<MODE>(p, mat, r + RPA * k, c,
                  *reinterpret_cast<const float4*>(strip + (RPA * k + lane / LPR) * PITCH + 4 * (lane % LPR)),
                  beside[k]);
    }
    wave_lds_order();
  }
};
constexpr int kStrip = 16 * Strip<GRAM, false>::PITCH;  // floats of LDS
template <int MODE>
__device__ __forceinline__ bool emits(const NsArgs& p, int tm, int tn, bool cols) {
  if (MODE == LAST) return cols == (p.r.flip != 0);
  return !cols || ((MODE == GRAM || MODE == POLY) && tm != tn);
}

// The W x W at (mw, nw), blocks (I, J) .. of a wavefront's, every strip's operands
// asked for at once.
template <int MODE, bool COLS, int W, int FM, int FN, int I = 0, int J = 0>
__device__ __forceinline__ void ns_emit(const NsArgs& p, int mat, int mw, int nw, const f32x4_t (&acc)[FM][FN],
                                        float* strip) {
  constexpr int N = W / 16;
  Strip<MODE, COLS, W> s[N];
#pragma unroll
  for (int q = 0; q < N; ++q) s[q].ask_for(p, mat, mw, nw, q);
#pragma unroll
  for (int q = 0; q < N; ++q) {
    f32x4_t blocks[N];
#pragma unroll
    for (int j = 0; j < N; ++j) blocks[j] = COLS ? acc[I + j][J + q] : acc[I + q][J + j];
    s[q].emit(p, mat, blocks, strip);
  }
}

// A T x T tile of a product of split matrices: A k-contiguous, B
// k-contiguous (GRAM, POLY: rows of the same matrix) or MN-major (X).  Four
// wavefronts of T/2 x T/2; slices of 32 k of all four parts in NS LDS stages, asked
// for NS - 1 slices ahead, the fragments of slice s + 1 read under the MFMA (48 of
// a tile of 128) of slice s.
template <int MODE, int T, int OCC, int NS>
__global__ __launch_bounds__(256, OCC) void ns_product(NsArgs p) {
  using namespace pipe;
  constexpr int BK = MODE == GRAM || MODE == POLY;
  constexpr int WT = T / 2, F = WT / 16;
  typedef Src<T, 1> SA;
  typedef Src<T, BK> SB;
  constexpr int REGION = SA::BYTES, SBYTES = 4 * REGION, L = 4 * SA::IPW;
  static_assert(SB::BYTES == REGION && (NS == 2 || NS == 4), "stages");
  // one array a stage: the compiler tracks loads to LDS array by array
  constexpr int LATER = NS == 4 ? SBYTES : 16;
  __shared__ __attribute__((aligned(1024))) char st0[SBYTES], st1[SBYTES], st2[LATER], st3[LATER];
  auto stage_ptr = [&](int k) -> char* { return k == 0 ? st0 : k == 1 ? st1 : k == 2 ? st2 : st3; };

  const int bid = xcd_remap(blockIdx.x, p.total);
  const int t = bid % p.per_matrix, range = bid / p.per_matrix % p.splits, mat = bid / p.per_matrix / p.splits;
  int tm, tn;
  if (BK) triangle(t, tm, tn);
  else grouped_tile(t, p.tiles_m, p.tiles_n, tm, tn);
  const int m0 = tm * T, n0 = tn * T;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  SA ah, al;
  SB bh, bl;
  auto as = [](const half_t* x) { return reinterpret_cast<const bf16*>(x); };
  const int M = p.M, N = p.N;
  ah.init(0, as(p.a.hi + mat * p.sa), p.lda, m0, M, p.K, wave, lane);
  al.init(0, as(p.a.lo + mat * p.sa), p.lda, m0, M, p.K, wave, lane);
  bh.init(0, as(p.b.hi + mat * p.sb), p.ldb, n0, N, p.K, wave, lane);
  bl.init(0, as(p.b.lo + mat * p.sb), p.ldb, n0, N, p.K, wave, lane);
  ah.clear(1);
  al.clear(1);
  bh.clear(1);
  bl.clear(1);
  // this range's slices (both it and K are multiples of 128)
  const int k0 = range * p.per * KS, n = min(p.per, p.K / KS - range * p.per);
  auto issue = [&](char* stage, int s) {
    if (s > 0 && s < n) {
      ah.advance();
      al.advance();
      bh.advance();
      bl.advance();
    } else {
      const int lim = s < n ? KS : 0;  // slices past the end: zeros
      ah.set(0, k0, lim);
      al.set(0, k0, lim);
      bh.set(0, k0, lim);
      bl.set(0, k0, lim);
    }
    ah.load(stage, wave);
    al.load(stage + REGION, wave);
    bh.load(stage + 2 * REGION, wave);
    bl.load(stage + 3 * REGION, wave);
  };
  Frag<T, 1, F> fa;
  Frag<T, BK, F> fb;
  fa.init(wm * WT, lane);
  fb.init(wn * WT, lane);
  f32x4_t acc[F][F];
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  halfx8_t ra[2][2][F], rb[2][2][F];
  auto read = [&](const char* stage, int buf) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < F; ++i) {
        ra[buf][h][i] = __builtin_bit_cast(halfx8_t, fa.read(stage + h * REGION, i));
        rb[buf][h][i] = __builtin_bit_cast(halfx8_t, fb.read(stage + (2 + h) * REGION, i));
      }
  };
  auto mma = [&](int buf) {
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rb[buf][q == 1][j], ra[buf][q == 0][i], acc[i][j], 0, 0, 0);
  };
  constexpr int NRD = 2 * F * (1 + (BK ? 1 : 2)), NMF = 3 * F * F;
  constexpr int DMA_EVERY = (NMF - NRD) / L > 0 ? (NMF - NRD) / L : 1;
  auto interleave = [&]() {
    int dma = 0;
#pragma unroll
    for (int q = 0; q < NMF; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
      if (q < NRD) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read
      else if ((q - NRD) % DMA_EVERY == 0 && dma < L) {
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // buffer load to LDS
        ++dma;
      }
    }
  };
#pragma unroll
  for (int k = 0; k < NS; ++k) issue(stage_ptr(k), k);
  FAL_WAITCNT(L * (NS - 1), 0);
  bar();
  read(st0, 0);
  // Step s: own loads of slice s + 1 and own reads of slice s are done, barrier
  // (slice s + 1 whole in LDS, slice s's stage free), slice s + NS into that
  // stage, the MFMA of slice s under the reads of slice s + 1.  (n is a multiple
  // of four)
  for (int s = 0; s < n; s += NS) {
#pragma unroll
    for (int U = 0; U < NS; ++U) {
      FAL_WAITCNT(L * (NS - 2), 0);
      bar();
      __builtin_amdgcn_sched_barrier(0);
      issue(stage_ptr(U), s + U + NS);
      read(stage_ptr((U + 1) % NS), (U + 1) & 1);
      mma(U & 1);
      interleave();
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  FAL_WAITCNT(0, 0);
  bar();

  if (MODE == GRAM && p.splits > 1) {
    float* o = p.part + ((int64_t)bid * 256 + threadIdx.x) * 4;
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j) *reinterpret_cast<f32x4_t*>(o + (i * F + j) * (int64_t)p.total * 1024) = acc[i][j];
    return;
  }
  constexpr int STRIP = 16 * Strip<MODE, false, WT>::PITCH;
  static_assert(4 * STRIP * 4 <= SBYTES, "epilogue staging");
  float* strip = reinterpret_cast<float*>(st0) + wave * STRIP;
  const int mw = m0 + wm * WT, nw = n0 + wn * WT;
  if (emits<MODE>(p, tm, tn, false)) ns_emit<MODE, false, WT, F, F>(p, mat, mw, nw, acc, strip);
  if (emits<MODE>(p, tm, tn, true)) ns_emit<MODE, true, WT, F, F>(p, mat, mw, nw, acc, strip);
}

// A tile's ranges added in order, and its epilogue: a workgroup for each strip of its
// wavefronts' 64 x 64 (one for a whole tile took 12.7 us for 18 tiles of 8 ranges,
// these 7.6).  F: blocks along a wavefront's columns.  The sums of block (i, j) lie
// `total` * 1024 floats from those of the next, a range's `tiles` * 1024.
template <bool COLS, int F>
__device__ __forceinline__ void join_strip(const NsArgs& p, int mat, int mw, int nw, const float* o, int64_t tiles, int I,
                                           int J, int q, float* strip) {
  Strip<GRAM, COLS> s;
  s.ask_for(p, mat, mw, nw, q);
  f32x4_t sum[4];
  const int64_t block = (int64_t)p.total * 1024, range = tiles * 1024;
  for (int r0 = 0; r0 < p.splits; r0 += 4) {
    f32x4_t v[4][4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (r0 + r < p.splits)
          v[r][j] = *reinterpret_cast<const f32x4_t*>(o + (r0 + r) * range +
                                                      (COLS ? F * (I + j) + J + q : F * (I + q) + J + j) * block);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (r0 + r < p.splits) sum[j] = r0 + r ? sum[j] + v[r][j] : v[r][j];
  }
  s.emit(p, mat, sum, strip);
}
__global__ __launch_bounds__(256, 2) void ns_join(NsArgs p) {
  __shared__ __attribute__((aligned(16))) float lds[4][kStrip];
  const int q = blockIdx.x & 3, t = blockIdx.x / 4 % p.per_matrix, mat = blockIdx.x / 4 / p.per_matrix;
  int tm, tn;
  triangle(t, tm, tn);
  const int wave = threadIdx.x >> 6, mw = tm * kTile + (wave >> 1) * 64, nw = tn * kTile + (wave & 1) * 64;
  const float* o = p.part + (((int64_t)mat * p.splits * p.per_matrix + t) * 256 + threadIdx.x) * 4;
  join_strip<false, 4>(p, mat, mw, nw, o, p.per_matrix, 0, 0, q, lds[wave]);
  if (tm != tn) join_strip<true, 4>(p, mat, mw, nw, o, p.per_matrix, 0, 0, q, lds[wave]);
}

// ----------------------------------------------------------- large tiles --
// X X^T of many columns on tiles of 256 x 256, a wavefront's 128 x 128: half the
// bytes through LDS for a product.  A slice's three products run one after the
// other, so that each part's fragments are read while two others multiply and no
// part is held twice:
//   A.hi B.lo  (reads B.hi),  A.hi B.hi  (reads A.lo),
//   barrier: this slice is read, the next one has landed,
//   A.lo B.hi  (reads the next slice's A.hi and B.lo, asks for the one after).
// Whole rounds of a tile a compute unit go first; what is left of the tiles is cut
// along k so that it fills the chip once more, and joined (2 x 2048 x 5504, 72 tiles
// in three ranges: 154 us and 22 joined, at the library's rate of a fp16 product;
// 272 tiles of 128 x 128 219).  The other products gain nothing: B X on 256 x 128
// tiles took 279 us against 251, A A of 2048 rows 63 and 26 joined against 86.
constexpr int kBig = 256;

__device__ __forceinline__ void big_tile(const NsArgs& p, int tile, int& mat, int& tm, int& tn) {
  mat = tile / p.per_matrix;
  triangle(tile % p.per_matrix, tm, tn);
}

__global__ __launch_bounds__(256, 1) void ns_big(NsArgs p) {
  using namespace pipe;
  constexpr int F = 8, WT = 128;
  typedef Src<kBig, 1> S;
  constexpr int REGION = S::BYTES, SBYTES = 4 * REGION, L = 4 * S::IPW;
  __shared__ __attribute__((aligned(1024))) char st0[SBYTES], st1[SBYTES];
  int tile, range = 0, slot = 0;
  if ((int)blockIdx.x < p.whole) {
    tile = xcd_remap(blockIdx.x, p.whole);
  } else {
    const int rest = p.tiles - p.whole;
    slot = xcd_remap(blockIdx.x - p.whole, p.total);
    tile = p.whole + slot % rest;
    range = slot / rest;
  }
  const bool cut = (int)blockIdx.x >= p.whole && p.splits > 1;
  int mat, tm, tn;
  big_tile(p, tile, mat, tm, tn);
  const int m0 = tm * kBig, n0 = tn * kBig;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int slices = p.K / KS, s0 = cut ? range * p.per : 0, n = cut ? min(p.per, slices - s0) : slices;

  S ah, al, bh, bl;
  auto start = [&](S& x, const half_t* at, int r0) {
    x.init(0, reinterpret_cast<const bf16*>(at + mat * p.sa), p.lda, r0, p.M, p.K, wave, lane);
    x.clear(1);
    x.start(p.lda, r0, p.M, p.K);
    x.so = (uint32_t)(s0 * KS) * x.ks;
  };
  start(ah, p.a.hi, m0);
  start(al, p.a.lo, m0);
  start(bh, p.a.hi, n0);
  start(bl, p.a.lo, n0);
  auto issue = [&](char* stage) {
    ah.load(stage, wave);
    al.load(stage + REGION, wave);
    bh.load(stage + 2 * REGION, wave);
    bl.load(stage + 3 * REGION, wave);
    ah.advance();
    al.advance();
    bh.advance();
    bl.advance();
  };
  Frag<kBig, 1, F> fa, fb;
  fa.init(wm * WT, lane);
  fb.init(wn * WT, lane);
  f32x4_t acc[F][F];
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  halfx8_t ahi[F], alo[F], bhi[F], blo[F];
  auto read = [&](halfx8_t (&r)[F], const Frag<kBig, 1, F>& f, const char* region) {
#pragma unroll
    for (int i = 0; i < F; ++i) r[i] = __builtin_bit_cast(halfx8_t, f.read(region, i));
  };
  auto mma = [&](const halfx8_t (&a)[F], const halfx8_t (&b)[F]) {
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[j], a[i], acc[i][j], 0, 0, 0);
  };
  // one LDS read an MFMA from the first on, loads after them
  auto interleave = [&](int reads, int loads) {
#pragma unroll
    for (int q = 0; q < F * F; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
      if (q < reads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read
      else if (q - reads < loads) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // buffer load to LDS
    }
  };
  // keeps 256 accumulators in the accumulation registers (left to itself the
  // allocator moves two of three through the others and back each slice)
  auto hold = [&]() {
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j) asm volatile("" : "+a"(acc[i][j]));
  };
  auto step = [&](char* now, const char* next) {
    hold();
    read(bhi, fb, now + 2 * REGION);
    mma(ahi, blo);
    interleave(F, 0);
    __builtin_amdgcn_sched_barrier(0);
    read(alo, fa, now + REGION);
    mma(ahi, bhi);
    interleave(F, 0);
    __builtin_amdgcn_sched_barrier(0);
    FAL_WAITCNT(0, 0);
    bar();
    __builtin_amdgcn_sched_barrier(0);
    issue(now);
    read(blo, fb, next + 3 * REGION);
    read(ahi, fa, next);
    mma(alo, bhi);
    interleave(2 * F, L);
    __builtin_amdgcn_sched_barrier(0);
  };
  issue(st0);
  issue(st1);
  FAL_WAITCNT(L, 0);
  bar();
  read(blo, fb, st0 + 3 * REGION);
  read(ahi, fa, st0);
  // (n is even.  Slices past it are asked for and not multiplied: what lies behind,
  // or zeros past the buffers' range.)
  for (int s = 0; s < n; s += 2) {
    step(st0, st1);
    step(st1, st0);
  }
  hold();
  FAL_WAITCNT(0, 0);
  bar();

  if (cut) {
    float* o = p.part + ((int64_t)slot * 256 + threadIdx.x) * 4;
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
      for (int j = 0; j < F; ++j) *reinterpret_cast<f32x4_t*>(o + (i * F + j) * (int64_t)p.total * 1024) = acc[i][j];
    return;
  }
  float* strip = reinterpret_cast<float*>(st0) + wave * kStrip;
  const int mw = m0 + wm * WT, nw = n0 + wn * WT;
  auto quarter = [&](auto hi, auto hj) {
    constexpr int I = 4 * decltype(hi)::value, J = 4 * decltype(hj)::value;
    // (the sides are multiples of 128: a quarter lies inside or past the end)
    if (mw + 16 * I >= p.M || nw + 16 * J >= p.M) return;
    ns_emit<GRAM, false, 64, F, F, I, J>(p, mat, mw + 16 * I, nw + 16 * J, acc, strip);
    if (tm != tn) ns_emit<GRAM, true, 64, F, F, I, J>(p, mat, mw + 16 * I, nw + 16 * J, acc, strip);
  };
  typedef std::integral_constant<int, 0> zero;
  typedef std::integral_constant<int, 1> one;
  quarter(zero(), zero());
  quarter(zero(), one());
  quarter(one(), zero());
  quarter(one(), one());
}

__global__ __launch_bounds__(256, 2) void ns_big_join(NsArgs p) {
  __shared__ __attribute__((aligned(16))) float lds[4][kStrip];
  const int q = blockIdx.x & 3, J = blockIdx.x & 4, I = blockIdx.x >> 1 & 4, rest = blockIdx.x >> 4;
  int mat, tm, tn;
  big_tile(p, p.whole + rest, mat, tm, tn);
  const int wave = threadIdx.x >> 6;
  const int mw = tm * kBig + (wave >> 1) * 128 + 16 * I, nw = tn * kBig + (wave & 1) * 128 + 16 * J;
  if (mw >= p.M || nw >= p.M) return;
  const float* o = p.part + ((int64_t)rest * 256 + threadIdx.x) * 4;
  float* strip = lds[wave];
  const int tiles = p.tiles - p.whole;
  join_strip<false, 8>(p, mat, mw, nw, o, tiles, I, J, q, strip);
  if (tm != tn) join_strip<true, 8>(p, mat, mw, nw, o, tiles, I, J, q, strip);
}

// How a product runs: tiles of side x side, the first `whole` of them (large ones
// only) uncut and the others in `splits` ranges of `per` slices.
struct Plan {
  int side, tiles, whole, splits, per;
  int64_t part() const {  // bytes of the ranges' sums
    return splits > 1 ? (int64_t)(tiles - whole) * splits * side * side * 4 : 0;
  }
};

// Tiles of 64 x 64 while two a compute unit hold them all: more workgroups, each a
// quarter as long (five steps of 384 x 384: 227 us on tiles of 128, 115 on these; 3 x
// 1001 x 333 268 and 165; 4 x 512 x 2048, whose B X would be 1024 of them, 269 with
// and 247 without).
constexpr int kFine = 64, kFineTiles = 512;

// X X^T, which may have many more slices than rows, on the tiles whose estimated time
// is the smallest (us: a slice of 32 k on a tile of each size, alone on its compute
// unit or sharing it; what each round and a joining launch add; ranges' sums written
// and read at 8 TB/s).  Tiles of 128 that leave half the compute units empty take K in
// ranges of at least four slices (256 x 4096: 209 us, 252 on fine tiles; 1024 x 2048
// 292 and 277; 3 x 1024 x 2048 502 and 526).
Plan plan_gram(int P, int K, int matrices) {
  constexpr double kBigSlice = 2.45, kPair = 1.04, kAlone = 0.65, kFineAlone = 0.27, kFineTwo = 0.4, kFinePair = 0.7;
  constexpr double kBigRound = 12.0, kRound = 8.0, kFineRound = 4.0, kJoin = 6.0;
  auto count = [&](int side) { return cdiv(P, side) * (cdiv(P, side) + 1) / 2 * matrices; };
  const int slices = K / pipe::KS;
  Plan b = {kBig, count(kBig), 0, 1, slices};
  b.whole = b.tiles / kOneRound * kOneRound;
  const int rest = b.tiles - b.whole;
  double big = b.whole / kOneRound * (kBigRound + slices * kBigSlice);
  if (rest) {
    const int s = std::max(1, std::min(kOneRound / rest, slices / 4)), each = cdiv(cdiv(slices, s), 2) * 2;
    const double join = kJoin + (double)rest * s * kBig * kBig * 4 / 4e6;
    if (s > 1 && (slices - each) * kBigSlice > join) {
      b.per = each;
      b.splits = cdiv(slices, each);
      big += join;
    }
    big += kBigRound + b.per * kBigSlice;
  }
  Plan t = {kTile, count(kTile), 0, 1, slices};
  if (t.tiles <= kOneRound / 2) {
    t.per = cdiv(cdiv(slices, std::min(kOneRound / t.tiles, slices / 4)), 4) * 4;
    t.splits = cdiv(slices, t.per);
  }
  const int n = t.tiles * t.splits, rounds = n / (2 * kOneRound), last = n % (2 * kOneRound);
  double small = n <= kOneRound ? kRound + t.per * kAlone : rounds * (kRound + t.per * kPair);
  if (n > kOneRound && last) small += kRound + t.per * (last > kOneRound ? kPair : kAlone);
  if (t.splits > 1) small += kJoin + t.part() / 4e6;
  const Plan f = {kFine, count(kFine), 0, 1, slices};
  const double filled = (double)(f.tiles - kOneRound) / kOneRound;
  const double fine = kFineRound + slices * (filled <= 0.0 ? kFineAlone : kFineTwo + filled * (kFinePair - kFineTwo));
  if (f.tiles <= kFineTiles && fine < std::min(big, small)) return f;
  return big < small ? b : t;
}

template <int MODE>
Plan plan(int M, int N, int K, int matrices) {
  if (MODE == GRAM) return plan_gram(M, K, matrices);
  auto count = [&](int side) {
    const int tm = M / side, tn = N / side;
    return (MODE == POLY ? tm * (tm + 1) / 2 : tm * tn) * matrices;
  };
  const int side = count(kFine) <= kFineTiles ? kFine : kTile;
  return {side, count(side), 0, 1, K / pipe::KS};
}

template <int MODE>
void launch(NsArgs p, int matrices, hipStream_t s) {
  const Plan q = plan<MODE>(p.M, p.N, p.K, matrices);
  p.tiles_m = p.M / q.side;
  p.tiles_n = p.N / q.side;
  p.per_matrix = q.tiles / matrices;
  p.splits = q.splits;
  p.per = q.per;
  p.tiles = q.tiles;
  p.whole = q.whole;
  p.total = (q.tiles - q.whole) * q.splits;
  if (MODE == GRAM && q.side == kBig) {
    hipLaunchKernelGGL(ns_big, dim3(q.whole + p.total), dim3(256), 0, s, p);
    if (q.splits > 1) hipLaunchKernelGGL(ns_big_join, dim3(16 * (q.tiles - q.whole)), dim3(256), 0, s, p);
    return;
  }
  if (q.side == kFine) hipLaunchKernelGGL((ns_product<MODE, kFine, 2, 4>), dim3(p.total), dim3(256), 0, s, p);
  else if (p.total <= kOneRound) hipLaunchKernelGGL((ns_product<MODE, kTile, 1, 4>), dim3(p.total), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((ns_product<MODE, kTile, 2, 2>), dim3(p.total), dim3(256), 0, s, p);
  if (q.splits > 1) hipLaunchKernelGGL(ns_join, dim3(4 * q.tiles), dim3(256), 0, s, p);
}

// --------------------------------------------------------- small matrices --
// A matrix whose parts fit the LDS of one compute unit goes through all its steps
// in one workgroup: one launch instead of 2 + 3 a step, each of which is latency
// (four matrices of 64 x 192, five steps: 17 launches 87 us a call, this 31; one of
// 128 x 160, the largest that fits, 85 and 84).
// LDS holds X [P][Q + 8] and, in one place one after the other, A and B [P][P + 8],
// hi and lo parts each; P is rounded up to 32, Q to 64, and zero there.
constexpr int kSmallLds = 155648, kSmallWaves = 16, kSmallSide = 128;

struct SmallArgs {
  int P, Q, flip, steps;
  float x_scale;     // of X: 2^ex
  float a_scale;     // accumulators to A: 2^(ea - 2 ex)
  float c_scale, ca, cb;  // B's parts: c 2^(eb - 2 ea), a 2^eb, b 2^(eb - ea)
  float apply_scale; // accumulators to X: 2^-eb
  float out_scale;   // ... to the result: 2^-(eb + ex)
};

__device__ __forceinline__ halfx8_t row8(const half_t* m, int pitch, int row0, int k0, int lane) {
  return *reinterpret_cast<const halfx8_t*>(m + (row0 + (lane & 15)) * pitch + k0 + 8 * (lane >> 4));
}
// The same of a matrix's columns: eight consecutive k of column n0 + lane % 16.
__device__ __forceinline__ halfx8_t col8(const half_t* m, int pitch, int n0, int k0, int lane) {
  const bf16* at = reinterpret_cast<const bf16*>(m + (k0 + 8 * (lane >> 4) + ((lane & 15) >> 2)) * pitch + n0 + 4 * (lane & 3));
  const i16x4_t v[2] = {lds_read_tr(at), lds_read_tr(at + 4 * pitch)};
  return *reinterpret_cast<const halfx8_t*>(v);
}
__device__ __forceinline__ void mma3(const halfx8_t (&a)[2], const halfx8_t (&b)[2], f32x4_t (&acc)[3]) {
  acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[0], a[1], acc[0], 0, 0, 0);
  acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[1], a[0], acc[1], 0, 0, 0);
  acc[2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[0], a[0], acc[2], 0, 0, 0);
}

// Workgroups in a row of the grid: 2^22 of them, a matrix each, would be 2^32 threads
// on one axis, one more than a launch takes.
constexpr int kSmallRow = 1 << 20;

// NB: blocks of 16 along P.
template <int NB>
__global__ __launch_bounds__(kSmallWaves * 64) void ns_small(Source s, SmallArgs a, NsArgs to, int count) {
  constexpr int P = 16 * NB, PA = P + 8, kBlocks = NB * (NB + 1) / 2, kHeld = (kBlocks + kSmallWaves - 1) / kSmallWaves;
  __shared__ __attribute__((aligned(16))) char lds[kSmallLds];
  __shared__ double red[kSmallWaves];
  const int PX = a.Q + 8;
  half_t* X[2] = {reinterpret_cast<half_t*>(lds), reinterpret_cast<half_t*>(lds) + P * PX};
  half_t* A[2] = {X[1] + P * PX, X[1] + P * PX + P * PA};
  constexpr int kThreads = kSmallWaves * 64;
  const int mat = blockIdx.y * kSmallRow + blockIdx.x, tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  if (mat >= count) return;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the momentum's update and the norm, then X; kBatch loads a thread under way
  constexpr int kBatch = 8;
  const int n = s.rows * s.cols;
  const int64_t base = mat * s.stride;
  auto batch = [&](int i0, float (&v)[kBatch], bool first) {
    float m[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int64_t i = base + min(i0 + k * kThreads, n - 1);
      if (s.g) {
        v[k] = s.g[i];
        m[k] = s.m[i];
      } else {
        v[k] = s.bf16_in ? to_f(static_cast<const bf16*>(s.x)[i]) : static_cast<const float*>(s.x)[i];
      }
    }
    if (s.g) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (first) {
          m[k] = fmaf(s.beta, m[k], v[k]);
          if (i0 + k * kThreads < n) s.m[base + i0 + k * kThreads] = m[k];
        }
        v[k] = s.nesterov ? fmaf(s.beta, m[k], v[k]) : m[k];
      }
    }
  };
  double sum = 0.0;
  for (int i0 = tid; i0 < n; i0 += kBatch * kThreads) {
    float v[kBatch];
    batch(i0, v, true);
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (i0 + k * kThreads < n) sum = fma((double)v[k], (double)v[k], sum);
  }
  sum = wave_sum_d(sum);
  if (lane == 0) red[wave] = sum;
  for (int i = tid; i < P * PX / 4; i += kThreads)
    reinterpret_cast<uint2*>(X[0])[i] = reinterpret_cast<uint2*>(X[1])[i] = make_uint2(0, 0);
  __syncthreads();
  double norm2 = 0.0;
  for (int w = 0; w < kSmallWaves; ++w) norm2 += red[w];
  const double inv = norm2 == 0.0 ? 0.0 : norm2 <= 1.7e308 ? (double)a.x_scale / sqrt(norm2) : __builtin_nan("");
  for (int i0 = tid; i0 < n; i0 += kBatch * kThreads) {
    float u[kBatch];
    batch(i0, u, false);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int i = i0 + b * kThreads;
      if (i >= n) continue;
      const int r = i / s.cols, k = i % s.cols, at = (a.flip ? k : r) * PX + (a.flip ? r : k);
      const float v = (float)((double)u[b] * inv);
      const half_t hi = static_cast<half_t>(v);
      X[0][at] = hi;
      X[1][at] = static_cast<half_t>(v - static_cast<float>(hi));
    }
  }
  __syncthreads();

  int bi[kHeld], bj[kHeld];  // this wavefront's blocks of A and B
#pragma unroll
  for (int i = 0; i < kHeld; ++i) triangle(min(wave + i * kSmallWaves, kBlocks - 1), bi[i], bj[i]);
  // four elements of a symmetric matrix, and their mirror images
  auto write_a = [&](int bi, int bj, const float (&v)[4]) {
    uint2 hi, lo;
    split4(v, hi, lo);
    const int m = 16 * bi + c, k = 16 * bj + 4 * g;
    *reinterpret_cast<uint2*>(A[0] + m * PA + k) = hi;
    *reinterpret_cast<uint2*>(A[1] + m * PA + k) = lo;
    if (bi != bj) {
      union { uint2 w; half_t h[4]; } h{hi}, l{lo};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        A[0][(k + e) * PA + m] = h.h[e];
        A[1][(k + e) * PA + m] = l.h[e];
      }
    }
  };
  for (int step = 0; step < a.steps; ++step) {
    // A = X X^T, blocks on and below the diagonal
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if (wave + i * kSmallWaves < kBlocks) {
        f32x4_t acc[3] = {};
        for (int k = 0; k < a.Q; k += 64) {
          halfx8_t x[2][2], y[2][2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              x[w][h] = row8(X[h], PX, 16 * bi[i], k + 32 * w, lane);
              y[w][h] = row8(X[h], PX, 16 * bj[i], k + 32 * w, lane);
            }
          mma3(x[0], y[0], acc);
          mma3(x[1], y[1], acc);
        }
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = ((acc[0][e] + acc[1][e]) + acc[2][e]) * a.a_scale;
        write_a(bi[i], bj[i], v);
      }
    }
    __syncthreads();
    // B = a I + b A + c A A, held in registers until A has been read
    float held[kHeld][4];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if (wave + i * kSmallWaves < kBlocks) {
        f32x4_t acc[3] = {};
#pragma unroll
        for (int k = 0; k < P; k += 32) {
          const halfx8_t x[2] = {row8(A[0], PA, 16 * bi[i], k, lane), row8(A[1], PA, 16 * bi[i], k, lane)};
          const halfx8_t y[2] = {row8(A[0], PA, 16 * bj[i], k, lane), row8(A[1], PA, 16 * bj[i], k, lane)};
          mma3(x, y, acc);
        }
        const int m = 16 * bi[i] + c, k = 16 * bj[i] + 4 * g;
        float old[4];
        join4(*reinterpret_cast<const uint2*>(A[0] + m * PA + k), *reinterpret_cast<const uint2*>(A[1] + m * PA + k), old);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          held[i][e] = fmaf((acc[0][e] + acc[1][e]) + acc[2][e], a.c_scale, fmaf(a.cb, old[e], m == k + e ? a.ca : 0.f));
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (wave + i * kSmallWaves < kBlocks) write_a(bi[i], bj[i], held[i]);
    __syncthreads();
    // X <- B X: a wavefront owns whole columns, so it may write where it has read
    const bool last = step + 1 == a.steps;
    for (int col = wave; col < a.Q / 16; col += kSmallWaves) {
      f32x4_t acc[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < P; k += 32) {
        const halfx8_t y[2] = {col8(X[0], PX, 16 * col, k, lane), col8(X[1], PX, 16 * col, k, lane)};
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const halfx8_t x[2] = {row8(A[0], PA, 16 * i, k, lane), row8(A[1], PA, 16 * i, k, lane)};
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y[0], x[1], acc[i], 0, 0, 0);
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y[1], x[0], acc[i], 0, 0, 0);
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y[0], x[0], acc[i], 0, 0, 0);
        }
      }
      wave_lds_order();
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int m = 16 * i + c, k = 16 * col + 4 * g;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][e];
        if (!last) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] *= a.apply_scale;
          uint2 hi, lo;
          split4(v, hi, lo);
          *reinterpret_cast<uint2*>(X[0] + m * PX + k) = hi;
          *reinterpret_cast<uint2*>(X[1] + m * PX + k) = lo;
        } else if (a.flip || !to.r.vec) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int row = a.flip ? k + e : m, at = a.flip ? m : k + e;
            put_one(to, mat, row, at, v[e], ask_one(to, mat, row, at));
          }
        } else {
          Beside w;
          ask<LAST>(to, mat, m, k, w);
          put<LAST>(to, mat, m, k, make_float4(v[0], v[1], v[2], v[3]), w);
        }
      }
      wave_lds_order();
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- sizes --
int pad(int n) { return (n + kTile - 1) / kTile * kTile; }
int64_t up(int64_t n) { return (n + 255) / 256 * 256; }

struct Sizes {
  int P, Q;
  int64_t x, a;  // bytes of one matrix's X and A, one part
  int chunk;     // matrices that go through together
  int nparts;
  int64_t part;  // bytes of the ranges' sums
};

// Matrices go through in as few batches of one size as keep the workspace near 2
// GiB (batches that fit the last-level cache instead, of 8 and 4 of 12 matrices of
// 768 x 4608, took 220 us of a product's time where all 12 together take 105: what
// counts is that a launch fills the chip).
Sizes sizes(const NewtonSchulz& s) {
  Sizes z;
  z.P = pad(std::min(s.rows, s.cols));
  z.Q = pad(std::max(s.rows, s.cols));
  z.x = (int64_t)z.P * z.Q * 2;
  z.a = (int64_t)z.P * z.P * 2;
  const int64_t most = std::max<int64_t>(1, ((int64_t)2 << 30) / (4 * z.x + 4 * z.a));
  const int64_t batches = (s.count + most - 1) / most;
  z.chunk = (int)((s.count + batches - 1) / batches);
  z.nparts = (int)std::min<int64_t>(kNormParts, ((int64_t)s.rows * s.cols + 4095) / 4096);
  z.part = 0;
  for (int n : {z.chunk, s.count % z.chunk})  // (a last batch may be smaller, and X X^T cut)
    if (n) z.part = std::max(z.part, plan_gram(z.P, z.Q, n).part());
  return z;
}

// The power of two that takes values up to `bound` below fp16's largest; at most 40,
// which keeps the products of scales in fp32's range (a bound of zero has no largest).
int exponent(double bound) {
  const double e = std::floor(std::log2(32768.0 / bound));
  return e < 40.0 ? (int)e : 40;
}

// The largest |f(t)| of a quadratic c0 + c1 t + c2 t^2 on [0, top].
double largest(double c0, double c1, double c2, double top) {
  auto f = [&](double t) { return std::fabs(c0 + t * (c1 + t * c2)); };
  double m = std::max(f(0.0), f(top));
  const double t = c2 != 0.0 ? -c1 / (2.0 * c2) : -1.0;
  return t > 0.0 && t < top ? std::max(m, f(t)) : m;
}

// Whether a matrix fits one workgroup, and its padded sides there.
bool small(const NewtonSchulz& s, SmallArgs* a) {
  a->P = (std::min(s.rows, s.cols) + 31) / 32 * 32;
  a->Q = (std::max(s.rows, s.cols) + 63) / 64 * 64;
  return a->P <= kSmallSide && 4ll * a->P * (a->Q + 8) + 4ll * a->P * (a->P + 8) <= kSmallLds;
}

}  // namespace

// Bounds of the singular values before each step (and after the last), of
// sigma (a + b sigma^2 + c sigma^4) from sigma <= 1; false where they pass 2^20.
bool newton_schulz_bounds(const NewtonSchulz& s, double* sigma) {
  sigma[0] = 1.0 + 1e-6;
  for (int k = 0; k < s.steps; ++k) {
    const double a = s.a, b = s.b, c = s.c, top = sigma[k];
    auto f = [&](double x) { return std::fabs(x * (a + x * x * (b + x * x * c))); };
    double m = f(top);
    // where a + 3 b t + 5 c t^2 = 0, t = sigma^2
    const double disc = 9.0 * b * b - 20.0 * a * c;
    double roots[2] = {-1.0, -1.0};
    if (c != 0.0 && disc >= 0.0) {
      roots[0] = (-3.0 * b + std::sqrt(disc)) / (10.0 * c);
      roots[1] = (-3.0 * b - std::sqrt(disc)) / (10.0 * c);
    } else if (c == 0.0 && b != 0.0) {
      roots[0] = -a / (3.0 * b);
    }
    for (double t : roots)
      if (t > 0.0 && t < top * top) m = std::max(m, f(std::sqrt(t)));
    // (roundings move a singular value by far less than this)
    sigma[k + 1] = m * (1.0 + 1e-3) + 1e-6;
    if (!(sigma[k + 1] < 1048576.0) || !(largest(a, b, c, top * top) < 1048576.0)) return false;
  }
  return true;
}

namespace {

// The whole call in one launch, with one set of scales: where the singular values'
// bounds of all steps lie within a factor of 16 (each factor of two costs the
// smallest elements a bit).
bool small_scales(const NewtonSchulz& s, const double* sigma, SmallArgs* a) {
  if (!small(s, a)) return false;
  double most = sigma[0], least = sigma[0], factor = 0.0;
  for (int k = 0; k < s.steps; ++k) {
    most = std::max(most, sigma[k]);
    least = std::min(least, sigma[k]);
    factor = std::max(factor, std::max(largest(s.a, s.b, s.c, sigma[k] * sigma[k]), std::fabs((double)s.a)));
  }
  if (most > 16.0 * least) return false;
  const int ex = exponent(most), ea = exponent(most * most), eb = exponent(factor);
  auto p2 = [](double v, int e) { return (float)std::ldexp(v, e); };
  a->flip = s.rows > s.cols;
  a->steps = s.steps;
  a->x_scale = p2(1.0, ex);
  a->a_scale = p2(1.0, ea - 2 * ex);
  a->c_scale = p2(s.c, eb - 2 * ea);
  a->ca = p2(s.a, eb);
  a->cb = p2(s.b, eb - ea);
  a->apply_scale = p2(1.0, -eb);
  a->out_scale = p2(1.0, -eb - ex);
  return true;
}

}  // namespace

int64_t newton_schulz_scratch(const NewtonSchulz& s) {
  double sigma[kMaxNewtonSteps + 1];
  SmallArgs a;
  if (newton_schulz_bounds(s, sigma) && small_scales(s, sigma, &a)) return 256;  // (none is used)
  const Sizes z = sizes(s);
  return up((int64_t)s.count * z.nparts * 8) + z.chunk * (4 * up(z.x) + 4 * up(z.a)) + z.part;
}

hipError_t newton_schulz(const NewtonSchulz& s, const MuonArgs* u, const void* x, void* out, void* scratch,
                         hipStream_t stream) {
  const Sizes z = sizes(s);
  double sigma[kMaxNewtonSteps + 1];
  if (!newton_schulz_bounds(s, sigma)) return hipErrorInvalidValue;
  const int flip = s.rows > s.cols;
  double* part = static_cast<double*>(scratch);
  char* base = static_cast<char*>(scratch) + up((int64_t)s.count * z.nparts * 8);
  auto take = [&](int64_t bytes) {
    half_t* t = reinterpret_cast<half_t*>(base);
    base += bytes;
    return t;
  };
  Split X[2], A, B;
  for (Split* m : {&X[0], &X[1]}) { m->hi = take(z.chunk * up(z.x)); m->lo = take(z.chunk * up(z.x)); }
  for (Split* m : {&A, &B}) { m->hi = take(z.chunk * up(z.a)); m->lo = take(z.chunk * up(z.a)); }
  float* sums = reinterpret_cast<float*>(base);

  Source src;
  memset(&src, 0, sizeof(src));
  src.x = x;
  src.bf16_in = s.dt == BF16;
  src.rows = s.rows; src.cols = s.cols; src.stride = s.stride;
  if (u) { src.g = u->grads; src.m = u->momentum; src.beta = u->beta; src.nesterov = u->nesterov; }
  Result res;
  memset(&res, 0, sizeof(res));
  res.rows = s.rows; res.cols = s.cols; res.flip = flip; res.stride = u ? s.stride : s.out_stride;
  res.out = out; res.bf16_out = s.dt == BF16;
  if (u) { res.master = u->master; res.decay = u->decay; res.step = u->step; }

  auto whole = [](const void* q, int64_t bytes) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && bytes % 16 == 0; };
  const int64_t es = s.dt == BF16 ? 2 : 4, each = (int64_t)s.rows * s.cols;
  const bool vec_in = u ? whole(u->grads, each * 4) && whole(u->momentum, s.stride * 4)
                        : whole(x, each * es) && s.stride * es % 16 == 0;
  // four columns of every row at once
  res.vec = s.cols % 4 == 0 && res.stride % 4 == 0 && reinterpret_cast<uintptr_t>(out) % (4 * es) == 0 &&
            (!u || reinterpret_cast<uintptr_t>(u->master) % 16 == 0);

  SmallArgs one;
  if (small_scales(s, sigma, &one)) {
    NsArgs to;
    memset(&to, 0, sizeof(to));
    to.r = res;
    to.scale = one.out_scale;
    const int row = std::min(s.count, kSmallRow);
    const dim3 grid(row, cdiv(s.count, row)), block(kSmallWaves * 64);
    switch (one.P) {
      case 32: hipLaunchKernelGGL(ns_small<2>, grid, block, 0, stream, src, one, to, s.count); break;
      case 64: hipLaunchKernelGGL(ns_small<4>, grid, block, 0, stream, src, one, to, s.count); break;
      case 96: hipLaunchKernelGGL(ns_small<6>, grid, block, 0, stream, src, one, to, s.count); break;
      default: hipLaunchKernelGGL(ns_small<8>, grid, block, 0, stream, src, one, to, s.count); break;
    }
    return hipGetLastError();
  }

  hipError_t e = hipSuccess;
  for (int c0 = 0; c0 < s.count && e == hipSuccess; c0 += z.chunk) {
    const int n = std::min(z.chunk, s.count - c0);
    const int64_t at = c0 * s.stride;
    Source in = src;
    Result to = res;
    if (u) { in.g += at; in.m += at; to.master += at; }
    else in.x = static_cast<const char*>(x) + at * (s.dt == BF16 ? 2 : 4);
    if (out) to.out = static_cast<char*>(out) + c0 * res.stride * (s.dt == BF16 ? 2 : 4);
    if (vec_in) hipLaunchKernelGGL(ns_norm<1>, dim3(z.nparts, n), dim3(256), 0, stream, in, part);
    else hipLaunchKernelGGL(ns_norm<0>, dim3(z.nparts, n), dim3(256), 0, stream, in, part);
    int ex = exponent(sigma[0]);
    hipLaunchKernelGGL(ns_first, dim3(z.Q / 64, z.P / 64, n), dim3(256), 0, stream, in, part, z.nparts, flip, X[0], z.P,
                       z.Q, (float)std::ldexp(1.0, ex));
    for (int k = 0; k < s.steps; ++k) {
      const Split &x0 = X[k & 1], &x1 = X[~k & 1];
      const double top = sigma[k] * sigma[k];
      const int ea = exponent(top), eb = exponent(std::max(largest(s.a, s.b, s.c, top), std::fabs((double)s.a))),
                en = exponent(sigma[k + 1]);
      const int64_t sx = (int64_t)z.P * z.Q, sp = (int64_t)z.P * z.P;
      NsArgs p;
      memset(&p, 0, sizeof(p));
      p.part = sums;
      // A = X X^T
      p.a = p.b = x0; p.lda = p.ldb = z.Q; p.sa = p.sb = sx; p.K = z.Q;
      p.c = A; p.ldc = z.P; p.sc = sp;
      p.M = p.N = z.P;
      p.scale = (float)std::ldexp(1.0, ea - 2 * ex);
      launch<GRAM>(p, n, stream);
      // B = a I + b A + c A A
      p.a = p.b = p.d = A; p.lda = p.ldb = p.ldd = z.P; p.sa = p.sb = p.sd = sp; p.K = z.P;
      p.c = B;
      p.scale = (float)std::ldexp((double)s.c, eb - 2 * ea);
      p.ca = (float)std::ldexp((double)s.a, eb);
      p.cb = (float)std::ldexp((double)s.b, eb - ea);
      launch<POLY>(p, n, stream);
      // X <- B X
      p.a = B; p.b = x0; p.ldb = z.Q; p.sb = sx;
      p.c = x1; p.ldc = z.Q; p.sc = sx;
      p.N = z.Q;
      if (k + 1 < s.steps) {
        p.scale = (float)std::ldexp(1.0, en - eb - ex);
        launch<APPLY>(p, n, stream);
      } else {
        p.scale = (float)std::ldexp(1.0, -eb - ex);
        p.r = to;
        launch<LAST>(p, n, stream);
      }
      ex = en;
    }
    e = hipGetLastError();
  }
  return e;
}

}  // namespace fal
