// Norms of queries and keys head by head, and the rotation of their positions,
// in one pass over packed [Q | K | V] rows.
//
// For a head x of hd elements with weight w, at position t:
//   hat = x / sqrt(mean(x^2) + eps),  n = hat w,
//   out = n with the pairs (n_a, n_b) of its first r elements turned by
//         t theta^(-2j/r), j the pair's number; V heads are copied.
// Backward, with dn = the gradient turned back:
//   dw = sum over tokens and heads of dn hat,
//   dx = (dn w - hat mean(dn w hat)) / sqrt(mean(x^2) + eps).
//
// Bound by memory: a row is read and written once (backward: rows and their
// gradients read, the new gradients written).  A wavefront owns a token; a lane
// owns eight consecutive elements of a head (16 bytes of bf16), so hd / 8 lanes
// hold a head and one access of the wavefront covers 512 elements of the row.
// All heads of a token share its angles: lane j computes the j-th pair's once,
// and the wavefront passes them round through LDS.  Angles are products in fp64,
// reduced to a turn before their sine and cosine in fp32: a position of 10^6
// loses nothing.  The next heads are asked for while one group of heads is worked on.
// Measured: 8 x 1024 tokens, 36 heads of 64 in bf16 17.5 us forward and 21.3
// backward (4.3 and 4.7 TB/s; a large copy reaches 4.9), 2 x 8192 tokens, 48 heads
// of 128 87 and 120 us (4.6 and 4.75).
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace fal {

namespace {

constexpr int kWaves = 4;
constexpr int kMaxPairs = 64;  // half of the widest head
// Workgroups of the backward, each with a row of the weights' sums: three a compute
// unit, what its registers allow at once (2 x 8192 tokens, 48 heads of 128: 120 us,
// the rate of a copy; with 1024, a third of which wait, 146; with 1024 at four a
// compute unit and registers in memory 130).
constexpr int kBwdBlocks = 768;

// Eight elements as they lie in memory, and widened.
template <typename T> struct Raw;
template <> struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<float4*>(p) = a;
    *reinterpret_cast<float4*>(p + 4) = b;
  }
};
template <> struct Raw<bf16> {
  uint4 w;
  __device__ __forceinline__ void load(const bf16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ void store(bf16* p) const { *reinterpret_cast<uint4*>(p) = w; }
};
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  union { bf16 h[8]; uint4 w; } u;
#pragma unroll
  for (int i = 0; i < 8; ++i) u.h[i] = from_f<bf16>(v[i]);
  *reinterpret_cast<uint4*>(p) = u.w;
}

// Sum over the G lanes of a head.
template <int G>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, FAL_WAVE);
  return v;
}

// The rotation of one lane's eight elements: element e becomes
// e cos + partner sin, sin with the partner's sign.
struct Turn {
  float c[8], s[8];
};

// How pairs lie: neighbours (2j, 2j + 1), or (j, j + r/2) with r/2 a multiple
// of 8 (the partner is the same element of another lane) or of 4 (the
// other half of another lane's eight).
enum Pairs : int { PAIRS_NEXT = 0, PAIRS_HALF8 = 1, PAIRS_HALF4 = 2 };

template <int PAIRS>
__device__ __forceinline__ void rotate(float (&v)[8], const Turn& t, int from_lo, int from_hi) {
  float o[8];
  if (PAIRS == PAIRS_NEXT) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = v[i ^ 1];
  } else if (PAIRS == PAIRS_HALF8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __shfl(v[i], from_lo, FAL_WAVE);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = __shfl(v[i ^ 4], i < 4 ? from_lo : from_hi, FAL_WAVE);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], t.c[i], o[i] * t.s[i]);
}

// What a lane knows before its first token.
template <int HD, int PAIRS>
struct Lane {
  static constexpr int G = HD / 8;      // lanes of a head
  static constexpr int HPW = 64 / G;    // heads a wavefront holds at once
  int head0, e0;                        // its head among those, its first element
  int from_lo, from_hi;                 // lanes that hold the partners of elements 0..3, 4..7
  double rate;                          // turns a position of pair `lane`
  __device__ __forceinline__ Lane(const HeadNorm& a, int lane) {
    head0 = lane / G;
    e0 = lane % G * 8;
    const int half = a.rotary / 2;
    auto partner = [&](int e) { return e < half ? e + half : e < a.rotary ? e - half : e; };
    from_lo = head0 * G + partner(e0) / 8;
    from_hi = head0 * G + partner(e0 + 4) / 8;
    // theta^(-2j/r) / (2 pi)
    rate = lane < half ? exp2(-lane * a.log2_theta_step) * 0.15915494309189535 : 0.0;
  }
  // The token's rotation, `table` being the wavefront's part of LDS; sign -1
  // turns back.
  __device__ __forceinline__ void turn(const HeadNorm& a, int64_t position, float sign, int lane, float2* table,
                                       Turn& t) const {
    const double turns = (double)position * rate;
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    __builtin_amdgcn_wave_barrier();
    table[lane] = make_float2(c, sign * s);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int half = a.rotary / 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = e0 + i;
      const bool second = PAIRS == PAIRS_NEXT ? i & 1 : e >= half;
      const int j = PAIRS == PAIRS_NEXT ? e / 2 : second ? e - half : e;
      const float2 cs = table[min(j, kMaxPairs - 1)];
      t.c[i] = e < a.rotary ? cs.x : 1.f;
      t.s[i] = e < a.rotary ? (second ? cs.y : -cs.y) : 0.f;
    }
  }
};

template <typename T>
__device__ __forceinline__ void weight8(const void* w, int e0, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = w ? to_f(static_cast<const T*>(w)[e0 + i]) : 1.f;
}

__device__ __forceinline__ bool live_token(const HeadNorm& a, int64_t m) {
  return !a.lens || (int)(m % a.T) < a.lens[m / a.T];
}
__device__ __forceinline__ int64_t position_of(const HeadNorm& a, int64_t m) {
  return a.positions ? (int64_t)a.positions[m] : m % a.T;
}

template <typename T, int HD, int PAIRS>
__global__ __launch_bounds__(kWaves * 64) void head_norm_fwd(HeadNorm a, const T* x, T* out) {
  typedef Lane<HD, PAIRS> L;
  __shared__ float2 table[kWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const L l(a, lane);
  float wq[8], wk[8];
  weight8<T>(a.wq, l.e0, wq);
  weight8<T>(a.wk, l.e0, wk);
  const int turned = a.H + a.Hkv, all = turned + a.Hkv;
  const bool in_place = x == out;
  for (int64_t m = (int64_t)blockIdx.x * kWaves + wave; m < a.tokens; m += (int64_t)gridDim.x * kWaves) {
    const T* xr = x + m * a.ldx + l.e0;
    T* yr = out + m * a.ldy + l.e0;
    if (!live_token(a, m)) {
      const float zero[8] = {};
      for (int h = l.head0; h < all; h += L::HPW) store8(yr + (int64_t)h * HD, zero);
      continue;
    }
    // (heads past the last one repeat it and are not stored: whole wavefronts run
    // the loop, since sums and partners come from other lanes)
    Raw<T> next;
    next.load(xr + (int64_t)min(l.head0, turned - 1) * HD);
    Turn t;
    l.turn(a, position_of(a, m), 1.f, lane, table[wave], t);
    for (int h0 = 0; h0 < turned; h0 += L::HPW) {
      const int h = h0 + l.head0;
      float v[8];
      next.get(v);
      if (h0 + L::HPW < turned) next.load(xr + (int64_t)min(h + L::HPW, turned - 1) * HD);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[i], v[i], sum);
      const float rstd = 1.f / sqrtf(head_sum<L::G>(sum) * (1.f / HD) + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = v[i] * rstd * (h < a.H ? wq[i] : wk[i]);
      rotate<PAIRS>(v, t, l.from_lo, l.from_hi);
      if (h < turned) store8(yr + (int64_t)h * HD, v);
    }
    if (!in_place)
      for (int h = turned + l.head0; h < all; h += L::HPW) {
        next.load(xr + (int64_t)h * HD);
        next.store(yr + (int64_t)h * HD);
      }
  }
}

// part: [gridDim.x][2][HD], a workgroup's sums for both weights (NULL: none
// are asked for).
template <typename T, int HD, int PAIRS>
__global__ __launch_bounds__(kWaves * 64) void head_norm_bwd(HeadNorm a, const T* x, const T* dout, T* dx, float* part) {
  typedef Lane<HD, PAIRS> L;
  __shared__ float2 table[kWaves][64];
  __shared__ float sums[kWaves][2][HD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const L l(a, lane);
  float wq[8], wk[8], dwq[8] = {}, dwk[8] = {};
  weight8<T>(a.wq, l.e0, wq);
  weight8<T>(a.wk, l.e0, wk);
  const int turned = a.H + a.Hkv, all = turned + a.Hkv;
  const bool in_place = dout == dx;
  for (int64_t m = (int64_t)blockIdx.x * kWaves + wave; m < a.tokens; m += (int64_t)gridDim.x * kWaves) {
    const T* xr = x + m * a.ldx + l.e0;
    const T* gr = dout + m * a.ldy + l.e0;
    T* dr = dx + m * a.lddx + l.e0;
    if (!live_token(a, m)) {
      const float zero[8] = {};
      for (int h = l.head0; h < all; h += L::HPW) store8(dr + (int64_t)h * HD, zero);
      continue;
    }
    Raw<T> nx, ng;
    nx.load(xr + (int64_t)min(l.head0, turned - 1) * HD);
    ng.load(gr + (int64_t)min(l.head0, turned - 1) * HD);
    Turn t;
    l.turn(a, position_of(a, m), -1.f, lane, table[wave], t);
    for (int h0 = 0; h0 < turned; h0 += L::HPW) {
      const int h = h0 + l.head0;
      float v[8], g[8];
      nx.get(v);
      ng.get(g);
      if (h0 + L::HPW < turned) {
        nx.load(xr + (int64_t)min(h + L::HPW, turned - 1) * HD);
        ng.load(gr + (int64_t)min(h + L::HPW, turned - 1) * HD);
      }
      if (h >= turned) {  // adds nothing to the weights' sums
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 0.f;
      }
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[i], v[i], sum);
      const float rstd = 1.f / sqrtf(head_sum<L::G>(sum) * (1.f / HD) + a.eps);
      rotate<PAIRS>(g, t, l.from_lo, l.from_hi);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] *= rstd;
        const float d = g[i] * v[i];
        if (h < a.H) dwq[i] += d;
        else dwk[i] += d;
        g[i] *= h < a.H ? wq[i] : wk[i];
        dot = fmaf(g[i], v[i], dot);
      }
      dot = head_sum<L::G>(dot) * (1.f / HD);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = rstd * fmaf(-v[i], dot, g[i]);
      if (h < turned) store8(dr + (int64_t)h * HD, g);
    }
    if (!in_place)
      for (int h = turned + l.head0; h < all; h += L::HPW) {
        ng.load(gr + (int64_t)h * HD);
        ng.store(dr + (int64_t)h * HD);
      }
  }
  if (!part) return;
  // lanes of the same elements, then the wavefronts, in a fixed order
#pragma unroll
  for (int i = 0; i < 8; ++i) {
#pragma unroll
    for (int o = 32; o >= L::G; o >>= 1) {
      dwq[i] += __shfl_xor(dwq[i], o, FAL_WAVE);
      dwk[i] += __shfl_xor(dwk[i], o, FAL_WAVE);
    }
    if (lane < L::G) {
      sums[wave][0][l.e0 + i] = dwq[i];
      sums[wave][1][l.e0 + i] = dwk[i];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * HD; i += kWaves * 64) {
    const int w = i / HD, e = i % HD;
    part[(int64_t)blockIdx.x * 2 * HD + i] = (sums[0][w][e] + sums[1][w][e]) + (sums[2][w][e] + sums[3][w][e]);
  }
}

// dw[e] = sum over workgroups of part[b][e], in fp64: 16 columns a workgroup,
// 64 threads a column, whose loads are all under way at once (16 threads a
// column that waited for each took 17 us for 1024 rows of 128, these 6.7, and 5.4
// for 768).
__global__ __launch_bounds__(1024) void head_norm_weights(const float* part, int nblk, int hd, float* dwq, float* dwk) {
  __shared__ double red[64][17];
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4, e = blockIdx.x * 16 + c;
  float v[kBwdBlocks / 64];
#pragma unroll
  for (int i = 0; i < kBwdBlocks / 64; ++i) v[i] = r + 64 * i < nblk ? part[(int64_t)(r + 64 * i) * 2 * hd + e] : 0.f;
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kBwdBlocks / 64; ++i) s += v[i];
  red[r][c] = s;
  __syncthreads();
  if (r >= 4) return;
  s = red[r][c];
#pragma unroll
  for (int i = 1; i < 16; ++i) s += red[r + 4 * i][c];
  red[r][c] = s;
  // (threads 0 .. 63 are one wavefront)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  if (r) return;
  s = (red[0][c] + red[1][c]) + (red[2][c] + red[3][c]);
  float* out = e < hd ? dwq : dwk;
  if (out) out[e % hd] = (float)s;
}

int fwd_blocks(const HeadNorm& a) { return (int)std::min<int64_t>((a.tokens + kWaves - 1) / kWaves, 1 << 20); }
int bwd_blocks(const HeadNorm& a) { return (int)std::min<int64_t>((a.tokens + kWaves - 1) / kWaves, kBwdBlocks); }

template <typename T, int HD>
hipError_t fwd(const HeadNorm& a, const T* x, T* out, hipStream_t s) {
  const dim3 grid(fwd_blocks(a)), block(kWaves * 64);
  if (a.interleaved) hipLaunchKernelGGL((head_norm_fwd<T, HD, PAIRS_NEXT>), grid, block, 0, s, a, x, out);
  else if (a.rotary % 16 == 0) hipLaunchKernelGGL((head_norm_fwd<T, HD, PAIRS_HALF8>), grid, block, 0, s, a, x, out);
  else hipLaunchKernelGGL((head_norm_fwd<T, HD, PAIRS_HALF4>), grid, block, 0, s, a, x, out);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t bwd(const HeadNorm& a, const T* x, const T* dout, T* dx, float* part, hipStream_t s) {
  const dim3 grid(bwd_blocks(a)), block(kWaves * 64);
  if (a.interleaved) hipLaunchKernelGGL((head_norm_bwd<T, HD, PAIRS_NEXT>), grid, block, 0, s, a, x, dout, dx, part);
  else if (a.rotary % 16 == 0)
    hipLaunchKernelGGL((head_norm_bwd<T, HD, PAIRS_HALF8>), grid, block, 0, s, a, x, dout, dx, part);
  else hipLaunchKernelGGL((head_norm_bwd<T, HD, PAIRS_HALF4>), grid, block, 0, s, a, x, dout, dx, part);
  return hipGetLastError();
}

}  // namespace

hipError_t head_norm_rope_fwd(DType dt, const HeadNorm& a, const void* x, void* out, hipStream_t s) {
#define FAL_FWD(HD)                                                                                          \
  case HD:                                                                                                   \
    return dt == BF16 ? fwd<bf16, HD>(a, static_cast<const bf16*>(x), static_cast<bf16*>(out), s)            \
                      : fwd<float, HD>(a, static_cast<const float*>(x), static_cast<float*>(out), s);
  switch (a.hd) {
    FAL_FWD(16) FAL_FWD(32) FAL_FWD(64) FAL_FWD(128)
  }
#undef FAL_FWD
  return hipErrorInvalidValue;
}

int64_t head_norm_rope_scratch(const HeadNorm& a) { return (int64_t)bwd_blocks(a) * 2 * a.hd; }

hipError_t head_norm_rope_bwd(DType dt, const HeadNorm& a, const void* x, const void* dout, void* dx, float* dwq,
                              float* dwk, float* part, hipStream_t s) {
  float* sums = dwq || dwk ? part : nullptr;
  hipError_t e = hipErrorInvalidValue;
#define FAL_BWD(HD)                                                                                             \
  case HD:                                                                                                      \
    e = dt == BF16 ? bwd<bf16, HD>(a, static_cast<const bf16*>(x), static_cast<const bf16*>(dout),              \
                                   static_cast<bf16*>(dx), sums, s)                                             \
                   : bwd<float, HD>(a, static_cast<const float*>(x), static_cast<const float*>(dout),           \
                                    static_cast<float*>(dx), sums, s);                                          \
    break;
  switch (a.hd) {
    FAL_BWD(16) FAL_BWD(32) FAL_BWD(64) FAL_BWD(128)
  }
#undef FAL_BWD
  if (e != hipSuccess || !sums) return e;
  hipLaunchKernelGGL(head_norm_weights, dim3(2 * a.hd / 16), dim3(1024), 0, s, part, bwd_blocks(a), a.hd, dwq, dwk);
  return hipGetLastError();
}

}  // namespace fal
