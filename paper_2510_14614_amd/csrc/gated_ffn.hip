// The gated feed-forward block y = (act(x Wg) * (x Wu)) Wd and its gradients.
//
//   g = x Wg, u = x Wu, h = act(g) u, y = h Wd                      (forward)
//   dh = dy Wd^T, dg = dh u act'(g), du = dh act(g),
//   dx = dg Wg^T + du Wu^T, dWg = x^T dg, dWu = x^T du, dWd = h^T dy (backward)
//
// Bound by the matrix cores: 6 M d f operations forward, 12 M d f backward.
// In bf16 two products run here: both projections in one kernel, whose tile
// holds the same columns of g and u, so that h leaves from the accumulators;
// and dh, whose epilogue reads g and u and writes dg, du and h.  The other
// products are plain and go through gemm().
//
// g and u are kept for the backward in fp32: dg and du multiply them once more,
// and bf16 values would add their rounding to the ones that dg and du, as
// operands, and dx, as the result, cannot do without.
#include <algorithm>
#include <cstring>

#include "common.h"
#include "gemm_pipe.h"
#include "kernels.h"

namespace fal {

namespace {

// The activation and its derivative.  bf16 blocks take the hardware's exp2 and
// reciprocal (one step of fp32 each, far below bf16's), fp32 ones the library's.
template <bool EXACT>
__device__ __forceinline__ void act_and_grad(int act, float x, float& a, float& da) {
  if (act == GATE_GELU_ERF) {
    // erfc keeps the relative accuracy of the left tail
    const float cdf = 0.5f * erfcf(x * -0.7071067811865476f);
    a = x * cdf;
    da = fmaf(x * 0.3989422804014327f, expf(-0.5f * x * x), cdf);
    return;
  }
  float w, slope;  // sigmoid(w), dw/dx
  if (act == GATE_SILU) {
    w = x;
    slope = 1.f;
  } else {
    constexpr float kC = 1.5957691216057308f;  // 2 sqrt(2/pi)
    const float x2 = fminf(x * x, 1e30f);      // keeps 0 * slope from becoming 0 * inf
    w = x * fmaf(x2, kC * 0.044715f, kC);
    slope = fmaf(x2, 3.f * kC * 0.044715f, kC);
  }
  float s;
  if (EXACT) s = 1.f / (1.f + expf(-w));
  else s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(w * -1.4426950408889634f));
  a = x * s;
  da = fmaf(a * (1.f - s), slope, s);
}

struct Gated {
  const bf16 *a, *b0, *b1;  // x, Wg, Wu; or dy, Wd
  int64_t lda, ldb0, ldb1;
  int M, N, K;              // rows, f, d
  int tiles_m, tiles_n, act;
  float* saved;             // [M][2 N]: g | u
  bf16 *h, *dg, *du;        // [M][N]
};

// One output tile of BM rows and BN columns of f.  Forward (BWD 0): both
// projections at once, x k-contiguous, weights MN-major.  Backward: dh, both
// operands k-contiguous.  The main loop is that of gemm_bf16_pipe: three stages of
// 32 k, the fragments of slice s + 1 read under the MFMAs of slice s, slice s + 2
// asked for behind them, one barrier a slice.
template <int BWD, int BM, int BN, int OCC>
__global__ __launch_bounds__(256, OCC) void gated_mfma(Gated p) {
  using namespace pipe;
  constexpr int NB = BWD ? 1 : 2;
  constexpr int WTM = BM / 2, WTN = BN / 2, FM = WTM / 16, FN = WTN / 16;
  typedef Src<BM, 1> SA;
  typedef Src<BN, BWD> SB;
  constexpr int SBYTES = SA::BYTES + NB * SB::BYTES;
  constexpr int L = SA::IPW + NB * SB::IPW;
  // one array a stage: the compiler tracks loads to LDS array by array
  constexpr int NS = 3;
  __shared__ __attribute__((aligned(1024))) char st0[SBYTES], st1[SBYTES], st2[SBYTES];
  auto stage_ptr = [&](int k) -> char* { return k == 0 ? st0 : k == 1 ? st1 : st2; };

  int tmi, tni;
  grouped_tile(xcd_remap(blockIdx.x, p.tiles_m * p.tiles_n), p.tiles_m, p.tiles_n, tmi, tni);
  const int m0 = tmi * BM, n0 = tni * BN;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;

  SA sa;
  SB sb, sc;
  sa.init(0, p.a, p.lda, m0, p.M, p.K, wave, lane);
  sb.init(0, p.b0, p.ldb0, n0, p.N, p.K, wave, lane);
  sa.clear(1);  // one segment only
  sb.clear(1);
  if (NB == 2) {
    sc.init(0, p.b1, p.ldb1, n0, p.N, p.K, wave, lane);
    sc.clear(1);
  }
  const int n = (p.K + KS - 1) / KS;
  // (no branch: slices past the end are out of both operands' ranges and read as
  // zeros, so the main loop is one straight block)
  sa.start(p.lda, m0, p.M, p.K);
  sb.start(p.ldb0, n0, p.N, p.K);
  if (NB == 2) sc.start(p.ldb1, n0, p.N, p.K);
  auto issue = [&](char* stage, int s) {
    sa.limit(p.K - s * KS);
    sb.limit(p.K - s * KS);
    sa.load(stage, wave);
    sb.load(stage + SA::BYTES, wave);
    if (NB == 2) sc.load(stage + SA::BYTES + SB::BYTES, wave);
    sa.advance();
    sb.advance();
    if (NB == 2) sc.advance();
  };

  Frag<BM, 1, FM> fa;
  Frag<BN, BWD, FN> fb;
  fa.init(wm * WTM, lane);
  fb.init(wn * WTN, lane);

  f32x4_t acc[NB][FM][FN];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[b][i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  bf16x8_t ra[2][FM], rb[2][NB][FN];
  auto read_b = [&](const char* stage, int b, int j) {
    return fb.read(stage + SA::BYTES + b * SB::BYTES, j);
  };
  auto read = [&](const char* stage, int buf) {
#pragma unroll
    for (int i = 0; i < FM; ++i) ra[buf][i] = fa.read(stage, i);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < FN; ++j) rb[buf][b][j] = read_b(stage, b, j);
  };
  auto step = [&](const char* stage, int cur) {
    const int nxt = cur ^ 1;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          acc[b][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(rb[cur][b][j], ra[cur][i], acc[b][i][j], 0, 0, 0);
          if (i == FM - 1) rb[nxt][b][j] = read_b(stage, b, j);
        }
      ra[nxt][i] = fa.read(stage, i);
    }
  };
  constexpr int RB = BWD ? 1 : 2;  // LDS reads of a fragment of B
  constexpr int ROW = NB * FN, NMF = FM * ROW;
  constexpr int DMA_EVERY = NMF / L > 0 ? NMF / L : 1;
  auto interleave = [&]() {
    int dma = 0;
#pragma unroll
    for (int q = 0; q < NMF; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
      if (q >= NMF - ROW) {
#pragma unroll
        for (int r = 0; r < RB; ++r) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read (B)
      }
      if ((q + 1) % ROW == 0) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // LDS read (A)
      if (q % DMA_EVERY == 0 && dma < L) {
        __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);  // buffer load to LDS
        ++dma;
      }
    }
  };
  // the reads that a step issues may be in flight at the next one's barrier;
  // the counter holds at most 15
  constexpr int LGK_N = FM + ROW * RB, LGK = LGK_N < 15 ? LGK_N : 15;

#pragma unroll
  for (int k = 0; k < NS - 1; ++k) issue(stage_ptr(k), k);
  FAL_WAITCNT(L * (NS - 2), 0);
  bar();
  read(st0, 0);
  // slices past the end load zeros in both operands and add nothing
  constexpr int UNR = 2 * NS;  // whole cycles of stages and of register buffers
  const int tend = (n + UNR - 1) / UNR * UNR;
  for (int t = 0; t < tend; t += UNR) {
#pragma unroll
    for (int U = 0; U < UNR; ++U) {
      FAL_WAITCNT(L * (NS - 3), LGK);
      bar();
      __builtin_amdgcn_sched_barrier(0);
      issue(stage_ptr((U + NS - 1) % NS), t + U + NS - 1);
      step(stage_ptr((U + 1) % NS), U & 1);
      interleave();
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  FAL_WAITCNT(0, 0);
  bar();

  // Epilogue: strips of 16 rows through LDS, so that consecutive lanes hold
  // consecutive columns; g, u and dh meet in one lane.  A strip goes in units of
  // up to four accesses; the backward asks for the g and u of a unit while it works on
  // the one before (8192 x 5504: 340 us where each access waited for its own, 322 so).
  constexpr int PITCH = NB * WTN + 4, LPR = WTN / 4, RPI = 64 / LPR;
  constexpr int APU = 16 / RPI < 4 ? 16 / RPI : 4, UPS = 16 / RPI / APU;  // accesses a unit, units a strip
  static_assert(2 * 16 * PITCH * 4 <= SBYTES, "epilogue staging");
  float* strip = reinterpret_cast<float*>(wm ? st1 : st0) + wn * 16 * PITCH;
  const int rr = lane / LPR, cc = lane % LPR * 4;
  const int64_t nn = n0 + wn * WTN + cc;
  const int mw = m0 + wm * WTM;
  float4 sg[2][APU], su[2][APU];
  // (addresses past the matrix are held at its end: no branch between the loads)
  const float* saved = p.saved + min(nn, (int64_t)p.N - 4);
  auto ask = [&](int unit) {
#pragma unroll
    for (int k = 0; k < APU; ++k) {
      const int64_t m = min(mw + (APU * unit + k) * RPI + rr, p.M - 1);
      sg[unit & 1][k] = *reinterpret_cast<const float4*>(saved + m * 2 * p.N);
      su[unit & 1][k] = *reinterpret_cast<const float4*>(saved + m * 2 * p.N + p.N);
    }
  };
  if (BWD) ask(0);
#pragma clang loop unroll(full)
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        *reinterpret_cast<float4*>(strip + (lane & 15) * PITCH + b * WTN + 16 * j + 4 * (lane >> 4)) =
            make_float4(acc[b][i][j][0], acc[b][i][j][1], acc[b][i][j][2], acc[b][i][j][3]);
    wave_lds_order();
#pragma unroll
    for (int k = 0; k < APU * UPS; ++k) {
      const int r = k * RPI + rr, unit = i * UPS + k / APU;
      if (BWD && k % APU == 0 && unit + 1 < FM * UPS) ask(unit + 1);
      const int64_t m = mw + 16 * i + r;
      const float4 v0 = *reinterpret_cast<const float4*>(strip + r * PITCH + cc);
      float4 v1 = make_float4(0.f, 0.f, 0.f, 0.f);
      if (NB == 2) v1 = *reinterpret_cast<const float4*>(strip + r * PITCH + WTN + cc);
      // (f is a multiple of 8: a lane's four columns are all inside or none is)
      const bool in = m < p.M && nn < p.N;
      const int64_t o = m * p.N + nn;
      if (!BWD) {
        if (p.saved && in) {
          // (read only by the backward: kept out of the caches)
          __builtin_nontemporal_store(f32x4_t{v0.x, v0.y, v0.z, v0.w},
                                      reinterpret_cast<f32x4_t*>(p.saved + m * 2 * p.N + nn));
          __builtin_nontemporal_store(f32x4_t{v1.x, v1.y, v1.z, v1.w},
                                      reinterpret_cast<f32x4_t*>(p.saved + m * 2 * p.N + p.N + nn));
        }
        const float g[4] = {v0.x, v0.y, v0.z, v0.w}, u[4] = {v1.x, v1.y, v1.z, v1.w};
        float h[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float a, da;
          act_and_grad<false>(p.act, g[c], a, da);
          h[c] = a * u[c];
        }
        if (in) st4(p.h + o, h);
      } else {
        const float4 g4 = sg[unit & 1][k % APU], u4 = su[unit & 1][k % APU];
        const float dh[4] = {v0.x, v0.y, v0.z, v0.w}, g[4] = {g4.x, g4.y, g4.z, g4.w}, u[4] = {u4.x, u4.y, u4.z, u4.w};
        float h[4], dg[4], du[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float a, da;
          act_and_grad<false>(p.act, g[c], a, da);
          h[c] = a * u[c];
          dg[c] = dh[c] * u[c] * da;
          du[c] = dh[c] * a;
        }
        if (in) {
          st4(p.h + o, h);
          st4(p.dg + o, dg);
          st4(p.du + o, du);
        }
      }
    }
    wave_lds_order();
  }
}

// ---------------------------------------------------------- few rows --
// Up to kFew rows of bf16 (single tokens of a few texts) are bound by reading the
// weights once: 67 MB of a 2048 x 5504 block, 14 us at 4.9 TB/s, which tiles of 128
// rows on the few compute units that their columns give took 107 us over.  Plain
// fp32 FMA keep up: M FMA an element and 16 bytes a load.  A workgroup takes 64
// columns (eight lanes of 16 bytes, whole 128-byte lines of the weight's rows) and
// a range of k; each of its 64 groups of lanes takes every 64th k of it, asks for
// its first eight rows of weights before anything else, and the groups are added
// through LDS.
// The ranges' sums go to scratch as fp32 and are added in order by whoever reads
// them: the down-projection for g and u (it applies the activation itself, so h is
// never rounded), a last small kernel for y.
constexpr int kFew = 8;
constexpr int kFewWaves = 8, kFewThreads = kFewWaves * 64, kFewGroups = kFewWaves * 8;
constexpr int kFewBatch = 8;     // rows of weights a lane has under way
constexpr int kFewSplits = 16;   // most ranges of the down-projection

__device__ __forceinline__ void widen8(const uint4& q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// One lane's rows of weights: every kFewGroups-th of [k, k1) from w on.
struct FewRows {
  uint4 q[kFewBatch];
  __device__ __forceinline__ void load(const bf16* w, int64_t ld, int k, int k1) {
#pragma unroll
    for (int i = 0; i < kFewBatch; ++i)
      q[i] = k + i * kFewGroups < k1 ? *reinterpret_cast<const uint4*>(w + (int64_t)i * kFewGroups * ld)
                                     : make_uint4(0, 0, 0, 0);
  }
  // v[m][e] += rows of xs [k][M] times the weights
  template <int M>
  __device__ __forceinline__ void add(const float* xs, int k, int k1, float (&v)[M][8]) const {
#pragma unroll
    for (int i = 0; i < kFewBatch; ++i) {
      if (k + i * kFewGroups >= k1) break;
      float a[8];
      widen8(q[i], a);
      const float* x = xs + (k + i * kFewGroups) * M;
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[m][e] = fmaf(x[m], a[e], v[m][e]);
    }
  }
};

// Sums a workgroup's groups of lanes: v is this lane's share of columns 8 (lane %
// 8) .. + 7; row m, column c of the sum goes to out[m * ld + c] (c < width).
// Between the eight groups of a wavefront the lanes exchange halves, so that each
// ends with one column of every row.
template <int M>
__device__ __forceinline__ void few_sum(float (&v)[M][8], float* lds, float* out, int64_t ld, int width) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool b0 = lane & 8, b1 = lane & 16, b2 = lane & 32;
  const int col = lane % 8 * 8 + (b0 ? 4 : 0) + (b1 ? 2 : 0) + (b2 ? 1 : 0);
#pragma unroll
  for (int m = 0; m < M; ++m) {
    float w[4], x[2];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = (b0 ? v[m][e + 4] : v[m][e]) + __shfl_xor(b0 ? v[m][e] : v[m][e + 4], 8, FAL_WAVE);
#pragma unroll
    for (int e = 0; e < 2; ++e) x[e] = (b1 ? w[e + 2] : w[e]) + __shfl_xor(b1 ? w[e] : w[e + 2], 16, FAL_WAVE);
    lds[(m * kFewWaves + wave) * 64 + col] = (b2 ? x[1] : x[0]) + __shfl_xor(b2 ? x[0] : x[1], 32, FAL_WAVE);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < M * 64; i += kFewThreads) {
    const int c = i & 63, m = i >> 6;
    const float* s = lds + m * kFewWaves * 64 + c;
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) t += s[w * 64];
    if (c < width) out[m * ld + c] = t;
  }
  __syncthreads();
}

// part[range][0 .. 1][M][f]: g (blockIdx.z 0) or u over a range of `per` k.  (Both
// in one workgroup took so many registers that a compute unit held one: 19.8 us
// for five rows of 2048 x 5504, these 13.0.)
template <int M>
__global__ __launch_bounds__(kFewThreads, 4) void few_gate(Gated p, int per, float* part) {
  __shared__ float lds[M * kFewWaves * 64];
  extern __shared__ float xs[];  // [per][M]
  const int k0 = blockIdx.y * per, n = min(p.K - k0, per);
  const int lane = threadIdx.x & 63, group = (threadIdx.x >> 6) * 8 + lane / 8;
  const int c = min((int)blockIdx.x * 64 + lane % 8 * 8, p.N - 8);  // (f is a multiple of 8)
  const int64_t ld = blockIdx.z ? p.ldb1 : p.ldb0;
  const bf16* w = (blockIdx.z ? p.b1 : p.b0) + (int64_t)(k0 + group) * ld + c;
  FewRows rows;
  rows.load(w, ld, group, n);
  for (int i = threadIdx.x; i < n / 8 * M; i += kFewThreads) {  // (d is a multiple of 8, per of 64)
    const int m = i % M, k = i / M * 8;
    float v[8];
    widen8(*reinterpret_cast<const uint4*>(p.a + m * p.lda + k0 + k), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) xs[(k + e) * M + m] = v[e];
  }
  __syncthreads();
  float v[M][8] = {};
  for (int k = group;;) {
    rows.add<M>(xs, k, n, v);
    k += kFewBatch * kFewGroups;
    if (k >= n) break;
    w += (int64_t)kFewBatch * kFewGroups * ld;
    rows.load(w, ld, k, n);
  }
  few_sum<M>(v, lds, part + ((int64_t)blockIdx.y * 2 + blockIdx.z) * M * p.N + blockIdx.x * 64, p.N,
             p.N - (int)blockIdx.x * 64);
}

// part[range][M][d]: h Wd over a range of f, h from `splits` parts of g and u;
// the first column of workgroups writes them to saved as well.  p.a unused; b0 Wd,
// K f, N d.
template <int M>
__global__ __launch_bounds__(kFewThreads, 4) void few_down(Gated p, int per, const float* gu, int splits, float* part) {
  __shared__ float lds[M * kFewWaves * 64];
  extern __shared__ float hs[];  // [per][M]
  const int k0 = blockIdx.y * per, n = min(p.K - k0, per);
  const int lane = threadIdx.x & 63, group = (threadIdx.x >> 6) * 8 + lane / 8;
  const bf16* w = p.b0 + (int64_t)(k0 + group) * p.ldb0 + min((int)blockIdx.x * 64 + lane % 8 * 8, p.N - 8);
  FewRows down;
  down.load(w, p.ldb0, group, n);
  const int64_t mf = (int64_t)M * p.K;
  for (int i = threadIdx.x; i < n / 4 * M; i += kFewThreads) {  // (f is a multiple of 8, per of 64)
    const int m = i / (n / 4), k = i % (n / 4) * 4;
    const float* s = gu + (int64_t)m * p.K + k0 + k;
    float g[4] = {}, u[4] = {};
    for (int r0 = 0; r0 < splits; r0 += 4) {
      float4 pg[4], pu[4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (r0 + r < splits) {
          pg[r] = *reinterpret_cast<const float4*>(s + (r0 + r) * 2 * mf);
          pu[r] = *reinterpret_cast<const float4*>(s + (r0 + r) * 2 * mf + mf);
        } else {
          pg[r] = pu[r] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        g[0] += pg[r].x; g[1] += pg[r].y; g[2] += pg[r].z; g[3] += pg[r].w;
        u[0] += pu[r].x; u[1] += pu[r].y; u[2] += pu[r].z; u[3] += pu[r].w;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float a, da;
      act_and_grad<false>(p.act, g[e], a, da);
      hs[(k + e) * M + m] = a * u[e];
    }
    if (p.saved && blockIdx.x == 0) {
      float* o = p.saved + (int64_t)m * 2 * p.K + k0 + k;
      *reinterpret_cast<float4*>(o) = make_float4(g[0], g[1], g[2], g[3]);
      *reinterpret_cast<float4*>(o + p.K) = make_float4(u[0], u[1], u[2], u[3]);
    }
  }
  __syncthreads();
  float v[M][8] = {};
  for (int k = group;;) {
    down.add<M>(hs, k, n, v);
    k += kFewBatch * kFewGroups;
    if (k >= n) break;
    w += (int64_t)kFewBatch * kFewGroups * p.ldb0;
    down.load(w, p.ldb0, k, n);
  }
  few_sum<M>(v, lds, part + (int64_t)blockIdx.y * M * p.N + blockIdx.x * 64, p.N, p.N - (int)blockIdx.x * 64);
}

// y[m][c] = sum of the parts, in order.
__global__ __launch_bounds__(256) void few_out(const float* part, int splits, int M, int d, bf16* y, int64_t ldy) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= M * d) return;
  float v[kFewSplits];
#pragma unroll
  for (int s = 0; s < kFewSplits; ++s) v[s] = s < splits ? part[(int64_t)s * M * d + i] : 0.f;
  float t = v[0];
#pragma unroll
  for (int s = 1; s < kFewSplits; ++s) t += v[s];
  y[(int64_t)(i / d) * ldy + i % d] = from_f<bf16>(t);
}

// How many ranges a product's k is cut into: as many rows as the workgroup's first
// loads ask for, fewer where that leaves compute units without a workgroup, more
// where the workgroups would not run all at once (2048 x 5504: 688 of 512 rows
// 14.3 us, 344 of 1024 13.0); a range's rows have to fit LDS.
constexpr int kFewSlots = 512;  // workgroups that run at once
constexpr int kFewLds = 11264;  // floats of a range's rows: with the sums, 61 KB
struct FewSplit {
  int splits, per;
};
FewSplit few_split(int K, int strips, int M) {
  int per = kFewGroups * kFewBatch;
  while (per > 2 * kFewGroups && cdiv(K, per) * strips < 256) per /= 2;
  while ((cdiv(K, per) > kFewSplits || (cdiv(K, per) * strips > kFewSlots && cdiv(K, 2 * per) * strips >= 256)) &&
         2 * per * M <= kFewLds)
    per *= 2;
  return {cdiv(K, per), per};
}
FewSplit few_up(const GatedFfn& a) { return few_split(a.d, 2 * cdiv(a.f, 64), a.M); }
FewSplit few_last(const GatedFfn& a) { return few_split(a.f, cdiv(a.d, 64), a.M); }

bool few_rows(DType dt, const GatedFfn& a) {
  return dt == BF16 && a.M <= kFew && few_last(a).splits <= kFewSplits;
}

template <int M>
hipError_t few_fwd(const GatedFfn& a, Gated p, const bf16* wd, bf16* y, float* scratch, hipStream_t s) {
  const FewSplit up = few_up(a), down = few_last(a);
  float* gu = scratch;
  float* part = scratch + (int64_t)up.splits * 2 * M * a.f;
  hipLaunchKernelGGL((few_gate<M>), dim3(cdiv(a.f, 64), up.splits, 2), dim3(kFewThreads), up.per * M * 4, s, p, up.per,
                     gu);
  p.b0 = wd; p.ldb0 = a.ldd; p.N = a.d; p.K = a.f;
  hipLaunchKernelGGL((few_down<M>), dim3(cdiv(a.d, 64), down.splits), dim3(kFewThreads), down.per * M * 4, s, p,
                     down.per, gu, up.splits, part);
  hipLaunchKernelGGL(few_out, dim3(cdiv((int64_t)M * a.d, 256)), dim3(256), 0, s, part, down.splits, M, a.d, y, a.ldy);
  return hipGetLastError();
}

// ------------------------------------------------ joined products --
// Elementwise kernels after products whose k was split among workgroups (or, in
// fp32, after whole ones): `parts` fp32 sums lie `stride` floats apart and are
// added in order, four columns a thread where rows allow it (V 4, else 1).
template <int V>
__device__ __forceinline__ void sum_parts(const float* p, int parts, int64_t stride, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = p[e];
#pragma unroll 4
  for (int i = 1; i < parts; ++i)
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] += p[i * stride + e];
}

// This thread's number (one axis of a grid holds fewer than 2^32 threads).
constexpr int64_t kJoinRow = 1 << 22;  // workgroups in a row of the grid
__device__ __forceinline__ int64_t join_thread() {
  return (blockIdx.y * kJoinRow + blockIdx.x) * 256 + threadIdx.x;
}

// h = act(g) u, g and u [M][f] parts; saved (g | u) may be NULL or, with one part,
// where g and u are.
template <typename T, int V>
__global__ __launch_bounds__(256) void join_gate(const float* g, const float* u, int64_t ld, int parts, int64_t stride,
                                                 int64_t n, int f, int act, float* saved, T* h) {
  const int64_t i = join_thread() * V;
  if (i >= n) return;
  const int64_t m = i / f, c = i % f;
  float gv[V], uv[V];
  sum_parts<V>(g + m * ld + c, parts, stride, gv);
  sum_parts<V>(u + m * ld + c, parts, stride, uv);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    float a, da;
    act_and_grad<sizeof(T) == 4>(act, gv[e], a, da);
    h[i + e] = from_f<T>(a * uv[e]);
    if (saved) {
      saved[m * 2 * f + c + e] = gv[e];
      saved[m * 2 * f + f + c + e] = uv[e];
    }
  }
}

// dg, du and h from parts of dh (one part may be dg) and the saved g | u.
template <typename T, int V>
__global__ __launch_bounds__(256) void join_gate_bwd(const float* dh, int parts, int64_t stride, const float* saved,
                                                     int64_t n, int f, int act, T* dg, T* du, T* h) {
  const int64_t i = join_thread() * V;
  if (i >= n) return;
  const int64_t m = i / f, c = i % f;
  float d[V];
  sum_parts<V>(dh + i, parts, stride, d);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float g = saved[m * 2 * f + c + e], u = saved[m * 2 * f + f + c + e];
    float a, da;
    act_and_grad<sizeof(T) == 4>(act, g, a, da);
    h[i + e] = from_f<T>(a * u);
    dg[i + e] = from_f<T>(d[e] * u * da);
    du[i + e] = from_f<T>(d[e] * a);
  }
}

// out[m][c] = the parts' sum.
template <typename T, int V>
__global__ __launch_bounds__(256) void join_rows(const float* part, int parts, int64_t n, int N, T* out, int64_t ldo) {
  const int64_t i = join_thread() * V;
  if (i >= n) return;
  float v[V];
  sum_parts<V>(part + i, parts, n, v);
#pragma unroll
  for (int e = 0; e < V; ++e) out[i / N * ldo + i % N + e] = from_f<T>(v[e]);
}

GemmProblem product(const void* A, int64_t lda, const void* B, int64_t ldb, int M, int N, int K, void* out,
                    int64_t ldo, int f32) {
  GemmProblem p;
  memset(&p, 0, sizeof(p));
  p.A = A; p.B = B; p.lda = lda; p.ldb = ldb;
  p.M = M; p.N = N; p.K = K;
  p.epi = EPI_STORE; p.out_f32 = f32; p.out = out; p.ldo = ldo;
  return p;
}

hipError_t run(DType dt, int a_kmaj, int b_kmaj, std::initializer_list<GemmProblem> ps, hipStream_t s) {
  GemmGroup g;
  memset(&g, 0, sizeof(g));
  for (const GemmProblem& p : ps) g.p[g.n++] = p;
  const char* why;
  return gemm(dt, a_kmaj, b_kmaj, g, 0, s, &why);
}

dim3 blocks_of(int64_t n, int per) {
  const int64_t blocks = (n + 256 * per - 1) / (256 * per), x = std::min<int64_t>(blocks, kJoinRow);
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

// The larger tile, two workgroups a compute unit, once it gives every compute unit
// two (8192 x 2048 x 5504, 2752 tiles: forward 407 us against 469 on those of 64
// columns, backward 317 against 402, measured side by side); three of 64 columns
// below that (1501 x 1000 x 2744, 264 large tiles: 46 against 39 forward, 64 against
// 38 backward).  Tiles of 256 rows, one workgroup a compute unit, whose epilogues
// nothing covers, took 474 and 386 where the larger tile took 412 and 322.
template <int BWD>
hipError_t launch_gated(Gated p, hipStream_t s) {
  constexpr int BN = BWD ? 256 : 128;
  const int64_t large = (int64_t)cdiv(p.M, 128) * cdiv(p.N, BN), small = (int64_t)cdiv(p.M, 128) * cdiv(p.N, 64);
  p.tiles_m = cdiv(p.M, 128);
  p.tiles_n = cdiv(p.N, large >= 512 ? BN : 64);
  if (large >= 512) hipLaunchKernelGGL((gated_mfma<BWD, 128, BN, 2>), dim3((unsigned)large), dim3(256), 0, s, p);
  else hipLaunchKernelGGL((gated_mfma<BWD, 128, 64, 3>), dim3((unsigned)small), dim3(256), 0, s, p);
  return hipGetLastError();
}

// bf16 products with few tiles of 128 x 128: k in up to `most` parts, each a problem
// of its own in one launch, whose fp32 sums the kernel after them adds.  Parts of at
// least 256 k, and no more of them than run at once (1501 x 1000 x 2744: 48 us whole,
// 25 in four and 5 joined; dx, two products of that size, 91 us whole, 34 and 6).
struct Cut {
  int parts, per;
};
Cut cut(int M, int N, int K, int products, int most) {
  const int64_t tiles = (int64_t)cdiv(M, 128) * cdiv(N, 128) * products;
  for (int s = most; s > 1; s /= 2) {
    const int per = (cdiv(K, s) + 63) / 64 * 64;
    if (tiles * s <= 512 && per >= 256 && cdiv(K, per) == s) return {s, per};
  }
  return {1, K};
}

int64_t round_up(int64_t n) { return (n + 255) / 256 * 256; }

// The same of fp32 sums over f: where tiles are few (forward and backward of
// 20 x 1000 x 3000: 199 us whole, 110 in parts; 500 x 2000 x 4000: 991 and 881;
// 64 x 64 x 256, where the join costs what it saves: 55), and from 4096 terms on,
// because a sum adds one rounding a term and four shorter ones halve the error
// (9504 terms: 1.2e-6 of the norm, 6e-7 in four; 1000 x 4096 x 11008: 7964 us
// whole, 7609 in parts).
Cut cut_f32(int M, int N, int K, int most) {
  const int per = (cdiv(K, most) + 3) / 4 * 4;
  const bool few = (int64_t)cdiv(M, 64) * cdiv(N, 64) * most <= 1024 && K >= 512;
  return K >= 4096 || few ? Cut{cdiv(K, per), per} : Cut{1, K};
}

// What a call cuts (parts 1: that product runs whole).
struct Cuts {
  Cut gate, down;  // forward: x Wg and x Wu, h Wd
  Cut dh, dx;      // backward: dy Wd^T, each of dx's two products
  bool apart;      // dx's two products are problems of their own
};
Cuts cuts(DType dt, const GatedFfn& a) {
  if (dt == F32) {
    const Cut whole = {1, a.d}, dx = cut_f32(a.M, a.d, a.f, 2);
    return {whole, cut_f32(a.M, a.d, a.f, 4), whole, dx, dx.parts > 1};
  }
  return {cut(a.M, a.f, a.d, 2, 2), cut(a.M, a.d, a.f, 1, 4), cut(a.M, a.f, a.d, 1, 4), cut(a.M, a.d, a.f, 2, 2),
          (int64_t)cdiv(a.M, 128) * cdiv(a.d, 128) <= 256};
}

// out [M, N] at ldo = the sum of all of g's problems, which write their parts here.
hipError_t run_parts(DType dt, int b_kmaj, GemmGroup& g, float* part, void* out, int64_t ldo, hipStream_t s) {
  const int M = g.p[0].M, N = g.p[0].N;
  const int64_t n = (int64_t)M * N;
  for (int i = 0; i < g.n; ++i) {
    g.p[i].out = part + i * n;
    g.p[i].ldo = N;
    g.p[i].out_f32 = 1;
  }
  const char* why;
  const hipError_t e = gemm(dt, 1, b_kmaj, g, 0, s, &why);
  if (e != hipSuccess) return e;
  if (dt == BF16)
    hipLaunchKernelGGL((join_rows<bf16, 4>), blocks_of(n, 4), dim3(256), 0, s, part, g.n, n, N, static_cast<bf16*>(out), ldo);
  else if (N % 4 == 0)
    hipLaunchKernelGGL((join_rows<float, 4>), blocks_of(n, 4), dim3(256), 0, s, part, g.n, n, N, static_cast<float*>(out),
                       ldo);
  else
    hipLaunchKernelGGL((join_rows<float, 1>), blocks_of(n, 1), dim3(256), 0, s, part, g.n, n, N, static_cast<float*>(out),
                       ldo);
  return hipGetLastError();
}

const void* at(DType dt, const void* p, int64_t elements) {
  return static_cast<const char*>(p) + elements * (dt == BF16 ? 2 : 4);
}

// y = h Wd, in parts of k where k.parts says so.
hipError_t down_product(DType dt, const GatedFfn& a, const Cut& k, const void* h, const void* wd, void* y, float* part,
                        hipStream_t s) {
  if (k.parts == 1) return run(dt, 1, 0, {product(h, a.f, wd, a.ldd, a.M, a.d, a.f, y, a.ldy, dt == F32)}, s);
  GemmGroup g;
  memset(&g, 0, sizeof(g));
  for (; g.n < k.parts; ++g.n) {
    const int k0 = g.n * k.per;
    g.p[g.n] = product(at(dt, h, k0), a.f, at(dt, wd, k0 * a.ldd), a.ldd, a.M, a.d, std::min(k.per, a.f - k0), nullptr,
                       0, 1);
  }
  return run_parts(dt, 0, g, part, y, a.ldy, s);
}

// dx = dg Wg^T + du Wu^T, in one launch over both or in parts.
hipError_t dx_product(DType dt, const GatedFfn& a, const Cuts& k, const void* dg, const void* du, const void* wg,
                      const void* wu, void* dx, float* part, hipStream_t s) {
  if (!k.apart) {
    GemmProblem p = product(dg, a.f, wg, a.ldg, a.M, a.d, a.f, dx, a.lddx, dt == F32);
    p.A2 = du; p.lda2 = a.f; p.B2 = wu; p.ldb2 = a.ldu; p.K2 = a.f;
    return run(dt, 1, 1, {p}, s);
  }
  GemmGroup g;
  memset(&g, 0, sizeof(g));
  for (int b = 0; b < 2; ++b)
    for (int i = 0; i < k.dx.parts; ++i) {
      const int k0 = i * k.dx.per;
      g.p[g.n++] = product(at(dt, b ? du : dg, k0), a.f, at(dt, b ? wu : wg, k0), b ? a.ldu : a.ldg, a.M, a.d,
                           std::min(k.dx.per, a.f - k0), nullptr, 0, 1);
    }
  return run_parts(dt, 1, g, part, dx, a.lddx, s);
}

}  // namespace

int64_t gated_ffn_scratch(DType dt, const GatedFfn& a, int backward) {
  const int64_t one = round_up((int64_t)a.M * a.f * (dt == BF16 ? 2 : 4)), mf = (int64_t)a.M * a.f * 4,
                md = (int64_t)a.M * a.d * 4;
  if (!backward && few_rows(dt, a))
    return 4 * a.M * ((int64_t)few_up(a).splits * 2 * a.f + (int64_t)few_last(a).splits * a.d);
  const Cuts k = cuts(dt, a);
  // (the parts of one product are read before the next one's are written)
  const int64_t down = k.down.parts > 1 ? k.down.parts * md : 0, dx = k.apart ? 2 * k.dx.parts * md : 0;
  // fp32: h, and g | u where they are not saved
  if (!backward) return (dt == F32 ? 3 * one : one) + std::max(k.gate.parts > 1 ? 2 * k.gate.parts * mf : 0, down);
  return 3 * one + std::max(k.dh.parts > 1 ? k.dh.parts * mf : 0, dx);
}

hipError_t gated_ffn_fwd(DType dt, const GatedFfn& a, const void* x, const void* wg, const void* wu, const void* wd,
                         void* y, float* saved, void* scratch, hipStream_t s) {
  hipError_t e;
  void* h = scratch;
  const int64_t n = (int64_t)a.M * a.f;
  const Cuts k = cuts(dt, a);
  if (dt == F32) {
    float* gu = saved ? saved : reinterpret_cast<float*>(static_cast<char*>(scratch) + round_up(n * 4));
    const int64_t ld = 2 * (int64_t)a.f;
    e = run(F32, 1, 0, {product(x, a.ldx, wg, a.ldg, a.M, a.f, a.d, gu, ld, 1),
                        product(x, a.ldx, wu, a.ldu, a.M, a.f, a.d, gu + a.f, ld, 1)}, s);
    if (e != hipSuccess) return e;
    if (a.f % 4 == 0)
      hipLaunchKernelGGL((join_gate<float, 4>), blocks_of(n, 4), dim3(256), 0, s, gu, gu + a.f, ld, 1, 0, n, a.f, a.act,
                         nullptr, static_cast<float*>(h));
    else
      hipLaunchKernelGGL((join_gate<float, 1>), blocks_of(n, 1), dim3(256), 0, s, gu, gu + a.f, ld, 1, 0, n, a.f, a.act,
                         nullptr, static_cast<float*>(h));
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    float* part = reinterpret_cast<float*>(static_cast<char*>(scratch) + 3 * round_up(n * 4));
    return down_product(F32, a, k.down, h, wd, y, part, s);
  }
  Gated p;
  memset(&p, 0, sizeof(p));
  const bf16* xb = static_cast<const bf16*>(x);
  const bf16 *gate = static_cast<const bf16*>(wg), *up = static_cast<const bf16*>(wu), *down = static_cast<const bf16*>(wd);
  p.a = xb; p.b0 = gate; p.b1 = up;
  p.lda = a.ldx; p.ldb0 = a.ldg; p.ldb1 = a.ldu;
  p.M = a.M; p.N = a.f; p.K = a.d; p.act = a.act;
  p.saved = saved;
  p.h = static_cast<bf16*>(h);
  if (few_rows(dt, a)) {
    bf16* out = static_cast<bf16*>(y);
    float* part = static_cast<float*>(scratch);
    switch (a.M) {
      case 1: return few_fwd<1>(a, p, down, out, part, s);
      case 2: return few_fwd<2>(a, p, down, out, part, s);
      case 3: return few_fwd<3>(a, p, down, out, part, s);
      case 4: return few_fwd<4>(a, p, down, out, part, s);
      case 5: return few_fwd<5>(a, p, down, out, part, s);
      case 6: return few_fwd<6>(a, p, down, out, part, s);
      case 7: return few_fwd<7>(a, p, down, out, part, s);
      default: return few_fwd<8>(a, p, down, out, part, s);
    }
  }
  float* part = reinterpret_cast<float*>(static_cast<char*>(scratch) + round_up(n * 2));
  if (k.gate.parts > 1) {
    // (two parts: as many problems as a launch holds)
    const int k1 = k.gate.per, k2 = a.d - k1;
    e = run(BF16, 1, 0, {product(xb, a.ldx, gate, a.ldg, a.M, a.f, k1, part, a.f, 1),
                         product(xb + k1, a.ldx, gate + k1 * a.ldg, a.ldg, a.M, a.f, k2, part + n, a.f, 1),
                         product(xb, a.ldx, up, a.ldu, a.M, a.f, k1, part + 2 * n, a.f, 1),
                         product(xb + k1, a.ldx, up + k1 * a.ldu, a.ldu, a.M, a.f, k2, part + 3 * n, a.f, 1)}, s);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((join_gate<bf16, 4>), blocks_of(n, 4), dim3(256), 0, s, part, part + 2 * n, a.f, 2, n, n, a.f,
                       a.act, saved, p.h);
    e = hipGetLastError();
  } else {
    e = launch_gated<0>(p, s);
  }
  if (e != hipSuccess) return e;
  return down_product(BF16, a, k.down, h, wd, y, part, s);
}

hipError_t gated_ffn_bwd(DType dt, const GatedFfn& a, const void* x, const void* wg, const void* wu, const void* wd,
                         const float* saved, const void* dy, void* dx, void* dwg, void* dwu, void* dwd, void* scratch,
                         hipStream_t s) {
  const int64_t n = (int64_t)a.M * a.f, one = round_up(n * (dt == BF16 ? 2 : 4));
  char* base = static_cast<char*>(scratch);
  void *dg = base, *du = base + one, *h = base + 2 * one;
  float* part = reinterpret_cast<float*>(base + 3 * one);
  const Cuts k = cuts(dt, a);
  const char* why;
  hipError_t e;
  if (dt == F32) {
    e = run(F32, 1, 1, {product(dy, a.ldy, wd, a.ldd, a.M, a.f, a.d, dg, a.f, 1)}, s);
    if (e != hipSuccess) return e;
    float *g32 = static_cast<float*>(dg), *u32 = static_cast<float*>(du), *h32 = static_cast<float*>(h);
    if (a.f % 4 == 0)
      hipLaunchKernelGGL((join_gate_bwd<float, 4>), blocks_of(n, 4), dim3(256), 0, s, g32, 1, 0, saved, n, a.f, a.act, g32,
                         u32, h32);
    else
      hipLaunchKernelGGL((join_gate_bwd<float, 1>), blocks_of(n, 1), dim3(256), 0, s, g32, 1, 0, saved, n, a.f, a.act, g32,
                         u32, h32);
    e = hipGetLastError();
  } else if (k.dh.parts > 1) {
    GemmGroup g;
    memset(&g, 0, sizeof(g));
    for (; g.n < k.dh.parts; ++g.n) {
      const int k0 = g.n * k.dh.per;
      g.p[g.n] = product(static_cast<const bf16*>(dy) + k0, a.ldy, static_cast<const bf16*>(wd) + k0, a.ldd, a.M, a.f,
                         std::min(k.dh.per, a.d - k0), part + g.n * n, a.f, 1);
    }
    e = gemm(BF16, 1, 1, g, 0, s, &why);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((join_gate_bwd<bf16, 4>), blocks_of(n, 4), dim3(256), 0, s, part, g.n, n, saved, n, a.f, a.act,
                       static_cast<bf16*>(dg), static_cast<bf16*>(du), static_cast<bf16*>(h));
    e = hipGetLastError();
  } else {
    Gated p;
    memset(&p, 0, sizeof(p));
    p.a = static_cast<const bf16*>(dy); p.b0 = static_cast<const bf16*>(wd);
    p.lda = a.ldy; p.ldb0 = a.ldd;
    p.M = a.M; p.N = a.f; p.K = a.d; p.act = a.act;
    p.saved = const_cast<float*>(saved);
    p.h = static_cast<bf16*>(h); p.dg = static_cast<bf16*>(dg); p.du = static_cast<bf16*>(du);
    e = launch_gated<1>(p, s);
  }
  if (e != hipSuccess) return e;
  if (dx) {
    e = dx_product(dt, a, k, dg, du, wg, wu, dx, part, s);
    if (e != hipSuccess) return e;
  }
  if (!dwg) return hipSuccess;
  const int f32 = dt == F32 || a.grads_f32;
  return run(dt, 0, 0, {product(x, a.ldx, dg, a.f, a.d, a.f, a.M, dwg, a.lddg, f32),
                        product(x, a.ldx, du, a.f, a.d, a.f, a.M, dwu, a.lddu, f32),
                        product(h, a.f, dy, a.ldy, a.f, a.d, a.M, dwd, a.lddd, f32)}, s);
}

}  // namespace fal
