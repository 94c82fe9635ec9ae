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

// fp32 at head_dim 128: the backward kernels need more registers than two
// wavefronts a SIMD have (bounded to 256 they spill: dQ 113 -> 148 us at 2
// sequences of 1999 tokens, 8 heads, window 300).
template <typename S, int HD>
constexpr bool kWide = HD == 128 && sizeof(S) == 4;
// dK/dV of wide bf16 heads: the keys stay in LDS rather than in registers, so
// that two workgroups (head_dim 64: three) fit a compute unit and cover each
// other's waits; at 128 the query tiles are also fetched when they are due, not
// one ahead, for the same reason (8192 tokens, 16 heads of 128, window 1024:
// 226 -> 173 us; 8 sequences of 1024, 12 heads of 64, window 256: 34 -> 30).
template <typename S, int HD>
constexpr bool kKeysInLds = HD >= 64 && sizeof(S) == 2;
// Wavefronts a SIMD that the backward kernels' registers are bounded to.
template <typename S, int HD>
constexpr int kWaves = kWide<S, HD> ? 1 : 2;
template <typename S, int HD>
constexpr int kWavesDkdv = kKeysInLds<S, HD> && HD == 64 ? 3 : kWaves<S, HD>;

template <int HD>
constexpr int n_tiles() { return HD < 32 ? 1 : HD / 32; }

// N groups of R LDS reads and the M MFMAs that they feed: the reads of LA
// groups stay in flight.  Ends the scheduling region.
template <int N, int R, int M, int LA>
__device__ __forceinline__ void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, R * LA, 0);
#pragma unroll
  for (int q = 0; q < N - LA; ++q) {
    __builtin_amdgcn_sched_group_barrier(0x008, M, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, M * LA, 0);
  __builtin_amdgcn_sched_barrier(0);
}
// ... of P products over head_dim, and of P sums over a tile's rows
template <typename S, int HD, int P>
__device__ __forceinline__ void dots_ahead() {
  if (sizeof(S) == 2 && HD >= 64) reads_ahead<P * HD / 16, 1, 1, 4>();
  if (sizeof(S) == 4) reads_ahead<P * HD / 8, 1, 4, 2>();
}
template <typename S, int HD, int P>
__device__ __forceinline__ void sums_ahead() {
  if (sizeof(S) == 2 && HD >= 64) reads_ahead<P * HD / 16, 2, 1, 4>();
  if (sizeof(S) == 4) reads_ahead<P * 16, (n_tiles<HD>() + 1) / 2, n_tiles<HD>(), 2>();
}

// x of this lane and of lane ^ 32: one swap of half wavefronts
__device__ __forceinline__ void both_halves(float x, float& lo, float& hi) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  lo = __uint_as_float(r[0]);
  hi = __uint_as_float(r[1]);
}

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
// zeros (a clamped row is read in their place).  A whole tile's addresses are
// a uniform base and the thread's own offset, computed once.
template <typename S, int HD>
struct Stage {
  static constexpr int E = 16 / (int)sizeof(S), CH = HD / E, N = (AT * CH + 255) / 256;
  uint4 v[N];
  const S* src;
  int64_t ld, own;
  __device__ __forceinline__ Stage(const S* src_, int64_t ld_, int tid) : src(src_), ld(ld_) {
    own = (tid / CH) * ld + E * (tid % CH);
  }
  __device__ __forceinline__ void load(int row0, int n, int tid) {
    if (row0 + AT <= n) {
      const S* tile = src + row0 * ld;
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (256 * (k + 1) <= AT * CH || tid + 256 * k < AT * CH)
          v[k] = *reinterpret_cast<const uint4*>(tile + k * (256 / CH) * ld + own);
      return;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = tid + 256 * k;
      const int row = min(row0 + i / CH, n - 1);
      if (256 * (k + 1) <= AT * CH || i < AT * CH)
        v[k] = *reinterpret_cast<const uint4*>(src + row * ld + E * (i % CH));
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

// What the kernels of dK and dV take of 64 queries from row0 on of a (sequence,
// head): -lse in log2 units and -D, a query a thread; zeros at or past n.  They
// are asked for with the tile, a wait less in every step (4 sequences of 2048
// tokens, 16 heads of 64 under the full mask: dK/dV 93.5 -> 86.3 us).
struct Stats {
  float l, d;
  __device__ __forceinline__ void load(const float* lse, const float* Dvec, int row0, int n, int tid) {
    if (tid < AT) {
      const int i = min(row0 + tid, n - 1);
      l = lse[i];
      d = Dvec[i];
    }
  }
  __device__ __forceinline__ void store(float* sL, float* sD, int row0, int n, int tid) {
    if (tid < AT) {
      sL[tid] = row0 + tid < n ? -l * kLog2e : 0.f;
      sD[tid] = row0 + tid < n ? -d : 0.f;
    }
  }
};

constexpr int kFewKeys = AT;

// The window's mask over a 32x32 score tile whose rows are the keys from kb on
// and whose lane has query tq, one of q0 .. q0 + 31: -inf for keys after the
// query (or past n), and for keys before its window and past the sinks.  Each
// edge is tested where it crosses the tile, without branches.
__device__ __forceinline__ void mask_keys(const WindowAttn& a, int kb, int q0, int tq, int n, int g, f32x16v& s) {
  const int key0 = kb + 4 * g;
  if (kb + 31 > q0 || kb + 31 >= n) {
    const int last = min(tq, n - 1) - key0;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = acc_row(r, 0) > last ? -INFINITY : s[r];
  }
  if (q0 + 31 - kb >= a.window) {
    const int before = tq - a.window - key0, sink = a.sinks - key0;
    if (kb >= a.sinks) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = acc_row(r, 0) <= before ? -INFINITY : s[r];
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        s[r] = ((int)(acc_row(r, 0) <= before) & (int)(acc_row(r, 0) >= sink)) ? -INFINITY : s[r];
    }
  }
}
// The same where the rows are the queries from qs on and the lane has the key,
// one of kw .. kw + 31.
__device__ __forceinline__ void mask_queries(const WindowAttn& a, int qs, int kw, int key, int g, f32x16v& s) {
  const int q0 = qs + 4 * g;
  if (qs < kw + 32) {
    const int first = key - q0;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = acc_row(r, 0) < first ? -INFINITY : s[r];
  }
  if (qs + 31 - kw >= a.window) {
    const int past = key < a.sinks ? 1 << 30 : key + a.window - q0;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = acc_row(r, 0) >= past ? -INFINITY : s[r];
  }
}

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
__device__ __forceinline__ void dot_rows(const bf16* s, int rowbase, int c, int g, const Own<bf16, HD>& o,
                                         f32x16v& acc) {
#pragma unroll
  for (int k = 0; k < HD / 16; ++k) acc = mfma32(frag_rows<HD>(s, rowbase, c, k, g), o.f[k], acc);
}
template <int HD>
__device__ __forceinline__ void dot_rows(const float* s, int rowbase, int c, int g, const Own<float, HD>& o,
                                         f32x16v& acc) {
  const float* row = s + (HD + 4) * (rowbase + c) + 4 * g;
#pragma unroll
  for (int k = 0; k < HD / 8; ++k) {
    const f32x4v a = *reinterpret_cast<const f32x4v*>(row + 8 * k);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], o.f[k][j], acc, 0, 0, 0);
  }
}

// The same with the own rows in LDS as well (bf16).
template <int HD>
__device__ __forceinline__ void dot_rows(const bf16* s, int rowbase, int c, int g, const bf16* own, f32x16v& acc) {
#pragma unroll
  for (int k = 0; k < HD / 16; ++k)
    acc = mfma32(frag_rows<HD>(s, rowbase, c, k, g), frag_rows<HD>(own, 0, c, k, g), acc);
}
template <int HD>
__device__ __forceinline__ void dot_rows(const float*, int, int, int, const float*, f32x16v&) {}

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

// Key tiles of a block of `rows` queries from qb on: `sink` tiles from key 0,
// then the window's tiles from `first` (a multiple of AT) up to `end`.
struct KeyTiles {
  int sink, first, end, count;
  __device__ __forceinline__ KeyTiles(const WindowAttn& a, int qb, int rows, int n) {
    end = min(n, qb + rows);
    first = max(0, qb - a.window + 1) / AT * AT;
    sink = (min(a.sinks, first) + AT - 1) / AT;
    count = sink + (end - first + AT - 1) / AT;
  }
  __device__ __forceinline__ int at(int i) const { return i < sink ? AT * i : first + AT * (i - sink); }
};

// A workgroup's four wavefronts own 32 rows each and walk both 32-row halves
// of every tile, or (SPLIT) in pairs the same 32 rows, one half of the tiles
// each, joining their sums at the end: half the rows and half the walk a
// workgroup.
template <bool SPLIT>
constexpr int block_rows() { return SPLIT ? 64 : 128; }

// LDS of a kernel: two tiles, the join's registers of two wavefronts, or a row
// of sums for each of 32 sink keys
template <typename S, int HD, bool SPLIT>
constexpr int lds_bytes() {
  const int tiles = 2 * tile_len<S, HD>() * (int)sizeof(S), join = SPLIT ? 2 * n_tiles<HD>() * 16 * 64 * 4 + 1024 : 0;
  const int sums = 32 * (HD + 1) * 4, most = tiles > join ? tiles : join;
  return (most > sums ? most : sums) / 16 * 16 + 16;
}

// Adds the second wavefront of a pair's sums to the first's.
template <int HD>
__device__ __forceinline__ void join_acc(float* lds, int wave, int lane, f32x16v (&acc)[n_tiles<HD>()]) {
  float* p = lds + (wave & 1) * (n_tiles<HD>() * 16 * 64) + lane;
  __syncthreads();
  if (wave >= 2) {
#pragma unroll
    for (int t = 0; t < n_tiles<HD>(); ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) p[64 * (16 * t + r)] = acc[t][r];
  }
  __syncthreads();
  if (wave < 2) {
#pragma unroll
    for (int t = 0; t < n_tiles<HD>(); ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][r] += p[64 * (16 * t + r)];
  }
}

}  // namespace

// ------------------------------------------------------------- forward --
// The last blocks first: the first ones, whose windows the sequence's start
// cuts short, then fill the launch's end (6 padded sequences of 1501 tokens, 16
// heads of 64, window 500: 29.4 -> 26.1 us; 4 of 2048 under the full mask, 68.8
// -> 55.0, and dQ 80.7 -> 66.5).  At 8192 tokens, 16 heads of 128, window 1024,
// after 300 ms of such calls: 98 us, 665 TFLOP/s of the visible pairs; at 8
// sequences of 1024, 12 heads of 64, window 256: 18 us, where the exponentials and the other vector work of a
// score (about 650 cycles a 32x32 tile against 256 of MFMA) and the single round
// of workgroups bound it.
template <typename S, int HD, bool SPLIT>
__global__ __launch_bounds__(256, 2) void window_attn_fwd(WindowAttn a, const S* qkv, S* O, float* lse) {
  constexpr int NT = n_tiles<HD>();
  __shared__ __attribute__((aligned(16))) char lds[lds_bytes<S, HD, SPLIT>()];
  S *sK = reinterpret_cast<S*>(lds), *sV = sK + tile_len<S, HD>();
  const int h = blockIdx.x, b = blockIdx.y, qb = block_rows<SPLIT>() * (gridDim.z - 1 - blockIdx.z);
  const int kvh = h / (a.H / a.Hkv);
  const S* Qg = qkv + (int64_t)b * a.T * a.ldq + h * HD;
  const S* Kg = qkv + (int64_t)b * a.T * a.ldq + (a.H + kvh) * HD;
  const S* Vg = Kg + a.Hkv * HD;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, c = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q0 = qb + (SPLIT ? wave & 1 : wave) * 32, tq = q0 + c;
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
    const KeyTiles kt(a, qb, block_rows<SPLIT>(), n);
    Stage<S, HD> rk(Kg, a.ldq, tid), rv(Vg, a.ldq, tid);
    rk.load(kt.at(0), n, tid);
    rv.load(kt.at(0), n, tid);
    for (int i = 0; i < kt.count; ++i) {
      const int k0 = kt.at(i);
      __syncthreads();
      rk.store(sK, k0, n, tid);
      rv.store(sV, k0, n, tid);
      __syncthreads();
      if (i + 1 < kt.count) {
        rk.load(kt.at(i + 1), n, tid);
        rv.load(kt.at(i + 1), n, tid);
      }
#pragma unroll
      for (int u = 0; u < (SPLIT ? 1 : AT / 32); ++u) {
        const int sub = SPLIT ? wave >> 1 : u;
        const int kb = k0 + 32 * sub;
        if (kb > q0 + 31 || kb >= n) break;
        if (kb >= a.sinks && q0 - (kb + 31) >= a.window) continue;  // before the window of every row
        f32x16v s = zero16();
        __builtin_amdgcn_sched_barrier(0);
        dot_rows<HD>(sK, 32 * sub, c, g, q, s);
        dots_ahead<S, HD, 1>();
        mask_keys(a, kb, q0, tq, n, g, s);
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
        float lo, hi;
        both_halves(mx, lo, hi);
        mx = fmaxf(lo, hi) * sl2;
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
        if (sizeof(S) == 4) __builtin_amdgcn_sched_barrier(0);
        add_rows<HD>(sV, 32 * sub, lane, s, acc);
        if (sizeof(S) == 4) sums_ahead<S, HD, 1>();
      }
    }
  }
  if (SPLIT) {  // join the pair's softmaxes
    float* p = reinterpret_cast<float*>(lds) + 2 * NT * 16 * 64 + 2 * (lane + 64 * (wave & 1));
    __syncthreads();
    if (wave >= 2) {
      p[0] = mref;
      p[1] = lsum;
    }
    __syncthreads();
    if (wave < 2) {
      const float m1 = p[0], top = fmaxf(mref, m1);
      const float f0 = mref == top ? 1.f : __builtin_amdgcn_exp2f(mref - top);
      const float f1 = m1 == top ? 1.f : __builtin_amdgcn_exp2f(m1 - top);
      lsum = lsum * f0 + p[1] * f1;
      mref = top;
      p[0] = f1;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] *= f0;
    }
    __syncthreads();
    if (wave >= 2) {
      const float f1 = p[0];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] *= f1;
    }
    join_acc<HD>(reinterpret_cast<float*>(lds), wave, lane, acc);
    if (wave >= 2) return;
  }
  const float l = lsum + __shfl_xor(lsum, 32, 64);
  if (tq < a.T) {
    put_row<S, HD>(O + ((int64_t)b * a.T + tq) * a.ldo + h * HD, g, acc, 1.f / l, tq < n);
    if (g == 0)
      lse[((int64_t)b * a.H + h) * a.T + tq] = tq < n ? (mref + log2f(l)) * 0.6931471805599453f : -INFINITY;
  }
}

// ----------------------------------------------------------- backward: dQ --
// Also writes D = rowsum(dO * O) for the kernels that follow.  O as it was
// stored carries its rounding into D, which a row of many keys averages out
// and one of few does not (bf16 gradients of a window of 2 keys: 2.7e-3 off
// against 2.2e-3 with D exact, of 20: 2.42e-3 against 2.36e-3; 1.65e-3 is the
// rounding of the gradients alone).  So bf16 rows of at most kFewKeys keys sum
// D = rowsum(P * dP) in a walk of their own: every row of a call whose window and
// sinks hold no more, over its few tiles, and under a longer window the first
// kFewKeys rows of a sequence, over the first tile (dQ of the first 8 rows
// 2.64e-3 off before, 2.18e-3 with it; no time beyond the noise of 1%).  118 us
// at the 8192 tokens above (826 TFLOP/s), 23 at the 8 x 1024.
template <typename S, int HD, bool SPLIT>
__global__ __launch_bounds__(256, (kWaves<S, HD>)) void window_attn_dq(WindowAttn a, const S* qkv, const S* O,
                                                                       const S* dO, const float* lse, float* Dvec,
                                                                       S* dqkv) {
  constexpr int NT = n_tiles<HD>();
  __shared__ __attribute__((aligned(16))) char lds[lds_bytes<S, HD, SPLIT>()];
  S *sK = reinterpret_cast<S*>(lds), *sV = sK + tile_len<S, HD>();
  const int h = blockIdx.x, b = blockIdx.y, qb = block_rows<SPLIT>() * (gridDim.z - 1 - blockIdx.z);
  const int kvh = h / (a.H / a.Hkv);
  const int64_t row0 = (int64_t)b * a.T;
  const S* Kg = qkv + row0 * a.ldq + (a.H + kvh) * HD;
  const S* Vg = Kg + a.Hkv * HD;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, c = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q0 = qb + (SPLIT ? wave & 1 : wave) * 32, tq = q0 + c;
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
    const KeyTiles kt(a, qb, block_rows<SPLIT>(), n);
    Stage<S, HD> rk(Kg, a.ldq, tid), rv(Vg, a.ldq, tid);
    // scores of 32 keys, and dP plus what dp0 holds; false if no row of the
    // wavefront sees them
    f32x16v dp0 = zero16();
    auto score = [&](int k0, int sub, f32x16v& s, f32x16v& dp) {
      const int kb = k0 + 32 * sub;
      if (kb > q0 + 31 || kb >= n || (kb >= a.sinks && q0 - (kb + 31) >= a.window)) return false;
      s = zero16();
      dp = dp0;
      dot_rows<HD>(sK, 32 * sub, c, g, q, s);
      dot_rows<HD>(sV, 32 * sub, c, g, d, dp);
      dots_ahead<S, HD, 2>();
      mask_keys(a, kb, q0, tq, n, g, s);
      return true;
    };
    const bool few = a.window + a.sinks <= kFewKeys;
    if (sizeof(S) == 2 && (few || qb == 0)) {
      float sum_pdp = 0.f;
      for (int i = 0; i < (few ? kt.count : 1); ++i) {
        rk.load(kt.at(i), n, tid);
        rv.load(kt.at(i), n, tid);
        __syncthreads();
        rk.store(sK, kt.at(i), n, tid);
        rv.store(sV, kt.at(i), n, tid);
        __syncthreads();
        for (int u = 0; u < (SPLIT ? 1 : AT / 32); ++u) {
          f32x16v s, dp;
          if ((!few && q0 >= kFewKeys) || !score(kt.at(i), SPLIT ? wave >> 1 : u, s, dp)) continue;
#pragma unroll
          for (int r = 0; r < 16; ++r) sum_pdp = fmaf(__builtin_amdgcn_exp2f(fmaf(s[r], sl2, -L2)), dp[r], sum_pdp);
        }
      }
      sum_pdp += __shfl_xor(sum_pdp, 32, 64);
      if (SPLIT) {  // both wavefronts of a pair take the sum of their halves
        float* sum = reinterpret_cast<float*>(lds);
        __syncthreads();
        sum[64 * wave + lane] = sum_pdp;
        __syncthreads();
        sum_pdp = sum[64 * (wave & 1) + lane] + sum[64 * (2 + (wave & 1)) + lane];
      }
      if (few || q0 < kFewKeys) D = sum_pdp;
    }
    if (g == 0 && tq < n && (!SPLIT || wave < 2)) Dvec[stat] = D;
#pragma unroll
    for (int r = 0; r < 16; ++r) dp0[r] = -D;  // the products then give dP - D
    rk.load(kt.at(0), n, tid);
    rv.load(kt.at(0), n, tid);
    for (int i = 0; i < kt.count; ++i) {
      const int k0 = kt.at(i);
      __syncthreads();
      rk.store(sK, k0, n, tid);
      rv.store(sV, k0, n, tid);
      __syncthreads();
      if (i + 1 < kt.count) {
        rk.load(kt.at(i + 1), n, tid);
        rv.load(kt.at(i + 1), n, tid);
      }
#pragma unroll
      for (int u = 0; u < (SPLIT ? 1 : AT / 32); ++u) {
        const int sub = SPLIT ? wave >> 1 : u;
        f32x16v s, dp;
        if (!score(k0, sub, s, dp)) continue;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[r], sl2, -L2));
          dp[r] *= p;
        }
        __builtin_amdgcn_sched_barrier(0);
        add_rows<HD>(sK, 32 * sub, lane, dp, dq);
        sums_ahead<S, HD, 1>();
      }
    }
  }
  if (SPLIT) {
    join_acc<HD>(reinterpret_cast<float*>(lds), wave, lane, dq);
    if (wave >= 2) return;
  }
  if (tq < a.T)
    put_row<S, HD>(dqkv + (row0 + tq) * a.lddq + h * HD, g, dq, 1.f / sqrtf((float)HD), tq < n);
}

// ------------------------------------------- backward: dK, dV of the sinks --
// Queries from `far` on see of the first key block only the sink keys.  One
// workgroup takes a chunk of them, of every query head of a group, and 32
// sink keys; of its wavefronts two sum dV and two dK, over one half of each
// tile (half the sums a wavefront, so three share a SIMD).  The halves are
// joined in LDS and written as fp32 partials [b][kv head][chunk][dK, dV]
// [sinks][HD].  19 us at the 8192 tokens above (16 sinks), 7 at the 8 x 1024 (4):
// reading the far queries' Q and dO, and the latency of a short chunk.
template <typename S, int HD>
__global__ __launch_bounds__(256, (kWaves<S, HD>)) void window_attn_sinks(WindowAttn a, const S* qkv, const S* dO,
                                                                          const float* lse, const float* Dvec,
                                                                          int rows, int far, int chunk, int nchunk,
                                                                          float* part) {
  constexpr int NT = n_tiles<HD>();
  __shared__ __attribute__((aligned(16))) char lds[lds_bytes<S, HD, true>()];
  S *sQ = reinterpret_cast<S*>(lds), *sdO = sQ + tile_len<S, HD>();
  __shared__ float sL[AT], sD[AT];  // of a tile's queries: -lse in log2 units, -D
  const int kvh = blockIdx.x, b = blockIdx.y, ck = blockIdx.z % nchunk, kw = 32 * (blockIdx.z / nchunk);
  const int grp = a.H / a.Hkv;
  const int64_t row0 = (int64_t)b * a.T;
  const S* Kg = qkv + row0 * a.ldq + (a.H + kvh) * HD;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, c = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = length_of(a, b), key = kw + c, sub = wave >> 1;
  const bool keys = wave & 1;  // this wavefront sums dK
  // (a key block past the first one's `rows` keys covers as many more queries)
  const int qbeg = max(far + ck * chunk, far + kw / rows * rows), qend = min(n, far + (ck + 1) * chunk);
  const float sl2 = kLog2e / sqrtf((float)HD);

  f32x16v acc[NT];
  zero_acc<HD>(acc);
  if (qbeg < qend) {
    Own<S, HD> k, v;
    k.load(Kg, a.ldq, key, n, g);
    if (keys) v.load(Kg + a.Hkv * HD, a.ldq, key, n, g);
    Stage<S, HD> rq(qkv + row0 * a.ldq + kvh * grp * HD, a.ldq, tid);
    Stage<S, HD> ro(dO + row0 * a.lddo + kvh * grp * HD, a.lddo, tid);
    Stats rs;
    for (int h = kvh * grp; h < (kvh + 1) * grp; ++h) {
      for (int q0 = qbeg; q0 < qend; q0 += AT) {
        const int64_t stat = ((int64_t)b * a.H + h) * a.T;
        rq.load(q0, qend, tid);
        ro.load(q0, qend, tid);
        rs.load(lse + stat, Dvec + stat, q0, qend, tid);
        __syncthreads();
        rq.store(sQ, q0, qend, tid);
        ro.store(sdO, q0, qend, tid);
        rs.store(sL, sD, q0, qend, tid);
        __syncthreads();
        f32x16v s = zero16();
        dot_rows<HD>(sQ, 32 * sub, c, g, k, s);
        if (keys) {
          f32x16v dp;
#pragma unroll
          for (int r = 0; r < 16; ++r) dp[r] = sD[32 * sub + acc_row(r, g)];
          dot_rows<HD>(sdO, 32 * sub, c, g, v, dp);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sl2, sL[32 * sub + acc_row(r, g)])) * dp[r];
          add_rows<HD>(sQ, 32 * sub, lane, s, acc);
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sl2, sL[32 * sub + acc_row(r, g)]));
          add_rows<HD>(sdO, 32 * sub, lane, s, acc);
        }
      }
      rq.src += HD;
      ro.src += HD;
    }
  }
  join_acc<HD>(reinterpret_cast<float*>(lds), wave, lane, acc);
  if (wave < 2 && key < a.sinks)
    put_row<float, HD>(part + (((((int64_t)b * a.Hkv + kvh) * nchunk + ck) * 2 + (1 - wave)) * a.sinks + key) * HD, g,
                       acc, 1.f, true);
}

// ------------------------------------------------------- backward: dK, dV --
// A group's query heads may be divided over `parts` workgroups, which then
// write fp32 sums [part][b][t][dK, dV][kv head][HD] for window_attn_kv_sum.
// 156 us at the 8192 tokens above (838 TFLOP/s), 28 at the 8 x 1024.
template <typename S, int HD, bool SPLIT>
__global__ __launch_bounds__(256, (kWavesDkdv<S, HD>)) void window_attn_dkdv(WindowAttn a, const S* qkv, const S* dO,
                                                                             const float* lse, const float* Dvec,
                                                                             const float* part, int nchunk, int parts,
                                                                             float* heads, S* dqkv) {
  constexpr int NT = n_tiles<HD>();
  constexpr bool KL = kKeysInLds<S, HD>, LATE = KL && HD == 128;
  __shared__ __attribute__((aligned(16))) S sK[KL ? block_rows<SPLIT>() / AT * tile_len<S, HD>() : 8];
  __shared__ __attribute__((aligned(16))) char lds[lds_bytes<S, HD, SPLIT>()];
  S *sQ = reinterpret_cast<S*>(lds), *sdO = sQ + tile_len<S, HD>();
  __shared__ float sL[AT], sD[AT];  // of a tile's queries: -lse in log2 units, -D
  const int kvh = blockIdx.x / parts, b = blockIdx.y, kb0 = block_rows<SPLIT>() * blockIdx.z;
  const int grp = a.H / a.Hkv / parts, h0 = blockIdx.x * grp;  // this workgroup's query heads
  const int64_t row0 = (int64_t)b * a.T;
  const S* Kg = qkv + row0 * a.ldq + (a.H + kvh) * HD;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, c = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = kb0 + (SPLIT ? wave & 1 : wave) * 32, key = kw + c;
  const int n = length_of(a, b);
  const float sl2 = kLog2e / sqrtf((float)HD);

  f32x16v dk[NT], dv[NT];
  zero_acc<HD>(dk);
  zero_acc<HD>(dv);
  if (kb0 < n) {
    Own<S, HD> k, v;
    if (KL) {
      for (int r0 = 0; r0 < block_rows<SPLIT>(); r0 += AT) {
        Stage<S, HD> rk(Kg, a.ldq, tid);
        rk.load(kb0 + r0, n, tid);
        rk.store(sK + r0 / AT * tile_len<S, HD>(), kb0 + r0, n, tid);
      }
    } else {
      k.load(Kg, a.ldq, key, n, g);
    }
    const S* ownK = sK + row_off<HD>(sK, kw - kb0);
    v.load(Kg + a.Hkv * HD, a.ldq, key, n, g);
    // query tiles kb0 + 64 i that some key of the block has in its window
    const int nq = (min(n - kb0, block_rows<SPLIT>() - 1 + a.window) + AT - 1) / AT;
    const int nit = grp * nq;
    Stage<S, HD> rq(qkv + row0 * a.ldq + h0 * HD, a.ldq, tid);
    Stage<S, HD> ro(dO + row0 * a.lddo + h0 * HD, a.lddo, tid);
    Stats rs;
    const float *hL = lse + ((int64_t)b * a.H + h0) * a.T, *hD = Dvec + ((int64_t)b * a.H + h0) * a.T;
    if (!LATE) {
      rq.load(kb0, n, tid);
      ro.load(kb0, n, tid);
      rs.load(hL, hD, kb0, n, tid);
    }
    int qi = 0;
    for (int it = 0; it < nit; ++it) {
      const int q0 = kb0 + AT * qi;
      if (LATE) {
        rq.load(q0, n, tid);
        ro.load(q0, n, tid);
        rs.load(hL, hD, q0, n, tid);
      }
      __syncthreads();
      rq.store(sQ, q0, n, tid);
      ro.store(sdO, q0, n, tid);
      rs.store(sL, sD, q0, n, tid);
      __syncthreads();
      if (++qi == nq) {
        qi = 0;
        rq.src += HD;
        ro.src += HD;
        hL += a.T;
        hD += a.T;
      }
      if (!LATE && it + 1 < nit) {
        rq.load(kb0 + AT * qi, n, tid);
        ro.load(kb0 + AT * qi, n, tid);
        rs.load(hL, hD, kb0 + AT * qi, n, tid);
      }
#pragma unroll
      for (int u = 0; u < (SPLIT ? 1 : AT / 32); ++u) {
        const int sub = SPLIT ? wave >> 1 : u;
        const int qs = q0 + 32 * sub;
        if (qs + 31 < kw || qs >= n) continue;                      // before this wavefront's keys, or past the end
        if (kw >= a.sinks && qs - (kw + 31) >= a.window) continue;  // past the window of all its keys
        f32x16v s = zero16(), dp;  // dp from -D on: the products give dP - D
#pragma unroll
        for (int r = 0; r < 16; ++r) dp[r] = sD[32 * sub + acc_row(r, g)];
        if (KL) dot_rows<HD>(sQ, 32 * sub, c, g, ownK, s);
        else dot_rows<HD>(sQ, 32 * sub, c, g, k, s);
        dot_rows<HD>(sdO, 32 * sub, c, g, v, dp);
        dots_ahead<S, HD, 2>();
        // queries past n have zero Q, dO, L and D: they add nothing
        mask_queries(a, qs, kw, key, g, s);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], sl2, sL[32 * sub + acc_row(r, g)]));
          dp[r] *= s[r];
        }
        __builtin_amdgcn_sched_barrier(0);
        add_rows<HD>(sdO, 32 * sub, lane, s, dv);
        add_rows<HD>(sQ, 32 * sub, lane, dp, dk);
        sums_ahead<S, HD, 2>();
      }
    }
  }
  if (SPLIT) {
    join_acc<HD>(reinterpret_cast<float*>(lds), wave, lane, dk);
    join_acc<HD>(reinterpret_cast<float*>(lds), wave, lane, dv);
  }
  if (part && parts == 1 && kb0 < a.sinks && kb0 < n) {
    // the far queries' partials: for each 32 keys the workgroup sums the
    // chunks into LDS, in order, and the keys' wavefront adds them
    float* sum = reinterpret_cast<float*>(lds);
    const float* base = part + ((int64_t)b * a.Hkv + kvh) * nchunk * 2 * a.sinks * HD;
    for (int k0 = kb0; k0 < min(kb0 + block_rows<SPLIT>(), a.sinks); k0 += 32) {
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        __syncthreads();
        const float* p = base + (which * a.sinks + k0) * HD;
        for (int i = tid; i < min(32, a.sinks - k0) * (HD / 4); i += 256) {
          f32x4v t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
          for (int ck = 0; ck < nchunk; ++ck)
            t += *reinterpret_cast<const f32x4v*>(p + (int64_t)ck * 2 * a.sinks * HD + 4 * i);
          float* to = sum + (HD + 1) * (i / (HD / 4)) + 4 * (i % (HD / 4));
#pragma unroll
          for (int j = 0; j < 4; ++j) to[j] = t[j];
        }
        __syncthreads();
        if (kw == k0 && key < a.sinks) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < (HD < 32 ? 8 : 16); ++r) {
              const float x = sum[(HD + 1) * c + 32 * t + acc_row(r, g)];
              if (which) dv[t][r] += x;
              else dk[t][r] += x;
            }
        }
      }
    }
  }
  if (SPLIT && wave >= 2) return;
  if (parts > 1) {
    if (key < n) {
      float* row = heads + ((((blockIdx.x % parts) * (int64_t)a.B + b) * a.T + key) * 2 * a.Hkv + kvh) * HD;
      put_row<float, HD>(row, g, dk, 1.f, true);
      put_row<float, HD>(row + a.Hkv * HD, g, dv, 1.f, true);
    }
    return;
  }
  if (key < a.T) {
    S* row = dqkv + (row0 + key) * a.lddq + (a.H + kvh) * HD;
    put_row<S, HD>(row, g, dk, 1.f / sqrtf((float)HD), key < n);
    put_row<S, HD>(row + a.Hkv * HD, g, dv, 1.f, key < n);
  }
}

// Joins the parts of a group's heads and, for sink keys, the far queries'
// chunks, each in order: four dims a thread.
template <typename S, int HD>
__global__ __launch_bounds__(256) void window_attn_kv_sum(WindowAttn a, const float* part, int nchunk, int parts,
                                                          const float* heads, S* dqkv) {
  const int width = 2 * a.Hkv * HD;
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, rows = (int64_t)a.B * a.T;
  if (i >= rows * width) return;
  const int64_t row = i / width;
  const int col = (int)(i % width), b = (int)(row / a.T), key = (int)(row % a.T);
  f32x4v t = {0.f, 0.f, 0.f, 0.f};
  if (key < length_of(a, b)) {
    for (int p = 0; p < parts; ++p) t += *reinterpret_cast<const f32x4v*>(heads + p * rows * width + i);
    if (part && key < a.sinks) {
      const int which = col / (a.Hkv * HD), kvh = col % (a.Hkv * HD) / HD, dim = col % HD;
      const float* p = part + (((int64_t)b * a.Hkv + kvh) * nchunk * 2 + which) * a.sinks * HD + key * HD + dim;
#pragma unroll 8
      for (int ck = 0; ck < nchunk; ++ck) t += *reinterpret_cast<const f32x4v*>(p + (int64_t)ck * 2 * a.sinks * HD);
    }
  }
  const float mul = col < a.Hkv * HD ? 1.f / sqrtf((float)HD) : 1.f;
  put4(dqkv + row * a.lddq + a.H * HD + col, t[0] * mul, t[1] * mul, t[2] * mul, t[3] * mul);
}

// ------------------------------------------------------------- launching --
namespace {

// Whether to halve the blocks: while whole ones would not fill the chip's 256
// compute units `per_cu` times over, what counts is the time of one (one
// sequence of 2048 tokens, 8 heads of 64, window 512, 128 workgroups: forward
// 16.8 -> 11.7 us, dQ 19.1 -> 14.2, dK/dV 23.6 -> 17.4); past that the halves
// read the other dimension's tiles twice as often (8 sequences of 1024, 12
// heads, window 256, 768 workgroups: 21.2 -> 23.6, 26.7 -> 31.0, 35.1 ->
// 37.6).
bool split_rows(const WindowAttn& a, int heads, int per_cu) {
  return (int64_t)heads * a.B * cdiv(a.T, 128) < 256 * per_cu;
}
// Workgroups that share a compute unit: as the registers have it, but two for the
// dK/dV of bf16 heads of 64, where three have place.  With whole blocks from 512
// workgroups on against 768, both passes of sequences of 2048 tokens: under a
// window of 512 72.6 against 74.4 us at 512 workgroups, 77.9 against 80.4 at 576,
// 82.6 against 83.1 at 640; under the full mask 146 against 133 at 512, 156
// against 152 at 640, 163 against 161 at 704.
template <typename S, int HD>
constexpr int kPerCu = HD < 64 ? 3 : 2;
template <typename S, int HD>
constexpr int kPerCuBwd = kWide<S, HD> ? 1 : kPerCu<S, HD>;
// The backward kernels.  A workgroup that has a compute unit to itself (kWide)
// runs in rounds of 256: halves are taken where they need fewer half rounds by
// more than the ninth that they cost (heads of 128, both passes: 384 workgroups
// of 2048 tokens, window 512, 789 -> 662 us; 896, window 300, 1138 -> 1087; but
// 1152, 1320 -> 1337, and 256 of 1999 tokens, window 300, dQ 113 -> 121), and
// where the longest block, which under a wide window sees most keys, would end
// last (256 of 4096 tokens, full mask: 2223 -> 1470).
template <typename S, int HD>
bool split_rows_bwd(const WindowAttn& a, int heads) {
  if (!kWide<S, HD>) return split_rows(a, heads, kPerCuBwd<S, HD>);
  const int64_t cols = (int64_t)heads * a.B;
  if (2 * ((int64_t)a.window + a.sinks) > a.T && cols * cdiv(a.T, 128) < 512) return true;
  const int64_t whole = (cols * cdiv(a.T, 128) + 255) / 256, halves = (cols * cdiv(a.T, 64) + 255) / 256;
  return 10 * halves < 18 * whole;
}

template <typename S, int HD, bool SPLIT>
hipError_t fwd(const WindowAttn& a, const void* qkv, void* O, float* lse, hipStream_t s) {
  hipLaunchKernelGGL((window_attn_fwd<S, HD, SPLIT>), dim3(a.H, a.B, cdiv(a.T, block_rows<SPLIT>())), dim3(256), 0, s,
                     a, static_cast<const S*>(qkv), static_cast<S*>(O), lse);
  return hipGetLastError();
}

template <typename S, int HD, bool SPLIT>
hipError_t dq(const WindowAttn& a, const void* qkv, const void* O, const void* dO, const float* lse, float* Dvec,
              void* dqkv, hipStream_t s) {
  hipLaunchKernelGGL((window_attn_dq<S, HD, SPLIT>), dim3(a.H, a.B, cdiv(a.T, block_rows<SPLIT>())), dim3(256), 0, s,
                     a, static_cast<const S*>(qkv), static_cast<const S*>(O), static_cast<const S*>(dO), lse, Dvec,
                     static_cast<S*>(dqkv));
  return hipGetLastError();
}

// How dK and dV of a shape are computed.
struct Plan {
  int parts;       // workgroups that share a key/value head's query heads
  bool split;      // blocks of 64 keys
  int far, chunk, nchunk;
  int64_t sinks, heads;  // floats of partial sums
};
template <typename S, int HD>
Plan plan_dkdv(const WindowAttn& a) {
  Plan p;
  // Shared key/value heads make few workgroups of much work: where halved
  // blocks would not fill the chip either, their query heads are divided until
  // they do (one sequence of 4096 tokens, 16 heads of 128 sharing 2, window
  // 1024, both passes: 376 -> 223 us), while the fp32 sums of the parts
  // fit the scratch.
  constexpr int kFull = kPerCuBwd<S, HD>;
  const int grp = a.H / a.Hkv;
  const int64_t per_part = (int64_t)a.B * a.T * 2 * a.Hkv * HD;
  p.parts = 1;
  if (split_rows(a, 2 * a.Hkv, kFull))
    for (int d = 2; d <= grp; ++d)
      if (grp % d == 0 && split_rows(a, a.Hkv * p.parts, kFull) && d * per_part <= kWindowPartFloats)
        p.parts = d;
  p.split = split_rows_bwd<S, HD>(a, a.Hkv * p.parts);
  // Queries from `far` on reach the first key block through its sink keys
  // only (the end of the last tile that its own range walks).  Their chunks:
  // enough workgroups to fill the chip twice over, and none under a tile.
  const int rows = p.split ? 64 : 128;
  p.far = (int)(((int64_t)a.window + rows - 1 + AT - 1) / AT * AT);
  p.nchunk = p.chunk = 0;
  if (a.sinks > 0 && p.far < a.T) {
    const int64_t have = (int64_t)a.B * a.Hkv * cdiv(a.sinks, 32);
    p.nchunk = (int)std::min<int64_t>((512 + have - 1) / have, cdiv(a.T - p.far, AT));
    p.chunk = cdiv(cdiv(a.T - p.far, p.nchunk), AT) * AT;
  }
  p.sinks = (int64_t)a.B * a.Hkv * p.nchunk * 2 * a.sinks * HD;
  p.heads = p.parts > 1 ? p.parts * per_part : 0;
  return p;
}

template <typename S, int HD, bool SPLIT>
hipError_t dkdv(const WindowAttn& a, const Plan& p, const void* qkv, const void* dO, const float* lse,
                const float* Dvec, float* part, void* dqkv, hipStream_t s) {
  const S *x = static_cast<const S*>(qkv), *g = static_cast<const S*>(dO);
  float* heads = part + p.sinks;
  if (p.nchunk > 0) {
    hipLaunchKernelGGL((window_attn_sinks<S, HD>), dim3(a.Hkv, a.B, p.nchunk * cdiv(a.sinks, 32)), dim3(256), 0, s, a,
                       x, g, lse, Dvec, block_rows<SPLIT>(), p.far, p.chunk, p.nchunk, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.nchunk == 0) part = nullptr;
  hipLaunchKernelGGL((window_attn_dkdv<S, HD, SPLIT>), dim3(a.Hkv * p.parts, a.B, cdiv(a.T, block_rows<SPLIT>())),
                     dim3(256), 0, s, a, x, g, lse, Dvec, part, p.nchunk, p.parts, heads, static_cast<S*>(dqkv));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  const int64_t quads = (int64_t)a.B * a.T * 2 * a.Hkv * HD / 4;
  hipLaunchKernelGGL((window_attn_kv_sum<S, HD>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, a, part,
                     p.nchunk, p.parts, heads, static_cast<S*>(dqkv));
  return hipGetLastError();
}

template <typename S, int HD>
hipError_t bwd(const WindowAttn& a, const void* qkv, const void* O, const void* dO, const float* lse, float* Dvec,
               float* part, void* dqkv, hipStream_t s) {
  const hipError_t e = split_rows_bwd<S, HD>(a, a.H) ? dq<S, HD, true>(a, qkv, O, dO, lse, Dvec, dqkv, s)
                                                     : dq<S, HD, false>(a, qkv, O, dO, lse, Dvec, dqkv, s);
  if (e != hipSuccess) return e;
  const Plan p = plan_dkdv<S, HD>(a);
  return p.split ? dkdv<S, HD, true>(a, p, qkv, dO, lse, Dvec, part, dqkv, s)
                 : dkdv<S, HD, false>(a, p, qkv, dO, lse, Dvec, part, dqkv, s);
}

template <typename S, int HD>
int64_t scratch(const WindowAttn& a) {
  const Plan p = plan_dkdv<S, HD>(a);
  return p.sinks + p.heads;
}

}  // namespace

#define FAL_BY_HEAD(S, CALL, bad)                                \
  switch (a.hd) {                                             \
    case 16: return CALL(S, 16);                              \
    case 32: return CALL(S, 32);                              \
    case 64: return CALL(S, 64);                              \
    case 128: return CALL(S, 128);                            \
    default: return bad;                                      \
  }

hipError_t window_attention_fwd(DType dt, const WindowAttn& a, const void* qkv, void* O, float* lse, hipStream_t s) {
#define FAL_FWD(S, HD)                                                       \
  (split_rows(a, a.H, kPerCu<S, HD>) ? fwd<S, HD, true>(a, qkv, O, lse, s)   \
                                     : fwd<S, HD, false>(a, qkv, O, lse, s))
  if (dt == BF16) FAL_BY_HEAD(bf16, FAL_FWD, hipErrorInvalidValue)
  FAL_BY_HEAD(float, FAL_FWD, hipErrorInvalidValue)
#undef FAL_FWD
}

hipError_t window_attention_bwd(DType dt, const WindowAttn& a, const void* qkv, const void* O, const void* dO,
                                const float* lse, float* Dvec, float* part, void* dqkv, hipStream_t s) {
#define FAL_BWD(S, HD) (bwd<S, HD>(a, qkv, O, dO, lse, Dvec, part, dqkv, s))
  if (dt == BF16) FAL_BY_HEAD(bf16, FAL_BWD, hipErrorInvalidValue)
  FAL_BY_HEAD(float, FAL_BWD, hipErrorInvalidValue)
#undef FAL_BWD
}

int64_t window_attention_scratch(DType dt, const WindowAttn& a) {
#define FAL_SCRATCH(S, HD) (scratch<S, HD>(a))
  if (dt == BF16) FAL_BY_HEAD(bf16, FAL_SCRATCH, 0)
  FAL_BY_HEAD(float, FAL_SCRATCH, 0)
#undef FAL_SCRATCH
}
#undef FAL_BY_HEAD

}  // namespace fal
