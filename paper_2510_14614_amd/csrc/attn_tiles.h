// Tiles and operand fragments shared by the attention kernels on the gfx950
// matrix cores: 64-row LDS tiles of a head's Q, K, V or dO, staged through
// registers, and the reads that feed v_mfma_f32_32x32x16_bf16.
#pragma once

#include <hip/hip_runtime.h>

#include "common.h"

namespace fal {

typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4v __attribute__((ext_vector_type(4)));
typedef float f32x16v __attribute__((ext_vector_type(16)));

constexpr int AT = 64;        // rows per LDS tile of the streamed dimension
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ f32x16v mfma32(bf16x8v a, bf16x8v b, f32x16v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ f32x16v zero16() {
  f32x16v z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// 8 bf16 made of two runs of 4 (each 8 bytes, 8-byte aligned)
__device__ __forceinline__ bf16x8v ld_2x4(const bf16* p0, const bf16* p1) {
  const bf16x4v a = *reinterpret_cast<const bf16x4v*>(p0);
  const bf16x4v b = *reinterpret_cast<const bf16x4v*>(p1);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ bf16x8v pack8(const f32x16v& v, int base) {
  bf16x8v o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = static_cast<bf16>(v[base + j]);
  return o;
}

// Row r of the 32x32 accumulator tile held by lane group g.
__device__ __forceinline__ int acc_row(int r, int g) { return 8 * (r >> 2) + 4 * g + (r & 3); }

// Tiles of AT rows (row0.., zero past T) of a head slice, staged through
// registers: load() issues the global loads (rows past T read a clamped
// row), store() writes LDS (zeroing rows past T).  Loading the next tile
// before computing on the current one keeps its memory latency behind the
// MFMA work.
//
// LDS tiles hold rows of HD contiguous elements, 16 rows to a group of
// 16 (HD + 8) elements; inside a group, row r sits in slot m(r) at a stride
// of HD + 8 elements.  Measured with the SQ LDS counters, a wavefront's
// 16-byte read occupies the LDS 4 cycles and an 8-byte transposing read 2
// when free of bank conflicts, a 16-byte write 8; for the access patterns
// of these tiles the conflicts follow 16 consecutive lanes (32 for the
// transposing read) per cycle over 256 bytes of banks.  A slot stride of
// HD + 8 elements puts slot j's 16-byte chunk c at bank group
// (j (HD/8 + 1) + c) mod 16, and the slots are permuted so that, with
// s(r) = 8 (r & 1) + 4 ((r >> 1) & 1) + ((r >> 2) & 3) the bank group of
// row r's chunk 0:
//  * row reads (16 consecutive rows, one chunk each) meet 16 values of s;
//  * transposing reads (4 consecutive rows, 4 adjacent chunks each) meet s
//    values 4 apart, so the rows' chunk runs tile the 16 bank groups;
//  * stores (8 lanes: 128 bytes of one row) cover distinct bank groups.
// The counters read no conflicts in any kernel of attention_mfma.hip; rows in
// order at the same stride left the transposing reads four-way conflicted at
// head_dim 128 and two-way at 64.  m(r) = s(r) at HD = 128 (stride 17
// chunks, 17 = 1 mod 16) and 9 s(r) mod 16 at HD = 64 (stride 9,
// 9 * 9 = 1 mod 16).  Narrower heads keep their rows in order: no inverse of
// their chunk stride puts row r + 8 at a fixed distance from row r.
// trow(a + b) = trow(a) + trow(b) for a a multiple of 16, and trow(r + 8) =
// trow(r) + trow8() for r % 16 < 8: callers split a row into a part known
// at compile time and a per-lane part, so every fragment offset is an
// immediate.
template <int HD>
__device__ __forceinline__ int trow(int r) {
  if (HD < 64) return (HD + 8) * r;
  const int x = r & 15;
  const int s = ((x & 1) << 3) | ((x & 2) << 1) | ((x >> 2) & 3);
  const int m = HD == 128 ? s : (9 * s) & 15;
  return (HD + 8) * (16 * (r >> 4) + m);
}
template <int HD>
constexpr int trow8() { return (HD < 64 ? 8 : 2) * (HD + 8); }
// elements of an AT-row tile
template <int HD>
constexpr int tile_elems() { return AT * (HD + 8); }

template <int HD>
struct RowTile {
  static constexpr int CH = HD / 8, N = (AT * CH + 255) / 256;
  uint4 v[N];
  __device__ __forceinline__ void load(const bf16* src, int64_t ld, int row0, int T, int tid) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = tid + 256 * k;
      const int r = i / CH, c = (i % CH) * 8;
      const int row = min(row0 + r, T - 1);
      if (i < AT * CH) v[k] = *reinterpret_cast<const uint4*>(src + (int64_t)row * ld + c);
    }
  }
  __device__ __forceinline__ void store(bf16* s, int row0, int T, int tid) const {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int i = tid + 256 * k;
      if (i >= AT * CH) continue;
      const int r = i / CH, c = i % CH;
      *reinterpret_cast<uint4*>(s + trow<HD>(r) + 8 * c) = row0 + r < T ? v[k] : make_uint4(0, 0, 0, 0);
    }
  }
};

// A or B operand fragment from an LDS tile: row rowbase + r (rowbase a
// multiple of 16), dims 16*kk + 8*g .. +7.
template <int HD>
__device__ __forceinline__ bf16x8v frag_rows(const bf16* s, int rowbase, int r, int kk, int g) {
  return *reinterpret_cast<const bf16x8v*>(s + trow<HD>(rowbase) + trow<HD>(r) + 16 * kk + 8 * g);
}

// Operand fragment for a contraction over the rows of an LDS tile (rowbase
// a multiple of 16): lane (c = lane % 32, g = lane / 32) gets column colbase + c
// of rows rowbase + {4g..4g+3, 8+4g..8+4g+3}, the order in which the
// accumulator registers of a 32x32 tile hold them.  ds_read_b64_tr_b16
// hands lane i of each 16-lane group element i % 4 of the 8-byte chunks
// addressed by lanes 4j + i / 4 (j = 0..3): lane L addresses row
// rowbase + 4g + L / 4 (then + 8), columns 4 (L % 4)..+3 of its group's 16.
typedef short i16x4v __attribute__((ext_vector_type(4)));
template <int HD>
__device__ __forceinline__ bf16x8v frag_tr(const bf16* s, int rowbase, int colbase, int lane) {
  const int L = lane & 15;
  // (head_dim 16 has 16 columns: the upper lanes repeat them)
  const int col = colbase + (HD < 32 ? 0 : 16 * ((lane >> 4) & 1)) + 4 * (L & 3);
  const bf16* p = s + trow<HD>(rowbase) + trow<HD>(4 * (lane >> 5) + (L >> 2)) + col;
  typedef __attribute__((address_space(3))) i16x4v lds_i16x4;
  const lds_i16x4* p0 = reinterpret_cast<const lds_i16x4*>((__attribute__((address_space(3))) const char*)p);
  const lds_i16x4* p1 =
      reinterpret_cast<const lds_i16x4*>((__attribute__((address_space(3))) const char*)(p + trow8<HD>()));
  const i16x4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(const_cast<lds_i16x4*>(p0));
  const i16x4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(const_cast<lds_i16x4*>(p1));
  const i16x4v* pa = &a;
  const i16x4v* pb = &b;
  return ld_2x4(reinterpret_cast<const bf16*>(pa), reinterpret_cast<const bf16*>(pb));
}

// Operand fragment straight from global memory (row of a head slice).
template <int HD>
__device__ __forceinline__ bf16x8v frag_global(const bf16* src, int64_t ld, int row, int T, int kk, int g) {
  if (row >= T) {
    bf16x8v z;
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = static_cast<bf16>(0.f);
    return z;
  }
  return *reinterpret_cast<const bf16x8v*>(src + (int64_t)row * ld + 16 * kk + 8 * g);
}

// Scheduling groups for a run of N MFMAs that take R LDS read instructions
// each: the reads of the next LA MFMAs stay in flight, so a fragment read
// is not waited for right before its MFMA (head_dim 128, where one
// wavefront per SIMD leaves nothing else to cover that wait).  Ends the
// scheduling region.
template <int N, int R, int LA>
__device__ __forceinline__ void lds_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, R * LA, 0);  // LDS reads of the first LA MFMAs
#pragma unroll
  for (int q = 0; q < N - LA; ++q) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);  // LDS reads of the MFMA LA ahead
  }
  __builtin_amdgcn_sched_group_barrier(0x008, LA, 0);
  __builtin_amdgcn_sched_barrier(0);
}

}  // namespace fal
