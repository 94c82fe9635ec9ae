// Shared by the kernels of 16-bit matrix products: operand slices copied from
// global memory straight into LDS, fragment reads from there, and the pieces
// of their epilogues.
//
// LDS layout of one operand in one stage (R rows of the output dimension,
// slices of 32 k):
//  * k-contiguous operand: R rows of 32 k (64 B), 16-byte chunk c of row r
//    stored at chunk c ^ ((r >> 2) & 3): the 16 rows of a fragment read
//    (one chunk each) fall in 16 different 16-byte bank groups.
//  * MN-major operand: 32 k-rows of R elements, 32-byte segment q of k-row k
//    stored at segment q ^ g(k), g(k) = (k & 3) | ((k >> 3) & 1) << 2: the
//    16 k-rows touched by one transposing read hit each 32-byte bank group
//    exactly twice (the minimum for 512 bytes).  Tiles of 64 rows have four
//    segments a k-row and start every second k-row 128 bytes apart:
//    g(k) = ((k >> 1) & 1) | ((k >> 3) & 1) << 1.
#pragma once

#include "common.h"
#include "gemm_tiles.h"

namespace fal {

// ----------------------------------------------------------- MFMA (bf16) --
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kRsrcWord3 = 0x00020000;  // gfx9-family buffer descriptor word 3

// An operand whose contraction dimension is strided (MN-major: the weight of
// a forward layer, both operands of a weight gradient) is staged as loaded,
// [k][row], and read back with the gfx950 LDS transpose load.
// ds_read_b64_tr_b16 gives lane i of each 16-lane group element i % 4 of the
// 8-byte chunks addressed by lanes 4j + i / 4 (j = 0..3); lane L therefore
// addresses k-row kb + L / 4, rows 4 (L % 4)..+3 of the fragment, and two
// reads (kb, kb + 4) return the eight consecutive k a 16x16x32 operand lane
// holds.
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;

__device__ __forceinline__ i16x4_t lds_read_tr(const bf16* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_i16x4_t*)((__attribute__((address_space(3))) char*)(const_cast<bf16*>(p))));
}

__device__ __forceinline__ void ld4(const bf16* p, float (&v)[4]) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xFFFF0000u);
  v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xFFFF0000u);
}
__device__ __forceinline__ void st4(bf16* p, const float (&v)[4]) {
  union { bf16 h[4]; uint2 w; } u;
#pragma unroll
  for (int c = 0; c < 4; ++c) u.h[c] = from_f<bf16>(v[c]);
  *reinterpret_cast<uint2*>(p) = u.w;
}

// Orders this wavefront's LDS writes before its later reads (and reads
// before later writes) without a workgroup barrier: LDS executes one
// wavefront's instructions in order, so only compiler motion must be stopped.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

namespace pipe {
constexpr int KS = 32;
constexpr uint32_t kOob = 0x80000000u;      // offset beyond any buffer range (ranges are < 2^31)

template <int R>
__device__ __forceinline__ int mn_g(int k) {
  return R >= 128 ? (k & 3) | (((k >> 3) & 1) << 2) : ((k >> 1) & 1) | (((k >> 3) & 1) << 1);
}

// Bytes that an operand's buffer spans from its element (r0, 0), r0 the tile's first
// row of the output dimension.  MN-major: up to the last whole 16-byte chunk of the
// last k-row's own Rmax elements, not to the end of its stride: of a matrix that is
// the right-hand columns of a wider one, what follows them there belongs to nobody.
// k-contiguous: whole strides; loads past K are pointed out of range one by one.
__host__ __device__ __forceinline__ int64_t operand_bytes(int kmaj, int64_t ld, int r0, int Rmax, int K) {
  return kmaj ? (Rmax - r0) * ld * 2 : ((K - 1) * ld + ((Rmax + 7) & ~7) - r0) * 2;
}

typedef __attribute__((address_space(3))) void lds_void_t;
__device__ __forceinline__ lds_void_t* lds_ptr(const void* p) {
  return (lds_void_t*)((__attribute__((address_space(3))) char*)(const_cast<void*>(p)));
}

// One operand's loader (both K segments) for slices W wide in K (32 or
// 64).  Load block i of this wavefront is block 4 i + wave of the stage
// region; its global offset is a per-lane part (which repeats with period
// NV in i) plus a wave-uniform step per i.
//  * k-contiguous: a block holds RPI = 1024 / 2W rows of W k; the 16-byte
//    chunk c of row r sits at c ^ kswz(r), kswz(r) = (r >> 2) & 3 for
//    64-byte rows and (r >> 1) & 7 for 128-byte rows.
//  * MN-major: a block holds 1024 / 2R k-rows of R elements, 32-byte
//    segment q of k-row k at q ^ g(k).
template <int W>
__device__ __forceinline__ int kswz(int r) { return W == 32 ? (r >> 2) & 3 : (r >> 1) & 7; }

template <int R, int KMAJ, int W = KS>
struct Src {
  static constexpr int BYTES = R * W * 2;                  // one stage region
  static constexpr int NINS = BYTES / 1024;                // 1 KiB load blocks per slice
  static constexpr int IPW = NINS / 4;                     // per wavefront
  static constexpr int CPR = R / 8;                        // MN-major: 16-byte chunks per k-row
  static constexpr int CPRK = W / 8;                       // k-contiguous: 16-byte chunks per row
  static constexpr int RPI = KMAJ ? 1024 / (2 * W) : 1024 / (2 * R);  // rows / k-rows per block
  // MN-major: the swizzle g(k) of a lane's k-row repeats every 16 k-rows
  static constexpr int NV = KMAJ ? 1 : ((4 * RPI) % 16 == 0 ? 1 : 16 / (4 * RPI));
  static_assert(NINS % 4 == 0 && IPW % NV == 0 && R >= 64, "tile too small for four wavefronts");
  uint32_t voff[2][NV];    // per segment
  uint32_t istep[2];       // bytes from block i to block i + 1 of this wavefront
  int kof;                 // k-contiguous: k offset of this lane's chunk within the slice
  uint64_t base[2];
  int nbytes[2];
  uint32_t kstep[2];       // bytes per k (k-contiguous: 2; MN-major: 2 ld)

  __device__ __forceinline__ void init(int seg, const bf16* X, int64_t ld, int r0, int Rmax, int Kseg, int wave,
                                       int lane) {
    base[seg] = reinterpret_cast<uint64_t>(KMAJ ? X + (int64_t)r0 * ld : X + r0);
    nbytes[seg] = (int)min<int64_t>(operand_bytes(KMAJ, ld, r0, Rmax, Kseg), 0x7fffffff);
    kstep[seg] = KMAJ ? 2u : (uint32_t)(ld * 2);
    istep[seg] = (uint32_t)(4 * RPI * ld * 2);
    if (KMAJ) {
      // kswz(row) does not depend on the block index i (rows advance by 4 RPI)
      const int row = wave * RPI + lane / CPRK;
      const int gc = (lane % CPRK) ^ kswz<W>(row);
      voff[seg][0] = (uint32_t)(((int64_t)row * ld + gc * 8) * 2);
      kof = gc * 8;
    } else {
      kof = 0;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int k = (4 * v + wave) * RPI + lane / CPR;
        const int gc = (lane % CPR) ^ (2 * mn_g<R>(k));
        voff[seg][v] = (uint32_t)(((int64_t)k * ld + gc * 8) * 2);
      }
    }
  }
  __device__ __forceinline__ void clear(int seg) {
    base[seg] = base[0];
    nbytes[seg] = 0;
    kstep[seg] = istep[seg] = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) voff[seg][v] = kOob;
  }

  // Load state: the slice the next load() fetches.
  uint32_t rlo, rhi;
  int rn;
  uint32_t so, is, ks;
  uint32_t vo[NV];
  // Point the state at the slice at k0 of segment seg; chunks at slice
  // offset >= lim are pointed out of range (lim: 0 for a slice past the
  // end, K - k0 in a k-contiguous tail slice, W otherwise).
  __device__ __forceinline__ void set(int seg, int k0, int lim) {
    const uint64_t b = seg ? base[1] : base[0];
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b);
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
    rlo = lo;
    rhi = hi;
    rn = __builtin_amdgcn_readfirstlane(seg ? nbytes[1] : nbytes[0]);
    ks = __builtin_amdgcn_readfirstlane(seg ? kstep[1] : kstep[0]);
    so = (uint32_t)k0 * ks;
    is = __builtin_amdgcn_readfirstlane(seg ? istep[1] : istep[0]);
    const bool bad = kof >= lim;
#pragma unroll
    for (int v = 0; v < NV; ++v) vo[v] = bad ? kOob : (seg ? voff[1][v] : voff[0][v]);
  }
  // set() to the first slice of segment 0 of an operand below 2 GiB, for kernels
  // whose state only advances from there.  Its bytes are counted without init()'s
  // 64-bit minimum: that is left in a vector register, uniform as it is, and a load
  // whose descriptor holds it becomes a loop over lanes.
  __device__ __forceinline__ void start(int64_t ld, int r0, int Rmax, int Kseg) {
    set(0, 0, W);
    rn = (int)operand_bytes(KMAJ, ld, r0, Rmax, Kseg);
  }
  // Next slice of the same segment (full and live).
  __device__ __forceinline__ void advance() { so += W * ks; }
  // Chunks of segment 0 at slice offset >= lim out of range from here on
  // (k-contiguous operands; an MN-major one's rows past K are out of its buffer's
  // range by themselves).
  __device__ __forceinline__ void limit(int lim) {
    if (KMAJ) vo[0] = kof >= lim ? kOob : voff[0][0];
  }
  // Issue this wavefront's loads of the current slice into the region at dst.
  __device__ __forceinline__ void load(char* dst, int wave) const {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>(((uint64_t)rhi << 32) | rlo), (short)0, rn, kRsrcWord3);
    // (the offsets go through locals: with member expressions as builtin
    // arguments the host pass drops the kernel's launch stubs)
#pragma unroll
    for (int i = 0; i < IPW; ++i) {
      const uint32_t v = vo[i % NV];
      const uint32_t o = so + (uint32_t)(i - i % NV) * is;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, lds_ptr(dst + (i * 4 + wave) * 1024), 16, v, o, 0, 0);
    }
  }
};

// Fragment reads from one stage region (byte addresses precomputed per
// lane); fragment f of MFMA k-step kk (0 .. W/32 - 1).
template <int R, int KMAJ, int NF, int W = KS>
struct Frag {
  static constexpr int NKK = W / 32;
  uint32_t off[KMAJ ? NKK : NF];
  // row0: first row of fragment 0 within the region (the wavefront tile's base)
  __device__ __forceinline__ void init(int row0, int lane) {
    if (KMAJ) {
      const int row = row0 + (lane & 15);
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk)
        off[kk] = (uint32_t)(row * 2 * W + ((((4 * kk + (lane >> 4)) ^ kswz<W>(row))) << 4));
    } else {
      const int k = 8 * (lane >> 4) + ((lane & 15) >> 2);
      const int g2 = 2 * mn_g<R>(k);
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const int mn0 = row0 + 16 * f;
        off[f] = (uint32_t)(k * 2 * R + (((((mn0 >> 3) ^ g2) + ((lane & 3) >> 1))) << 4) + 8 * (lane & 1));
      }
    }
  }
  __device__ __forceinline__ bf16x8_t read(const char* region, int f, int kk = 0) const {
    if (KMAJ) return *reinterpret_cast<const bf16x8_t*>(region + off[kk] + f * 16 * 2 * W);
    const bf16* p = reinterpret_cast<const bf16*>(region + off[f]) + kk * 32 * R;
    const i16x4_t lo = lds_read_tr(p), hi = lds_read_tr(p + 4 * R);
    const i16x4_t v8[2] = {lo, hi};
    return *reinterpret_cast<const bf16x8_t*>(v8);
  }
};

// s_waitcnt with vmcnt(v) and lgkmcnt(l) (gfx9 encoding; expcnt not waited)
#define FAL_WAITCNT(v, l) __builtin_amdgcn_s_waitcnt(((v) & 15) | (((v) >> 4) << 14) | (7 << 4) | ((l) << 8))
__device__ __forceinline__ void bar() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
}  // namespace pipe

}  // namespace fal
