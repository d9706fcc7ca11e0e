// Tiles of a matrix product on the matrix cores: operands from memory through LDS into registers.
//
// C[m][n] = sum_k P[m][k] Q[n][k] in fp32 from 16-bit operands, each of which lies in memory with k or with its other index next to each other.  A
// workgroup takes BM x BN of C, its waves (WM x WN of them) a part each, in steps of 64 k.  A lane ends up with four values of consecutive m of one n.
//
// Memory to LDS goes without registers, 16 bytes a lane, lane behind lane; which 16 bytes a lane fetches is free, and is chosen so that what
// the lanes then read from LDS lies in different banks:
//   k next to each other:  row of 64 k = 8 pieces of 16 bytes, piece c at c ^ (row & 7); a lane reads a piece, eight k of its row
//   m next to each other:  row of B m = B / 8 pieces, piece c of row k at c ^ swizzle(k); the transposing LDS read hands a lane four k of its m
#pragma once

#include "pt_common.h"

namespace pt_mfma {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int BK = 64;
#ifdef NOPRIO
#define PRIO(x)
#else
#define PRIO(x) __builtin_amdgcn_s_setprio(x)
#endif


template <int DT>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (DT == PT_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// One operand of a product.
struct Operand {
  const void* at;
  uint64_t pitch;            // bytes from one row in memory to the next
  uint32_t extent;           // of m (or n); what lies behind is loaded from inside and its results are not used
  uint32_t k;                // k that may be read; the other operand is zero behind it, up to a multiple of 64
};

// KC: k lies next to each other.
template <bool KC, int B, int THREADS>
struct Stage {
  static constexpr int PER_ROW = KC ? BK / 8 : B / 8;                      // pieces of 16 bytes
  static constexpr int N = B * BK / 8 / THREADS;                           // pieces a lane fetches for a step
  static constexpr int BYTES = B * BK * 2;
  static_assert(N >= 1, "more lanes than pieces");
  uint64_t base;
  uint64_t step;
  uint32_t off[N];
  uint32_t pitch, k;

  static __device__ __forceinline__ uint32_t swizzle(uint32_t row) {
    if constexpr (KC) return row & 7;
    else return (((row & 3) | ((row >> 1) & 4)) * 2) & (PER_ROW - 1);
  }
  __device__ __forceinline__ void init(const Operand& o, uint32_t mn0, uint32_t k0) {
    pitch = uint32_t(o.pitch);
    k = o.k;
    base = uint64_t(o.at) + (KC ? mn0 * o.pitch + uint64_t(k0) * 2 : k0 * o.pitch + uint64_t(mn0) * 2);
    step = KC ? BK * 2 : BK * o.pitch;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t s = threadIdx.x + i * THREADS, row = s / PER_ROW;
      uint32_t c = (s % PER_ROW) ^ swizzle(row);
      if constexpr (KC) off[i] = min(row, o.extent - 1 - mn0) * pitch + c * 16;
      else {
        if (mn0 + c * 8 >= o.extent) c = 0;
        off[i] = row * pitch + c * 16;
      }
    }
  }
  // Fetches step k0 to `to`.
  __device__ __forceinline__ void fetch(lds_char* to, uint32_t k0) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0xffffffffu, 0x27000);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (k0 + BK <= k) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(to + (wave * 64 + i * THREADS) * 16), 16, off[i], 0, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t s = threadIdx.x + i * THREADS, row = s / PER_ROW, c = (s % PER_ROW) ^ swizzle(row);
        uint32_t o = off[i];
        if constexpr (KC) { if (k0 + c * 8 >= k) o -= c * 16; }
        else { if (k0 + row >= k) o -= (k0 + row - (k - 1)) * pitch; }
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(to + (wave * 64 + i * THREADS) * 16), 16, o, 0, 0, 0);
      }
    }
    base += step;
  }
  // The lane's eight k (32 kk + 8 (lane / 16) on) of row mn + lane % 16.
  static __device__ __forceinline__ s16x8 read(const lds_char* from, uint32_t mn, int kk) {
    const uint32_t lane = threadIdx.x & 63, g = lane >> 4, i = lane & 15;
    if constexpr (KC) {
      const uint32_t row = mn + i;
      return *(const __attribute__((address_space(3))) s16x8*)(from + row * (BK * 2) + (((kk * 4 + g) ^ swizzle(row)) * 16));
    } else {
      s16x4 h[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const uint32_t row = kk * 32 + g * 8 + q * 4 + (i >> 2), c = (mn >> 3) + ((i & 3) >> 1);
        h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(from + row * (B * 2) + ((c ^ swizzle(row)) * 16) + (i & 1) * 8));
      }
      return __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

// The product of a tile: `steps` steps of 64 k.  lds: 2 * BYTES of it.
template <int DT, bool PK, bool QK, int BM, int BN, int WM, int WN>
struct Tile {
  static constexpr int THREADS = 64 * WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
  typedef Stage<PK, BM, THREADS> SP;
  typedef Stage<QK, BN, THREADS> SQ;
  static constexpr int BYTES = SP::BYTES + SQ::BYTES;
  f32x4 acc[FM][FN];

  __device__ __forceinline__ uint32_t wave_m() const { return (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WM) * TM; }
  __device__ __forceinline__ uint32_t wave_n() const { return (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WM) * TN; }

  struct Frags { s16x8 a[FM], b[FN]; };
  __device__ __forceinline__ void read(Frags& f, const lds_char* from, uint32_t wm, uint32_t wn, int kk) const {
#pragma unroll
    for (int i = 0; i < FM; ++i) f.a[i] = SP::read(from, wm + i * 16, kk);
#pragma unroll
    for (int j = 0; j < FN; ++j) f.b[j] = SQ::read(from + SP::BYTES, wn + j * 16, kk);
  }
  __device__ __forceinline__ void multiply(const Frags& f) {
    __builtin_amdgcn_sched_barrier(0);
    PRIO(1);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mfma<DT>(f.a[i], f.b[j], acc[i][j]);
    PRIO(0);
    __builtin_amdgcn_sched_barrier(0);
  }

  // Two steps' operands are in LDS, half a step's in registers: what a half needs is read from LDS while the half before is multiplied, and a
  // step is fetched while the one before it is multiplied.  The workgroup meets in the middle of a step, when every wave has read the last of
  // one buffer: that one is fetched into then, and the other one has arrived.
  __device__ __forceinline__ void run(lds_char* lds, const Operand& p, const Operand& q, uint32_t m0, uint32_t n0, uint32_t k0, uint32_t steps) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (!steps) return;
    SP sp;
    SQ sq;
    sp.init(p, m0, k0);
    sq.init(q, n0, k0);
    const uint32_t wm = wave_m(), wn = wave_n();
    sp.fetch(lds, k0);
    sq.fetch(lds + SP::BYTES, k0);
    if (steps > 1) {
      sp.fetch(lds + BYTES, k0 + BK);
      sq.fetch(lds + BYTES + SP::BYTES, k0 + BK);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(SP::N + SQ::N) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    Frags f0, f1;
    read(f0, lds, wm, wn, 0);
    for (uint32_t s = 0; s < steps; ++s) {
      lds_char* here = lds + (s & 1) * BYTES;
      lds_char* there = lds + ((s + 1) & 1) * BYTES;
      read(f1, here, wm, wn, 1);
      multiply(f0);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (s + 2 < steps) {
        sp.fetch(here, k0 + (s + 2) * BK);
        sq.fetch(here + SP::BYTES, k0 + (s + 2) * BK);
      }
      if (s + 1 < steps) read(f0, there, wm, wn, 0);
      multiply(f1);
    }
  }
};

}  // namespace pt_mfma
