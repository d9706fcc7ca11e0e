// Tiles of a matrix product on the matrix cores: operands from memory through LDS into registers.
//
// C[m][n] = sum_k P[m][k] Q[n][k] in fp32 from 16-bit operands, each of which lies in memory with k or with its other index next to each other.  A
// workgroup takes BM x BN of C, its waves (WM x WN of them) a part each, in steps of 64 k.  A lane ends up with four values of consecutive m of one n.
//
// Memory to LDS goes without registers, 16 bytes a lane, lane behind lane; which 16 bytes a lane fetches is free, and is chosen so that what
// the lanes then read from LDS lies in different banks:
//   k next to each other:  row of 64 k = 8 pieces of 16 bytes, piece c at c ^ (row & 7); a lane reads a piece, eight k of its row
//   m next to each other:  row of B m = B / 8 pieces, piece c of row k at c ^ swizzle(k); the transposing LDS read hands a lane four k of its m
// What bounds it is how densely the matrix instructions of a wave follow each other, and the power they take: 256 x 256 tiles by eight waves, two to a SIMD,
// 8192 x 8192 x 4096: 1400 TFLOP/s in each of the three layouts that the head's products take (k next to each other in both operands, in one, in none).
#pragma once

#include "pt_common.h"

namespace pt_mfma {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int BK = 64, TWO = 2 * BK;
template <int DT>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (DT == PT_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// One operand of a product.  What lies behind its m (or n) and behind its last k is loaded as zero, or, of m and n, as what lies between its rows: the
// result is not used.  Where k lies next to each other it is a multiple of 64.
struct Operand {
  const void* at;
  uint64_t pitch;            // bytes from one row in memory to the next
  uint32_t extent;           // of m (or n)
  uint32_t k;
};

// KC: k lies next to each other.
template <bool KC, int B, int THREADS>
struct Stage {
  static constexpr int PER_ROW = KC ? BK / 8 : B / 8;                      // pieces of 16 bytes
  static constexpr int N = B * BK / 8 / THREADS;                           // pieces a lane fetches for a step
  static constexpr int BYTES = B * BK * 2;
  static_assert(N >= 1 && THREADS % PER_ROW == 0 && THREADS / PER_ROW % (KC ? 8 : 16) == 0, "a lane's pieces lie alike in their rows");
  uint64_t base, end, step;  // of the step to be fetched next; behind the operand's last element
  uint64_t stop;             // `base` behind the last step
  uint32_t off, rows;        // the lane's first piece, and from there to its next one
  uint32_t lane_at;          // where in a buffer the lane's first k of the first row of its wave lies

  static __device__ __forceinline__ uint32_t swizzle(uint32_t row) {
    if constexpr (KC) return row & 7;
    else return (((row & 3) | ((row >> 1) & 4)) * 2) & (PER_ROW - 1);
  }
  // wave: the first row of the lane's wave, a multiple of what the wave takes (a power of two).
  __device__ __forceinline__ void init(const Operand& o, uint32_t mn0, uint32_t k0, uint32_t wave) {
    const uint32_t g = (threadIdx.x >> 4) & 3, l = threadIdx.x & 15;
    if constexpr (KC) lane_at = (wave + l) * (BK * 2) + ((g ^ swizzle(l)) * 16);
    else {
      const uint32_t row = g * 8 + (l >> 2), c = (wave >> 3) + ((l & 3) >> 1);
      lane_at = row * (B * 2) + ((c ^ swizzle(row)) * 16) + (l & 1) * 8;
    }
    base = uint64_t(o.at) + (KC ? mn0 * o.pitch + uint64_t(k0) * 2 : k0 * o.pitch + uint64_t(mn0) * 2);
    end = uint64_t(o.at) + (KC ? (o.extent - 1) * o.pitch + uint64_t(o.k) * 2 : (o.k - 1) * o.pitch + uint64_t(o.extent) * 2);
    stop = KC ? base + uint64_t(o.k - min(k0, o.k)) * 2 : end;
    step = KC ? BK * 2 : BK * o.pitch;
    const uint32_t row = threadIdx.x / PER_ROW, c = (threadIdx.x % PER_ROW) ^ swizzle(row);
    off = row * uint32_t(o.pitch) + c * 16;
    rows = THREADS / PER_ROW * uint32_t(o.pitch);
  }
  // Fetches piece i of the lane's N of the step at `base` to `to`.  The hardware checks the range.
  __device__ __forceinline__ void fetch(lds_char* to, int i) const {
    const uint64_t left = base < stop ? end - base : 0;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, left > 0xffffffffull ? 0xffffffffu : uint32_t(left), 0x27000);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(to + (wave * 64 + i * THREADS) * 16), 16, off, i * rows, 0, 0);
  }
  __device__ __forceinline__ void advance() { base += step; }
  // The lane's eight k (32 kk + 8 (lane / 16) on) of row 16 i + lane % 16 of its wave's.
  __device__ __forceinline__ s16x8 read(const lds_char* from, int i, int kk) const {
    if constexpr (KC) {
      return *(const __attribute__((address_space(3))) s16x8*)(from + (lane_at ^ (kk * 64)) + i * (16 * BK * 2));
    } else {
      const lds_char* at = from + (lane_at ^ (i * 32)) + kk * (32 * B * 2);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 4 * B * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

// The product of a tile: `twos` times two steps of 64 k.
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
  SP sp;
  SQ sq;

  __device__ __forceinline__ void read(Frags& f, const lds_char* from, int kk, int r) const {
    if (r < FN) f.b[r] = sq.read(from + SP::BYTES, r, kk);
    else f.a[r - FN] = sp.read(from, r - FN, kk);
  }

  // Multiplies half a step, and in between reads another half (READ) and fetches a step (FETCH): a wave issues in order, so what waits for its
  // turn at the LDS would hold the products up if it were not spread over them.
  template <bool READ, bool FETCH>
  __device__ __forceinline__ void half(const Frags& now, Frags& then, const lds_char* from, int kk, lds_char* to) {
    constexpr int READS = FM + FN, FETCHES = SP::N + SQ::N, PRODUCTS = FM * FN, PER = 3;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < PRODUCTS; ++x) {
      acc[x / FN][x % FN] = mfma<DT>(now.a[x / FN], now.b[x % FN], acc[x / FN][x % FN]);
      if (x % PER == PER - 1 || x + 1 == PRODUCTS) {
        __builtin_amdgcn_sched_barrier(0);
        const int slot = x / PER, slots = (PRODUCTS + PER - 1) / PER;
        const int f0 = slot, f1 = x + 1 == PRODUCTS ? (FETCHES > slots ? FETCHES : slots) : slot + 1;
        if (FETCH)
#pragma unroll
          for (int i = f0; i < f1 && i < FETCHES; ++i) { if (i < SP::N) sp.fetch(to, i); else sq.fetch(to + SP::BYTES, i - SP::N); }
        const int r1 = x + 1 == PRODUCTS ? READS : slot + 1;
        if (READ)
#pragma unroll
          for (int r = slot; r < r1 && r < READS; ++r) read(then, from, kk, r);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  static __device__ __forceinline__ void meet() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  // A step whose first half is in f0; the step after the next is fetched.
  __device__ __forceinline__ void step(Frags& f0, Frags& f1, lds_char* now, lds_char* then) {
    half<true, false>(f0, f1, now, 1, nullptr);
    meet();
    half<true, true>(f1, f0, then, 0, now);
    sp.advance();
    sq.advance();
  }
  __device__ __forceinline__ void fetch(lds_char* to) {
#pragma unroll
    for (int i = 0; i < SP::N; ++i) sp.fetch(to, i);
#pragma unroll
    for (int i = 0; i < SQ::N; ++i) sq.fetch(to + SP::BYTES, i);
    sp.advance();
    sq.advance();
  }

  // Two steps' operands are in LDS, half a step's in registers: what a half needs is read from LDS while the half before is multiplied, and a
  // step is fetched while the one before it is multiplied.  The workgroup meets in the middle of a step, when every wave has read the last of
  // one buffer: that one is fetched into then, and the other one has arrived.
  // Steps are taken in twos, and the last two fetch two more that nothing needs: one loop without exceptions, whose sums stay in their
  // registers.  even, odd: the buffers of even and odd steps, BYTES each, two arrays: a transposing read waits for all fetches that the compiler
  // cannot tell from what it reads.
  __device__ __forceinline__ void run(lds_char* even, lds_char* odd, const Operand& p, const Operand& q, uint32_t m0, uint32_t n0, uint32_t k0,
                                      uint32_t twos) {
    clear();
    add(even, odd, p, q, m0, n0, k0, twos);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // To the sums so far.  Between two of them the workgroup has to meet.
  __device__ __forceinline__ void add(lds_char* even, lds_char* odd, const Operand& p, const Operand& q, uint32_t m0, uint32_t n0, uint32_t k0,
                                      uint32_t twos) {
    if (!twos) return;
    sp.init(p, m0, k0, wave_m());
    sq.init(q, n0, k0, wave_n());
    fetch(even);
    fetch(odd);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(SP::N + SQ::N) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    Frags f0, f1;
#pragma unroll
    for (int r = 0; r < FM + FN; ++r) read(f0, even, 0, r);
#pragma unroll 1
    for (; twos; --twos) {
      step(f0, f1, even, odd);
      step(f0, f1, odd, even);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  }
};

// Of four values of consecutive m a lane has of fragment i (two words of 16-bit numbers, a) and of fragment i + 1 (b): eight of one of the two.
// Lanes 0-15 and 32-47 keep i and get its next four from the 16 lanes behind them, those give it for i + 1.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 eight(u32x2 a, u32x2 b) {
  const u32x2 x = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false), y = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
  return u32x4{x[0], y[0], x[1], y[1]};
}
// Where those eight begin, from the first m of fragment i on.
__device__ __forceinline__ uint32_t eight_at() { const uint32_t g = (threadIdx.x >> 4) & 3; return (g & 1) * 16 + (g >> 1) * 8; }

}  // namespace pt_mfma
