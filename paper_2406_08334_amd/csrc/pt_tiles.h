// How the tiles of a matrix product are laid over the chip, shared between workgroups, joined and stored.
#pragma once

#include "pt_mfma.h"
#include "pt_update.h"

#include <algorithm>

namespace pt_mfma {

typedef u32x4 u32x4_a __attribute__((aligned(2)));
typedef u32x2 u32x2_a __attribute__((aligned(2)));

inline uint64_t up(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }

// One row of 16-bit words, at any address, into one of Kd words that begins at a multiple of 16 bytes; zero behind its end.  FINITE: and where all bits of `exponent`
// are set, infinities and NaN.
template <bool FINITE = false>
__device__ __forceinline__ void copy_row(const PT_GLOBAL uint16_t* from, PT_GLOBAL uint16_t* to, uint32_t d, uint32_t Kd, uint32_t lane, uint32_t lanes,
                                         uint32_t exponent = 0) {
#pragma unroll 4
  for (uint32_t c = lane * 8; c < Kd; c += lanes * 8) {
    u32x4 q = {0, 0, 0, 0};
    if (c + 8 <= d) q = *(const PT_GLOBAL u32x4_a*)(from + c);
    else
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j)
        if (c + j < d) q[j / 2] |= uint32_t(from[c + j]) << (16 * (j & 1));
    if constexpr (FINITE) {
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] &= ((q[j] & exponent) == exponent ? 0u : 0xffffu) | ((q[j] >> 16 & exponent) == exponent ? 0u : 0xffff0000u);
    }
    *(PT_GLOBAL u32x4*)(to + c) = q;
  }
}

// Tiles of the products and how their waves lie in them.  `SLOTS` of them run at a time, TWO_NS is what two steps of them take then (measured), and
// PART_NS what a tile of partial sums costs that is written and read once more.
//   Big   the fewest reads of LDS a product: 1440 TFLOP/s while all 256 run.  4096 x 1600 x 32000: 1.24 ms; in Mid alone 1.57
//   Mid   where that few tiles of Big would leave the chip idle.  300 x 1024 x 2000: 55 us; in Big alone 78.  8192 x 512 x 1000: 95; 121
//   Few   up to FEW_ROWS rows, which take as long as the weight takes to read.  64 x 1600 x 50257: 137 us; in Mid alone 156; 64 x 4096 x 32000, the loss: 53; 67
// Which is taken is a matter of what each would need by these figures (mid_tiles, mid_hidden, weight_tiles).
template <int BM_, int BN_, int WM_, int WN_, int SLOTS_, int TWO_NS_> struct Cfg {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, THREADS = 64 * WM_ * WN_, SLOTS = SLOTS_, TWO_NS = TWO_NS_, PART_NS = BM_ * BN_ / 625;
  template <int DT, bool PK, bool QK> using Of = Tile<DT, PK, QK, BM_, BN_, WM_, WN_>;
};
typedef Cfg<256, 256, 2, 4, 256, 2970> Big;
typedef Cfg<128, 128, 2, 2, 512, 1910> Mid;
typedef Cfg<128, 64, 4, 1, 256, 1700> Few;

// How the tiles of a gradient are done: `whole` by one workgroup each, and `tail`, those of the last round, by `n` each, which share its k and leave sums to
// be added; and when they are done, in ns.  (512 x 4096 x 32000: 690 us without, 450 with; 1000 x 768 x 5000: 112, 76.)
struct Split { uint32_t whole, tail, n; uint64_t ns; };
// over: ns of a tile beside its products.
template <class C> __host__ __device__ inline Split split(uint32_t tiles, uint32_t twos, uint32_t over = 3000) {
  const uint64_t round = uint64_t(twos) * C::TWO_NS + over;
  Split best = {tiles, 0, 1, (tiles + C::SLOTS - 1) / C::SLOTS * round};
  const uint32_t tail = tiles % C::SLOTS, whole = tiles - tail;
  if (!tail) return best;
  for (uint32_t n : {2u, 3u, 4u, 6u, 8u, 12u, 16u, 24u, 32u, std::min(32u, uint32_t(C::SLOTS) / tail)}) {
    if (n < 2 || n * 2 > twos) continue;
    const uint64_t ns = whole / C::SLOTS * round + (tail * n + C::SLOTS - 1) / C::SLOTS * (uint64_t((twos + n - 1) / n) * C::TWO_NS + over) +
                        uint64_t(tail) * n * C::PART_NS + 4000;
    if (ns < best.ns) best = {whole, tail, n, ns};
  }
  return best;
}

// Tile i of tm x tn: the 32 of an XCD that run at a time make patches of about 4 n x 8 m, which share what they read.  (Patches of 8 n: 8192 (6144) x 4096 x
// 32000 3870 us instead of 3800, 4096 x 4096 x 32000 835, 827; 16 n: 3940, 855; 2 n: 3850, 832.)
__device__ __forceinline__ void tile_at(uint32_t i, uint32_t tm, uint32_t tn, uint32_t& m, uint32_t& n) {
  constexpr uint32_t PATCH = 4;
  const uint32_t g = i / (PATCH * tm), n0 = g * PATCH, gn = min(PATCH, tn - n0), r = i - g * PATCH * tm;
  n = n0 + r % gn;
  m = r / gn;
}
// The XCDs, which workgroups go to in turn, get numbers next to each other: of `total` that of workgroup `id`, if there is one.  (Numbers as they come:
// 16384 x 5120 x 32000 14.25 ms instead of 13.8, 1531 x 771 x 50257 685 us, 648.)
__device__ __forceinline__ bool xcd_of(uint32_t id, uint32_t total, uint32_t& i) {
  const uint32_t per = (total + 7) / 8;
  i = (id & 7) * per + (id >> 3);
  return (id >> 3) < per && i < total;
}
__device__ __forceinline__ bool tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t& m, uint32_t& n) {
  uint32_t i;
  if (!xcd_of(id, tm * tn, i)) return false;
  tile_at(i, tm, tn, m, n);
  return true;
}
// Tile and part of a workgroup of a split product; sums: where its sums go, or NULL: they are all there is.
__host__ __device__ inline uint32_t split_grid(const Split& s) { return (s.whole + 7) / 8 * 8 + (s.tail * s.n + 7) / 8 * 8; }
template <class C>
__device__ __forceinline__ bool part_of(const Split& s, uint32_t id, uint32_t tm, uint32_t tn, float* room, uint32_t& m, uint32_t& n, uint32_t& part,
                                        PT_GLOBAL float*& sums) {
  uint32_t i;
  const uint32_t first = (s.whole + 7) / 8 * 8;
  part = 0;
  sums = nullptr;
  if (id < first) {
    if (!xcd_of(id, s.whole, i)) return false;
  } else {
    if (!xcd_of(id - first, s.tail * s.n, i)) return false;
    sums = (PT_GLOBAL float*)room + size_t(i) * (C::BM * C::BN);
    part = i / s.tail;
    i = s.whole + i % s.tail;
  }
  tile_at(i, tm, tn, m, n);
  return true;
}
inline uint32_t tile_grid(uint64_t tm, uint64_t tn) { return uint32_t((tm * tn + 7) / 8 * 8); }

// Tiles of the gradients at the end of the width: of Big's, 256 wide, what is left of the width is often a small part (width 1600: 64 of it), and takes a
// narrower tile (4096 x 1600 x 32000: 1258 us without, 1238 with).  f: called with the tile.
template <int DT, class C, bool PK, bool QK, class F>
__device__ __forceinline__ void with_tile(uint32_t left, F&& f) {
  if constexpr (C::BM == 256) {
    if (left <= 64) return f(Tile<DT, PK, QK, 64, C::BN, 1, 8>{});
    if (left <= 128) return f(Tile<DT, PK, QK, 128, C::BN, 2, 4>{});
  }
  f(typename C::template Of<DT, PK, QK>{});
}

// A lane's sums of rows j of a tile, into the tile's place among those of several workgroups.
template <class C, class T>
__device__ __forceinline__ void leave(const T& t, int j, PT_GLOBAL float* sums) {
  const uint32_t lane = threadIdx.x & 63;
  PT_GLOBAL float* row = sums + (t.wave_n() + j * 16 + (lane & 15)) * C::BM + t.wave_m() + (lane >> 4) * 4;
#pragma unroll
  for (int i = 0; i < T::FM; ++i) *(PT_GLOBAL f32x4*)(row + i * 16) = t.acc[i][j];
}

// Adds up what several workgroups a tile have left, four results of a row at a time, by JOINERS workgroups at most: that many at once, and few if the rows
// turn out to need none.  f: called with place (m, n) and sum.
constexpr uint32_t JOINERS = 2048;
template <class C> inline uint32_t joiners(uint32_t tail) { return std::min<uint32_t>(JOINERS, tail * (C::BM * C::BN / 1024)); }
template <class C, class F>
__device__ __forceinline__ void join_tiles(const float* room, const Split& s, uint32_t tm, uint32_t tn, F&& f, uint32_t block = blockIdx.x,
                                           uint32_t blocks = gridDim.x) {
  constexpr uint32_t TILE = C::BM * C::BN;
  const size_t next = size_t(s.tail) * TILE;
  for (uint32_t i = block; i < s.tail * (TILE / 1024); i += blocks) {
    const uint32_t j = i / (TILE / 1024), e = i % (TILE / 1024) * 1024 + threadIdx.x * 4;
    uint32_t m, n;
    tile_at(s.whole + j, tm, tn, m, n);
    const PT_GLOBAL float* sums = (const PT_GLOBAL float*)room + size_t(j) * TILE + e;
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (uint32_t k = 0; k < s.n; ++k) x += *(const PT_GLOBAL f32x4*)(sums + k * next);
    f(m * C::BM + e % C::BM, n * C::BN + e / C::BM, x);
  }
}

// Of a row of d 16-bit numbers, at any address, the eight from m on.
__device__ __forceinline__ void store8(PT_GLOBAL uint16_t* row, uint32_t m, uint32_t d, u32x4 w) {
  if (m + 8 <= d) *(PT_GLOBAL u32x4_a*)(row + m) = w;
  else
#pragma unroll
    for (uint32_t q = 0; q < 8; ++q)
      if (m + q < d) row[m + q] = uint16_t(w[q / 2] >> (16 * (q & 1)));
}

__device__ __forceinline__ void store4(PT_GLOBAL uint16_t* row, uint32_t m, uint32_t d, u32x2 w) {
  if (m + 4 <= d) *(PT_GLOBAL u32x2_a*)(row + m) = w;
  else
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q)
      if (m + q < d) row[m + q] = uint16_t(w[q / 2] >> (16 * (q & 1)));
}

}  // namespace pt_mfma
