// What the operators on rows share: eight or four 16-bit elements of a row at any address, e4m3 codes, sums over rows of partial sums.
#pragma once

#include "pt_tiles.h"

namespace pt_rows_ops {

using namespace pt_mfma;

// Eight elements of a row of d (m: below 2^31) from m on, zero behind its end, in two parts, so that no load waits for another: `fetch` loads the row's last
// eight where fewer than eight are left, and nothing that is not the row's; `place` then moves those to their places.
__device__ __forceinline__ u32x4 fetch8(const PT_GLOBAL uint16_t* row, uint32_t m, uint32_t d) {
  if (d >= 8) return *(const PT_GLOBAL u32x4_a*)((const PT_GLOBAL char*)row + min(m, d - 8) * 2);
  u32x4 q = {0, 0, 0, 0};
#pragma unroll 1
  for (uint32_t j = d; j > m; --j) q = u32x4{q.x << 16 | row[j - 1], q.y << 16 | q.x >> 16, q.z << 16 | q.y >> 16, q.w << 16 | q.z >> 16};
  return q;
}
__device__ __forceinline__ u32x4 place8(u32x4 q, uint32_t m, uint32_t d) {
  if (d >= 8 && m > d - 8) {
    const uint32_t k = m - (d - 8);                        // elements that are not its own
    uint64_t lo = uint64_t(q.y) << 32 | q.x, hi = uint64_t(q.w) << 32 | q.z;
    if (k >= 4) { lo = k < 8 ? hi >> (16 * (k - 4)) : 0; hi = 0; }
    else { lo = lo >> (16 * k) | hi << (64 - 16 * k); hi >>= 16 * k; }
    q = u32x4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
  }
  return q;
}
__device__ __forceinline__ u32x4 load8(const PT_GLOBAL uint16_t* row, uint32_t m, uint32_t d) { return place8(fetch8(row, m, d), m, d); }
// Four, the same.
__device__ __forceinline__ u32x2 fetch4(const PT_GLOBAL uint16_t* row, uint32_t m, uint32_t d) {
  if (d >= 4) return *(const PT_GLOBAL u32x2_a*)((const PT_GLOBAL char*)row + min(m, d - 4) * 2);
  u32x2 q = {0, 0};
#pragma unroll 1
  for (uint32_t j = d; j > m; --j) q = u32x2{q.x << 16 | row[j - 1], q.y << 16 | q.x >> 16};
  return q;
}
__device__ __forceinline__ u32x2 place4(u32x2 q, uint32_t m, uint32_t d) {
  if (d >= 4 && m > d - 4) {
    const uint32_t k = m - (d - 4);
    const uint64_t w = k < 4 ? (uint64_t(q.y) << 32 | q.x) >> (16 * k) : 0;
    q = u32x2{uint32_t(w), uint32_t(w >> 32)};
  }
  return q;
}
__device__ __forceinline__ u32x2 load4(const PT_GLOBAL uint16_t* row, uint32_t m, uint32_t d) { return place4(fetch4(row, m, d), m, d); }
template <int DT>
__device__ __forceinline__ f32x4 decode4(u32x2 q) {
  return f32x4{decode16<DT>(q.x & 0xffffu), decode16<DT>(q.x >> 16), decode16<DT>(q.y & 0xffffu), decode16<DT>(q.y >> 16)};
}
template <int DT>
__device__ __forceinline__ void decode8(u32x4 q, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = decode16<DT>(q[j] & 0xffffu);
    x[2 * j + 1] = decode16<DT>(q[j] >> 16);
  }
}
template <int DT>
__device__ __forceinline__ u32x4 encode8(const float (&x)[8]) {
  const u32x2 a = encode16x4<DT>(f32x4{x[0], x[1], x[2], x[3]}), b = encode16x4<DT>(f32x4{x[4], x[5], x[6], x[7]});
  return u32x4{a.x, a.y, b.x, b.y};
}

constexpr float TOP8 = 448.0f, LEAST8 = 0x1p-100f;
// A row's scale and what its elements are multiplied by, from the bits of the largest magnitude (any NaN's are more than inf's).
struct Scale8 { float scale, inv; };
__device__ __forceinline__ Scale8 scale8(uint32_t big) {
  if (big > 0x7f7fffffu) return {__builtin_nanf(""), __builtin_nanf("")};
  const float x = __uint_as_float(big);
  return x < LEAST8 ? Scale8{0.0f, 0.0f} : Scale8{x / TOP8, TOP8 / x};
}
// Eight codes, to the nearest: x inv is 448 at most but for its rounding, which stays below the next number.
__device__ __forceinline__ u32x2 codes8(const float (&x)[8], float inv) {
  u32x2 q;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h] * inv, x[4 * h + 1] * inv, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2] * inv, x[4 * h + 3] * inv, w, true);
    q[h] = uint32_t(w);
  }
  return q;
}
// Results that pass by once: stores of eight elements with a hint, so that they don't take the cache from what is read (RMS norm of 8192 x 4096 48.4 -> 46.0 us, rows8
// of 13824 x 5120 62.7 -> 59.3, RMS gradients 56.0 -> 54.6).  Hints on the loads cost what the cache still holds: norm of 2048 x 4096 11.4 -> 15.3.
__device__ __forceinline__ void pass8(PT_GLOBAL uint16_t* row, uint32_t m, uint32_t d, u32x4 w) {
  if (m + 8 <= d) __builtin_nontemporal_store(w, (PT_GLOBAL u32x4_a*)(row + m));
  else store8(row, m, d, w);
}
// Eight bytes of a row of d, at any address, from m on, the same.
typedef u32x2 u32x2_b __attribute__((aligned(1)));
typedef u32x4 u32x4_b __attribute__((aligned(1)));
__device__ __forceinline__ void pass8b(PT_GLOBAL uint8_t* row, uint32_t m, uint32_t d, u32x2 w) {
  if (m + 8 <= d) __builtin_nontemporal_store(w, (PT_GLOBAL u32x2_b*)(row + m));
  else
#pragma unroll
    for (uint32_t q = 0; q < 8; ++q)
      if (m + q < d) row[m + q] = uint8_t(w[q / 4] >> (8 * (q & 3)));
}

// Sums of the columns of `rows` rows of partial sums, in a fixed order, to 16 bits, by a workgroup of 256: 16 columns, and of the rows a sixteenth a lane.
// (64 columns a workgroup are few workgroups: 512 rows of 4096 in 6.2 us.)
constexpr uint32_t COLUMNS = 16;
template <int DT>
__device__ __forceinline__ void add_columns(const float* part, uint32_t rows, uint64_t pitch, uint32_t width, uint16_t* out, uint32_t block) {
  __shared__ float s_x[16][COLUMNS + 1];
  const uint32_t c = block * COLUMNS + threadIdx.x % COLUMNS, group = threadIdx.x / COLUMNS;
  float x = 0.0f;
  if (c < width) {
    const PT_GLOBAL float* p = (const PT_GLOBAL float*)part + c;
#pragma unroll 16
    for (uint32_t r = group; r < rows; r += 16) x += p[r * pitch];
  }
  s_x[group][threadIdx.x % COLUMNS] = x;
  __syncthreads();
  if (threadIdx.x >= COLUMNS || c >= width) return;
  x = s_x[0][threadIdx.x];
#pragma unroll
  for (int g = 1; g < 16; ++g) x += s_x[g][threadIdx.x];
  ((PT_GLOBAL uint16_t*)out)[c] = uint16_t(encode16<DT>(x));
}
inline uint32_t column_blocks(uint32_t width) { return (width + COLUMNS - 1) / COLUMNS; }

}  // namespace pt_rows_ops
