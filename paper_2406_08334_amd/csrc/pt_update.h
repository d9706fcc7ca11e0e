// What every update on the GPU shares: the 16-bit formats, the nine constants and the fp32 operation sequence of one element.
#pragma once

#include "pt_common.h"

#include <hip/hip_fp16.h>

#pragma clang fp contract(off)

template <int DT>
__device__ __forceinline__ float decode16(uint32_t w16) {
  if (DT == PT_BF16) {
    return __uint_as_float(w16 << 16);
  } else {
    __half_raw r; r.x = (unsigned short)w16;
    return __half2float(__half(r));
  }
}

template <int DT>
__device__ __forceinline__ uint32_t encode16(float x) {
  if (DT == PT_BF16) {
    const uint32_t u = __float_as_uint(x);
    const uint32_t nan = (u >> 16) | 0x0040u;                          // NaN stays NaN
    const uint32_t rne = (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;       // round to nearest, ties to even
    return (u & 0x7fffffffu) > 0x7f800000u ? nan : rne;                // a select: a branch per element was compiled before
  } else {
    // The recast rounds the STORED fp32 master weight.  Without this barrier the compiler
    // folds the producing fma and the conversion into one mixed-precision fma that rounds
    // the exact result straight to fp16, which can differ from RNE16(RNE32(.)) by one ulp.
    asm volatile("" : "+v"(x));
    __half_raw r = __half_raw(__float2half_rn(x));
    return (uint32_t)r.x;
  }
}

typedef float pt_f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t pt_u32x2 __attribute__((ext_vector_type(2)));
// To the nearest 16-bit numbers, two an instruction.
template <int DT>
__device__ __forceinline__ pt_u32x2 encode16x4(pt_f32x4 x) {
  if constexpr (DT == PT_BF16) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(pt_u32x2, __builtin_convertvector(x, bf16x4));
  } else {
    return pt_u32x2{encode16<DT>(x[0]) | encode16<DT>(x[1]) << 16, encode16<DT>(x[2]) | encode16<DT>(x[3]) << 16};
  }
}

struct Consts { float b1, b2, omb1, omb2, decay, step_size, rsb2, eps, gm; };

// g: the gradient as stored; decay: the element's decay factor.  s: sqrt of the new variance.
__device__ __forceinline__ void update_element(const Consts& k, float decay, float g, float& w, float& m, float& v, float& s) {
  // one correctly rounded binary32 operation per line; contraction is off
  g = g * k.gm;
  float t1 = k.omb1 * g;
  float mn = __builtin_fmaf(k.b1, m, t1);
  float t2 = k.omb2 * g;
  t2 = t2 * g;
  float vn = __builtin_fmaf(k.b2, v, t2);
  s = __builtin_sqrtf(vn);
  float d = __builtin_fmaf(s, k.rsb2, k.eps);
  float u = mn / d;
  float t3 = w * decay;
  float wn = __builtin_fmaf(-k.step_size, u, t3);
  m = mn; v = vn; w = wn;
}
