// Matrix product with bias, activation, gate, dropout and residual in its epilogue, and its gradients.
//
//   out       z = x W^T + bias, out = residual + D(act(z) gate), z in 16 bits if it is to be kept: one product, the rest on its sums in registers
//   slope     dz = D(d_out gate act'(pre)) in 16 bits, d_gate, and sums of dz's columns for the bias; copies of operands that the products cannot take
//   d_x       = dz W,  d_weight = dz^T x
//
// Up to 32 rows out is a matter of reading the weight (k_linear_thin); beyond, and for the gradients, tiles of pt_mfma.h.
// Products bound the large ones: 8192 x 4096 x 8192 bf16 410 us, 1340 TFLOP/s, where a large library product reaches 1473 at best and 1410 here; 8192 x 1600 x 6400 with
// bias, gelu and z kept 191 (a round of tiles 39 of products, 17 of epilogue, which nothing else of its compute unit hides); e4m3 8192 x 4096 x 11008 344 us,
// 2150 TFLOP/s (library, without scales of rows: 324).  Gradients of 8192 x 4096 x 11008 1247 us: 511 + 537 at 1440 and 1380 TFLOP/s, slope 167 at 5.4 TB/s.
#include "pt_random.h"
#include "pt_rows.h"

using namespace pt_rows_ops;

namespace {

// ---- activations ------------------------------------------------------------------------------------------

constexpr int ANY = -1;      // of activations: whichever the call says
constexpr float LOG2E = 1.44269504088896340736f, TANH_2A = 1.59576912160573071176f, TANH_B = 0.044715f;       // 2 sqrt(2 / pi)

__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -LOG2E)); }

// The normal distribution's function, and exp(-z^2 / 2).  Of |z| sqrt(1/2) = u, with t = 1 / (1 + 7/16 u): erfc(u) / 2 = t P(t) exp(-u^2), P of degree seven
// fitted to erfcx over u up to 14 (relative error 1.7e-7); in fp32 2^-19 of the result up to |z| = 5, 2^-18 up to 9.
__device__ __forceinline__ float normal(float z, float& e) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(z), 0.30935921676911455f, 1.0f));
  float p = 0.03591368817931173f;
  for (float c : {-0.14291292135087455f, 0.15869404565010323f, -0.017569269200825362f, 0.11137608263966191f, 0.10724730147205802f, 0.12385262848412495f,
                  0.1233984909969888f})
    p = __builtin_fmaf(p, t, c);
  e = __builtin_amdgcn_exp2f((z * z) * (-0.5f * LOG2E));
  const float q = p * t * e;
  return z < 0.0f ? q : 1.0f - q;
}

template <int ACT>
__device__ __forceinline__ float act(float z) {
  if constexpr (ACT == PT_ACT_RELU) return z < 0.0f ? 0.0f : z;
  else if constexpr (ACT == PT_ACT_SILU) return z * sigmoid(z);
  else if constexpr (ACT == PT_ACT_GELU_TANH) return z * sigmoid(TANH_2A * __builtin_fmaf(TANH_B * z, z * z, z));     // (1 + tanh(u)) / 2 = sigmoid(2 u)
  else if constexpr (ACT == PT_ACT_GELU) { float e; return z * normal(z, e); }
  else return z;
}
// z f, where f is 0 below -FAR: at -inf, which z beyond the type is kept as, the limit, 0; NaN comes from f.  (Not for out, where only a sum that is infinite itself is
// -inf, and its product with 0 NaN: 8192 x 1600 x 6400 with gelu 204.5 -> 207.7 us, 8192 x 4096 x 11008 with silu 578 -> 584.)
constexpr float FAR = 128.0f;
__device__ __forceinline__ float times(float z, float f) { return __builtin_fmaxf(z, -FAR) * f; }
// act(z) and its derivative, which beyond FAR is 0 or 1 in fp32 (its terms there would be products of 0 and inf), as are the factors of z.
template <int ACT>
__device__ __forceinline__ float act(float z, float& slope) {
  const float c = z < -FAR ? -FAR : z > FAR ? FAR : z;
  if constexpr (ACT == PT_ACT_RELU) {
    slope = z > 0.0f ? 1.0f : 0.0f;
    return act<ACT>(z);
  } else if constexpr (ACT == PT_ACT_SILU) {
    const float f = sigmoid(z);
    slope = f * __builtin_fmaf(c, 1.0f - f, 1.0f);
    return times(z, f);
  } else if constexpr (ACT == PT_ACT_GELU_TANH) {
    const float f = sigmoid(TANH_2A * __builtin_fmaf(TANH_B * c, c * c, c));
    slope = __builtin_fmaf(c * f * (1.0f - f), TANH_2A * __builtin_fmaf(3.0f * TANH_B * c, c, 1.0f), f);
    return times(z, f);
  } else if constexpr (ACT == PT_ACT_GELU) {
    float e;
    const float f = normal(c, e);
    slope = __builtin_fmaf(c * 0.39894228040143267794f, e, f);
    return times(z, f);
  }
  slope = 1.0f;
  return z;
}

// f: called with the activation as a constant.
template <class F> __host__ __device__ __forceinline__ auto with_act(int a, F&& f) {
  switch (a) {
    case PT_ACT_RELU: return f(std::integral_constant<int, PT_ACT_RELU>{});
    case PT_ACT_GELU: return f(std::integral_constant<int, PT_ACT_GELU>{});
    case PT_ACT_GELU_TANH: return f(std::integral_constant<int, PT_ACT_GELU_TANH>{});
    case PT_ACT_SILU: return f(std::integral_constant<int, PT_ACT_SILU>{});
    default: return f(std::integral_constant<int, PT_ACT_NONE>{});
  }
}

// ---- epilogues ---------------------------------------------------------------------------------------------

// Results in 16 bits as they are.  m: of the row's elements, n: rows.
struct Plain {
  uint16_t* out;
  uint64_t stride;
  uint32_t extent_m, extent_n;

  template <int DT, int ACT, class C, class T>
  __device__ __forceinline__ void tile(const T& t, uint32_t m0, uint32_t n0, lds_char*, lds_char*) const {
    const uint32_t lane = threadIdx.x & 63, mw = m0 + t.wave_m();
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const uint32_t n = n0 + t.wave_n() + j * 16 + (lane & 15);
      const bool live = n < extent_n;
      PT_GLOBAL uint16_t* row = (PT_GLOBAL uint16_t*)out + (live ? n : 0) * stride;
#pragma unroll
      for (int i = 0; i < T::FM; i += 2) {
        const u32x4 x = eight(encode16x4<DT>(t.acc[i][j]), encode16x4<DT>(t.acc[i + 1][j]));       // lanes without a row take part in the exchange
        if (live) store8(row, mw + i * 16 + eight_at(), extent_m, x);
      }
    }
  }
  template <int DT>
  __device__ __forceinline__ void four(uint32_t m, uint32_t n, f32x4 x) const {
    if (n < extent_n && m < extent_m) store4((PT_GLOBAL uint16_t*)out + n * stride, m, extent_m, encode16x4<DT>(x));
  }
};

// m: outs, n: rows.
struct Layer {
  const uint16_t *bias, *gate, *residual;
  uint16_t *pre, *out;
  const float *x_scale, *weight_scale;
  uint64_t gate_stride, residual_stride, pre_stride, out_stride;
  uint32_t extent_m, extent_n;
  int act;
  pt_random::Drop drop;
  uint64_t words;            // of random numbers in a row
  bool direct;               // whole tiles on their sums where they are

  // z of N outs of row n from their sums: scales in 8 bits and bias, of the outs m on.
  template <int DT, int N> struct Columns {
    float scale[N], bias[N];
    __device__ __forceinline__ void load(const Layer& e, uint32_t m) {
#pragma unroll
      for (int q = 0; q < N; ++q) {
        scale[q] = e.weight_scale ? ((const PT_GLOBAL float*)e.weight_scale)[min(m + q, e.extent_m - 1)] : 1.0f;
        bias[q] = 0.0f;
      }
      if (!e.bias || m >= e.extent_m) return;
#pragma unroll
      for (int q = 0; q < N; q += 4) {
        const f32x4 b = decode4<DT>(load4((const PT_GLOBAL uint16_t*)e.bias, m + q, e.extent_m));
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[q + i] = b[i];
      }
    }
    __device__ __forceinline__ void z(const Layer& e, float x_scale, float (&x)[N]) const {
      if (e.x_scale) {
#pragma unroll
        for (int q = 0; q < N; ++q) x[q] = x[q] * x_scale * scale[q];
      }
      if (e.bias) {
#pragma unroll
        for (int q = 0; q < N; ++q) x[q] += bias[q];
      }
    }
  };
  __device__ __forceinline__ uint64_t counter(uint32_t m, uint32_t n) const { return drop.key() + (n * words + m / 4 + 1) * pt_random::PHI; }
  // From there to the result; g, r: gate and residual; counter: of the first four's random numbers.
  template <int ACT, int N>
  __device__ __forceinline__ void result(float (&y)[N], uint64_t counter, const float (&g)[N], const float (&r)[N]) const {
    const auto each = [&](auto a) {
#pragma unroll
      for (int q = 0; q < N; ++q) y[q] = ::act<a()>(y[q]);
    };
    if constexpr (ACT == ANY) with_act(act, each);
    else each(std::integral_constant<int, ACT>{});
    if (gate) {
#pragma unroll
      for (int q = 0; q < N; ++q) y[q] *= g[q];
    }
    if (drop.off) {
#pragma unroll
      for (int q = 0; q < N; q += 4) drop.apply(counter + q / 4 * pt_random::PHI, y + q);
    }
    if (residual) {
#pragma unroll
      for (int q = 0; q < N; ++q) y[q] += r[q];
    }
  }

  // A tile all of which there is, on its sums where they are: four of consecutive outs of a row and of the 16 outs behind, exchanged for eight as arrays are read and
  // written.  For one activation: five of 64 sums each do not fit the instruction cache.  (Through LDS, as at the edges: 8192 x 1600 x 6144 167.7 us instead of
  // 149.4, of which the products 127; 8192 x 4096 x 8192 434, 410; but with a gate, which is read in
  // pieces of lines then, 8192 x 4096 x 11008 671, 690; rows at odd addresses 8192 x 1600 x 6401 174, 188, with a residual 8192 x 768 x 3083 68, 83.)
  template <int DT, int ACT, class T>
  __device__ __forceinline__ void whole(const T& t, uint32_t m0, uint32_t n0) const {
    constexpr int PAIRS = T::FM / 2, PARTS = PAIRS * T::FN;
    typedef f32x4 f32x4_a __attribute__((aligned(4)));
    const uint32_t lane = threadIdx.x & 63, mw = m0 + t.wave_m(), mb = mw + (lane >> 4) * 4, n = n0 + t.wave_n() + (lane & 15), m8 = mw + eight_at();
    const uint64_t from = drop.off ? counter(mb, n) : 0, row_step = words * pt_random::PHI;
    u32x4 qr = {0, 0, 0, 0};
    const auto at = [&](const uint16_t* x, uint64_t stride, int part) { return (PT_GLOBAL u32x4_a*)((PT_GLOBAL uint16_t*)x + (n + part / PAIRS * 16) * stride + m8 + part % PAIRS * 32); };
    const auto fetch = [&](int part) {
      if (residual) qr = *at(residual, residual_stride, part);
    };
    fetch(0);
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
      const int i = part % PAIRS * 2, j = part / PAIRS;
      const u32x4 now_r = qr;
      if (part + 1 < PARTS) fetch(part + 1);
      f32x4 x[2] = {t.acc[i][j], t.acc[i + 1][j]};
      if (x_scale) {
        const float s = ((const PT_GLOBAL float*)x_scale)[n + j * 16];
#pragma unroll
        for (int h = 0; h < 2; ++h) x[h] = x[h] * s * *(const PT_GLOBAL f32x4_a*)((const PT_GLOBAL float*)weight_scale + mb + (i + h) * 16);
      }
      if (bias) {
#pragma unroll
        for (int h = 0; h < 2; ++h) x[h] += decode4<DT>(*(const PT_GLOBAL u32x2_a*)((const PT_GLOBAL uint16_t*)bias + mb + (i + h) * 16));
      }
      if (pre) *at(pre, pre_stride, part) = eight(encode16x4<DT>(x[0]), encode16x4<DT>(x[1]));
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 4; ++q) x[h][q] = ::act<ACT>(x[h][q]);
      if (drop.off) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint64_t z = pt_random::mix64(from + j * 16 * row_step + (i + h) * 4 * pt_random::PHI);
#pragma unroll
          for (int q = 0; q < 4; ++q) x[h][q] = drop.of(z, q, x[h][q]);
        }
      }
      if (residual) {                                      // the exchange is its own inverse
        const u32x4 y = eight(u32x2{now_r.x, now_r.y}, u32x2{now_r.z, now_r.w});
        x[0] += decode4<DT>(u32x2{y.x, y.y});
        x[1] += decode4<DT>(u32x2{y.z, y.w});
      }
      *at(out, out_stride, part) = eight(encode16x4<DT>(x[0]), encode16x4<DT>(x[1]));
      __builtin_amdgcn_sched_barrier(0);                   // there are no registers for more than that at a time
    }
  }

  // A wave's sums go through LDS, 16 rows at a time, so that a lane has eight outs of a row, the lanes of a row all that the wave has of it, and what is loaded
  // and stored is whole lines; in a loop, as four times five activations of 128 sums a lane would not fit the instruction cache.  What is loaded for a
  // turn is under way during the one before.  The wave's own part of the buffers: 16 bytes of piece c of row n at c ^ n.
  template <int DT, int ACT, class C, class T>
  __device__ __forceinline__ void tile(T& t, uint32_t m0, uint32_t n0, lds_char* even, lds_char* odd) const {
    if constexpr (ACT != ANY && T::TM * C::WM == C::BM) {  // not a narrower one
      if (direct && m0 + C::BM <= extent_m && n0 + C::BN <= extent_n) return whole<DT, ACT>(t, m0, n0);
    }
    constexpr uint32_t TM = T::TM, ROW = TM * 4, LANES = TM / 8, STEP = 64 / LANES, TURNS = 16 / STEP, G = TURNS < 2 ? 1 : 2, WAVES = T::THREADS / 64;
    static_assert(TM >= 32 && (WAVES + 1) / 2 * 16 * ROW <= T::BYTES, "the waves' parts fit the buffers");
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 15;
    lds_char* own = (wave & 1 ? odd : even) + (wave >> 1) * (16 * ROW);
    const uint32_t r = lane / LANES, c = lane % LANES, m = m0 + t.wave_m() + c * 8, first = n0 + t.wave_n();
    const uint64_t from = drop.off ? counter(m, first + r) : 0, row_step = words * pt_random::PHI;
    u32x4 qg[G] = {}, qr[G] = {};
    float qs[G] = {};
    const auto fetch = [&](uint32_t it) {
#pragma unroll
      for (uint32_t turn = 0; turn < G; ++turn) {
        const uint32_t n = min(first + (it * G + turn) * STEP + r, extent_n - 1);
        if (x_scale) qs[turn] = ((const PT_GLOBAL float*)x_scale)[n];
        if (gate) qg[turn] = fetch8((const PT_GLOBAL uint16_t*)gate + n * gate_stride, m, extent_m);
        if (residual) qr[turn] = fetch8((const PT_GLOBAL uint16_t*)residual + n * residual_stride, m, extent_m);
      }
    };
    Columns<DT, 8> columns;
    fetch(0);
    columns.load(*this, m);
    __syncthreads();                                       // every wave has read its last operands
#pragma unroll 1
    for (uint32_t it = 0; it < T::FN * TURNS / G; ++it) {
#pragma unroll
      for (int k = 0; k < T::FN; ++k)
        if (it == k * TURNS / G)
#pragma unroll
          for (int i = 0; i < T::FM; ++i) *(lds_f32x4*)(own + l * ROW + ((i * 4 + (lane >> 4)) ^ (l & (TM / 4 - 1))) * 16) = t.acc[i][k];
      u32x4 now_g[G], now_r[G];
      float now_s[G];
      f32x4 x[G][2];
#pragma unroll
      for (uint32_t turn = 0; turn < G; ++turn) {
        const uint32_t row = (it * G + turn) % TURNS * STEP + r;
        now_g[turn] = qg[turn]; now_r[turn] = qr[turn]; now_s[turn] = qs[turn];
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) x[turn][h] = *(lds_f32x4*)(own + row * ROW + ((c * 2 + h) ^ (row & (TM / 4 - 1))) * 16);
      }
      if ((it + 1) * G < T::FN * TURNS) fetch(it + 1);
#pragma unroll
      for (uint32_t turn = 0; turn < G; ++turn) {
        const uint32_t n = first + (it * G + turn) * STEP + r;
        if (n >= extent_n || m >= extent_m) continue;
        float y[8], g[8], b[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) y[q] = x[turn][q / 4][q % 4];
        columns.z(*this, now_s[turn], y);
        if (pre) store8((PT_GLOBAL uint16_t*)pre + n * pre_stride, m, extent_m, encode8<DT>(y));
        if (gate) decode8<DT>(place8(now_g[turn], m, extent_m), g);
        if (residual) decode8<DT>(place8(now_r[turn], m, extent_m), b);
        result<ACT>(y, from + (it * G + turn) * STEP * row_step, g, b);
        store8((PT_GLOBAL uint16_t*)out + n * out_stride, m, extent_m, encode8<DT>(y));
      }
    }
  }
  template <int DT>
  __device__ __forceinline__ void four(uint32_t m, uint32_t n, f32x4 x) const {
    if (n >= extent_n || m >= extent_m) return;
    float y[4] = {x[0], x[1], x[2], x[3]}, g[4] = {}, r[4] = {};
    const auto get = [&](const uint16_t* from, uint64_t stride, float (&to)[4]) {
      const f32x4 b = decode4<DT>(load4((const PT_GLOBAL uint16_t*)from + n * stride, m, extent_m));
#pragma unroll
      for (int i = 0; i < 4; ++i) to[i] = b[i];
    };
    if (gate) get(gate, gate_stride, g);
    if (residual) get(residual, residual_stride, r);
    Columns<DT, 4> columns;
    columns.load(*this, m);
    columns.z(*this, x_scale ? ((const PT_GLOBAL float*)x_scale)[n] : 1.0f, y);
    if (pre) store4((PT_GLOBAL uint16_t*)pre + n * pre_stride, m, extent_m, encode16x4<DT>(f32x4{y[0], y[1], y[2], y[3]}));
    result<ANY>(y, drop.off ? counter(m, n) : 0, g, r);
    store4((PT_GLOBAL uint16_t*)out + n * out_stride, m, extent_m, encode16x4<DT>(f32x4{y[0], y[1], y[2], y[3]}));
  }
};

// ---- products ------------------------------------------------------------------------------------------------

struct ProductArgs {
  Operand p, q;
  uint32_t extent_m, extent_n, twos;
  float* sums;
  Split split;
  bool low;                  // of d_x: rows LOW on are what rounding the rows LOW before has left
};

// Up to LOW rows what rounding dz leaves is multiplied as rows of its own, which lie LOW behind, in tiles that have room for them.  It is of few rows and outs that single
// roundings show: gradients of one row and 64 outs would have up to 2.1 times the error of rounding the result alone (of many rows 1.4).  1 x 4096 x 11008 56.5 -> 60.2
// us, 16 x 4096 x 11008 59.1 -> 61.1, as x is copied and dz twice as long.  An infinite operand is no matter of what is left (0 inf is NaN): in d_x it adds to finite sums
// only, which have no such operand, and for d_weight x is copied without them.
constexpr uint32_t LOW = 32;
static_assert(Few::BN == 2 * LOW, "both in a tile");

// MUL: PT_BF16, PT_FP16 or PT_E4M3, what is multiplied; DT: what the epilogue reads and writes.
template <int MUL, int DT, int ACT, class C, bool PK, bool QK, class E>
__device__ __forceinline__ void product_tile(const ProductArgs& a, const E& e, lds_char* even, lds_char* odd, uint32_t block) {
  uint32_t tm, tn, part;
  PT_GLOBAL float* left;
  if (!part_of<C>(a.split, block, (a.extent_m + C::BM - 1) / C::BM, (a.extent_n + C::BN - 1) / C::BN, a.sums, tm, tn, part, left)) return;
  const uint32_t t0 = left ? uint32_t(uint64_t(a.twos) * part / a.split.n) : 0, t1 = left ? uint32_t(uint64_t(a.twos) * (part + 1) / a.split.n) : a.twos;
  with_tile<MUL, C, PK, QK>(a.extent_m - tm * C::BM, [&](auto t) {
    typedef decltype(t) T;
    t.run(even, odd, a.p, a.q, tm * C::BM, tn * C::BN, t0 * TWO, t1 - t0);
    if constexpr (C::BN == 2 * LOW && !PK) {
      if (a.low) {
#pragma unroll
        for (int j = 0; j < T::FN / 2; ++j)
#pragma unroll
          for (int i = 0; i < T::FM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float x = t.acc[i][j][q];
            t.acc[i][j][q] = __builtin_fabsf(x) < __builtin_inff() ? x + t.acc[i][j + T::FN / 2][q] : x;
          }
      }
    }
    if (left) {
#pragma unroll
      for (int j = 0; j < T::FN; ++j) leave<C>(t, j, left);
      return;
    }
    e.template tile<DT, ACT, C>(t, tm * C::BM, tn * C::BN, even, odd);
  });
}

template <int MUL, int DT, int ACT, class C, bool PK, bool QK, class E>
__global__ void __launch_bounds__(C::THREADS) k_linear_product(const ProductArgs a, const E e) {
  constexpr int BYTES = C::template Of<MUL, PK, QK>::BYTES;
  __shared__ __attribute__((aligned(16))) char even[BYTES], odd[BYTES];
  product_tile<MUL, DT, ACT, C, PK, QK>(a, e, (lds_char*)even, (lds_char*)odd, blockIdx.x);
}

template <int DT, class C, class E>
__device__ __forceinline__ void join_product(const ProductArgs& a, const E& e, uint32_t block, uint32_t blocks) {
  join_tiles<C>(a.sums, a.split, (a.extent_m + C::BM - 1) / C::BM, (a.extent_n + C::BN - 1) / C::BN,
                [&](uint32_t m, uint32_t n, f32x4 x) { e.template four<DT>(m, n, x); }, block, blocks);
}
template <int DT, class C, class E>
__global__ void __launch_bounds__(256) k_linear_join(const ProductArgs a, const E e) {
  join_product<DT, C>(a, e, blockIdx.x, gridDim.x);
}

// Both gradients in one launch, where neither fills the chip for long: 1531 x 771 x 3083 in 29 us, one after the other 21 + 22 and a gap.  C: the tiles of d_x.
template <int DT, class C>
__global__ void __launch_bounds__(256) k_linear_both(const ProductArgs x, const Plain ex, const ProductArgs w, const Plain ew, uint32_t blocks_x) {
  static_assert(C::THREADS == 256 && Mid::THREADS == 256, "one launch");
  constexpr int BYTES = std::max(C::template Of<DT, false, true>::BYTES, Mid::Of<DT, false, false>::BYTES);
  __shared__ __attribute__((aligned(16))) char even[BYTES], odd[BYTES];
  if (blockIdx.x < blocks_x) product_tile<DT, DT, ANY, C, false, true>(x, ex, (lds_char*)even, (lds_char*)odd, blockIdx.x);
  else product_tile<DT, DT, ANY, Mid, false, false>(w, ew, (lds_char*)even, (lds_char*)odd, blockIdx.x - blocks_x);
}

// What is left of the gradients: sums of several workgroups a tile, and of the bias's columns.
struct BiasArgs {
  const float* part;
  uint32_t rows, pitch, outs;
  uint16_t* d_bias;
};
template <int DT, class C>
__global__ void __launch_bounds__(256) k_linear_ends(const ProductArgs x, const Plain ex, const ProductArgs w, const Plain ew, const BiasArgs b, uint32_t blocks_x,
                                                     uint32_t blocks_w) {
  if (blockIdx.x < blocks_x) join_product<DT, C>(x, ex, blockIdx.x, blocks_x);
  else if (blockIdx.x < blocks_x + blocks_w) join_product<DT, Mid>(w, ew, blockIdx.x - blocks_x, blocks_w);
  else add_columns<DT>(b.part, b.rows, b.pitch, b.outs, b.d_bias, blockIdx.x - blocks_x - blocks_w);
}
template <int DT>
__global__ void __launch_bounds__(256) k_linear_bias(const BiasArgs b) { add_columns<DT>(b.part, b.rows, b.pitch, b.outs, b.d_bias, blockIdx.x); }

// Up to 32 rows: they take as long as the weight takes to read, which each wave has on its way straight into the registers that are multiplied: 16 MT outs a workgroup, of
// which a wave takes 64 U bytes of k in every WAVES times as many.  Any address, stride and width; no workspace.
// (Before, tiles of Few: 1 x 4096 x 11008 34.7 -> 17.4 us, 5.2 TB/s; 17 rows 33.5 -> 22.4; 32 x 1600 x 6400 13.8 -> 8.4; but 32 x 11008 x 4096 28.0 -> 31.3: few outs and
// many rows of long k are read as often as the weight.)
inline bool thin(uint64_t rows, uint64_t outs, uint64_t bytes) { return rows <= 16 || (rows <= 32 && (outs > 6128 || bytes <= 16384)); }

struct ThinArgs {
  const char *x, *weight;
  uint64_t x_pitch, weight_pitch;          // bytes
  uint32_t rows, outs, bytes;              // of a row
};

// 16 bytes of a row from `at` on, zero behind its end.
template <int MUL>
__device__ __forceinline__ u32x4 end16(const PT_GLOBAL char* row, uint32_t at, uint32_t bytes) {
  if constexpr (MUL != PT_E4M3) return load8((const PT_GLOBAL uint16_t*)row, at / 2, bytes / 2);
  u32x4 q = {0, 0, 0, 0};
#pragma unroll
  for (uint32_t j = 0; j < 16; ++j)
    if (at + j < bytes) q[j / 4] |= uint32_t(uint8_t(row[at + j])) << (8 * (j & 3));
  return q;
}

template <int MUL, int DT, int MT, int RT, int U, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) k_linear_thin(const ThinArgs a, const Layer e) {
  constexpr uint32_t CHUNK = U * 64;
  constexpr int N = MT * RT;
  __shared__ __attribute__((aligned(16))) f32x4 s_acc[WAVES][N][64];
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 15, g = lane >> 4, m0 = blockIdx.x * (16 * MT);
  const PT_GLOBAL char *w[MT], *x[RT];
#pragma unroll
  for (int i = 0; i < MT; ++i) w[i] = (const PT_GLOBAL char*)a.weight + min(m0 + i * 16 + l, a.outs - 1) * a.weight_pitch;
#pragma unroll
  for (int i = 0; i < RT; ++i) x[i] = (const PT_GLOBAL char*)a.x + min(i * 16 + l, a.rows - 1) * a.x_pitch;
  f32x4 acc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const uint32_t whole = a.bytes / CHUNK;
  struct Step { u32x4 w[U][MT], x[U][RT]; } now, next;
  const auto load = [&](Step& to, uint32_t c) {
    const uint32_t at = c * CHUNK + g * 16;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < MT; ++i) to.w[u][i] = *(const PT_GLOBAL u32x4_b*)(w[i] + at + u * 64);
#pragma unroll
      for (int i = 0; i < RT; ++i) to.x[u][i] = *(const PT_GLOBAL u32x4_b*)(x[i] + at + u * 64);
    }
  };
  const auto multiply = [&](const Step& s, int u) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < RT; ++j) acc[i * RT + j] = mfma<MUL>(__builtin_bit_cast(s16x8, s.w[u][i]), __builtin_bit_cast(s16x8, s.x[u][j]), acc[i * RT + j]);
  };
  if (wave < whole) load(next, wave);
#pragma unroll 1
  for (uint32_t c = wave; c < whole; c += WAVES) {
    now = next;
    if (c + WAVES < whole) load(next, c + WAVES);
#pragma unroll
    for (int u = 0; u < U; ++u) multiply(now, u);
  }
  if (wave == whole % WAVES)               // what is left
#pragma unroll 1
    for (uint32_t at = whole * CHUNK; at < a.bytes; at += 64) {
#pragma unroll
      for (int i = 0; i < MT; ++i) now.w[0][i] = end16<MUL>(w[i], at + g * 16, a.bytes);
#pragma unroll
      for (int i = 0; i < RT; ++i) now.x[0][i] = end16<MUL>(x[i], at + g * 16, a.bytes);
      multiply(now, 0);
    }
#pragma unroll
  for (int i = 0; i < N; ++i) s_acc[wave][i][lane] = acc[i];
  __syncthreads();
#pragma unroll 1
  for (uint32_t i = wave; i < uint32_t(N); i += WAVES) {
    f32x4 sum = s_acc[0][i][lane];
#pragma unroll
    for (uint32_t k = 1; k < uint32_t(WAVES); ++k) sum += s_acc[k][i][lane];
    e.template four<DT>(m0 + i / RT * 16 + g * 4, i % RT * 16 + l, sum);
  }
}

// Rows whose beginnings, distances or ends the products cannot take: they load 16 bytes a lane past registers.
struct CopyArgs {
  const void* from;
  uint64_t stride;
  uint32_t rows, width, pitch;             // elements; pitch: of a copied row, which is zero behind its end
  void* to;
  uint32_t low;                            // 0, or how many rows there are: they go to rows 0 on and, but for infinities and NaN, to rows LOW on, zero up to LOW and 2 LOW
                                           // (rows is that then)
  uint32_t exponent;                       // of infinities and NaN
};
inline uint32_t copy_blocks(const CopyArgs& a) { return (a.rows + 3) / 4; }
// Of one or two bytes an element, four rows by a workgroup of 256.
template <int BYTES>
__device__ __forceinline__ void copy_rows(const CopyArgs& a, uint32_t block) {
  const uint32_t r = __builtin_amdgcn_readfirstlane(block * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  if (r >= a.rows) return;
  if constexpr (BYTES == 2) {
    const uint32_t from = a.low ? r % LOW : r, width = a.low && from >= a.low ? 0 : a.width;
    const PT_GLOBAL uint16_t* row = (const PT_GLOBAL uint16_t*)a.from + from * a.stride;
    PT_GLOBAL uint16_t* to = (PT_GLOBAL uint16_t*)a.to + size_t(r) * a.pitch;
    if (a.low && r >= LOW) copy_row<true>(row, to, width, a.pitch, lane, 64, a.exponent);
    else copy_row(row, to, width, a.pitch, lane, 64);
  } else {
    const PT_GLOBAL char* row = (const PT_GLOBAL char*)a.from + r * a.stride;
    PT_GLOBAL char* to = (PT_GLOBAL char*)a.to + size_t(r) * a.pitch;
#pragma unroll 4
    for (uint32_t c = lane * 16; c < a.pitch; c += 1024)
      *(PT_GLOBAL u32x4*)(to + c) = c + 16 <= a.width ? u32x4(*(const PT_GLOBAL u32x4_b*)(row + c)) : end16<PT_E4M3>(row, c, a.width);
  }
}
// Both operands; either may have no rows.
template <int BYTES>
__global__ void __launch_bounds__(256) k_linear_copy(const CopyArgs x, const CopyArgs w) {
  const uint32_t blocks = (x.rows + 3) / 4;
  if (blockIdx.x < blocks) copy_rows<BYTES>(x, blockIdx.x);
  else copy_rows<BYTES>(w, blockIdx.x - blocks);
}

// ---- slope ---------------------------------------------------------------------------------------------------

struct SlopeArgs {
  const uint16_t *d_out, *pre, *gate;
  uint16_t *dz, *d_gate;     // dz: rows of `pitch`, zero behind outs; or NULL: it is d_out
  float* part;               // [rows / rows_each][pitch]: sums of the columns, or NULL
  uint64_t d_out_stride, pre_stride, gate_stride, d_gate_stride;
  pt_random::Drop drop;
  uint64_t words;
  uint32_t rows, outs, pitch, rows_each, strips;       // strips of 512 columns
  int act;
  bool low;                  // 2 LOW rows of dz
};

// 512 columns, eight a lane, of rows_each rows, a quarter of which is a wave's.  Bound by memory.  The last workgroups copy what has to be copied of the
// operands: two launches less.
template <int DT>
__global__ void __launch_bounds__(256) k_linear_slope(const SlopeArgs a, const CopyArgs x, const CopyArgs w, uint32_t blocks) {
  if (blockIdx.x >= blocks) {
    const uint32_t i = blockIdx.x - blocks, blocks_x = (x.rows + 3) / 4;
    if (i < blocks_x) copy_rows<2>(x, i);
    else copy_rows<2>(w, i - blocks_x);
    return;
  }
  __shared__ float s_part[4][512];
  const uint32_t by = blockIdx.x / a.strips, bx = blockIdx.x - by * a.strips;
  const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = bx * 512 + lane * 8;
  const uint32_t first = by * a.rows_each, end = min(a.low ? LOW : a.rows, first + a.rows_each);
  const uint64_t from = a.drop.key() + (c / 4 + 1) * pt_random::PHI, row_step = a.words * pt_random::PHI;
  float sum[8] = {};
  if (c < a.pitch)
    with_act(a.act, [&](auto act) {
      for (uint32_t r = first + wave; r < end; r += 4) {
        u32x4 qe = {0, 0, 0, 0}, qz = qe, qg = qe;
        if (r >= a.rows) {                                 // of 2 LOW
          *(PT_GLOBAL u32x4*)((PT_GLOBAL uint16_t*)a.dz + size_t(r) * a.pitch + c) = qe;
          *(PT_GLOBAL u32x4*)((PT_GLOBAL uint16_t*)a.dz + size_t(r + LOW) * a.pitch + c) = qe;
          continue;
        }
        qe = fetch8((const PT_GLOBAL uint16_t*)a.d_out + r * a.d_out_stride, c, a.outs);
        if (a.pre) qz = fetch8((const PT_GLOBAL uint16_t*)a.pre + r * a.pre_stride, c, a.outs);
        if (a.gate) qg = fetch8((const PT_GLOBAL uint16_t*)a.gate + r * a.gate_stride, c, a.outs);
        float e[8], z[8], g[8], slope[8];
        decode8<DT>(place8(qe, c, a.outs), e);
        // last of all, so that what is dropped adds nothing, whatever pre and gate hold there
        const uint64_t z0 = a.drop.off ? pt_random::mix64(from + r * row_step) : 0, z1 = a.drop.off ? pt_random::mix64(from + r * row_step + pt_random::PHI) : 0;
        const auto drop = [&](float (&x)[8]) {
          if (!a.drop.off) return;
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = a.drop.of(j < 4 ? z0 : z1, j & 3, x[j]);
        };
        if (a.pre) {
          decode8<DT>(place8(qz, c, a.outs), z);
#pragma unroll
          for (int j = 0; j < 8; ++j) z[j] = ::act<act()>(z[j], slope[j]);
          if (a.d_gate) {
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] *= e[j];
            drop(z);
            store8((PT_GLOBAL uint16_t*)a.d_gate + r * a.d_gate_stride, c, a.outs, encode8<DT>(z));
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] *= slope[j];
        }
        if (a.gate) {
          decode8<DT>(place8(qg, c, a.outs), g);
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] *= g[j];
        }
        drop(e);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (c + j >= a.outs) e[j] = 0.0f;
          sum[j] += e[j];
        }
        if (a.dz) {
          const u32x4 w = encode8<DT>(e);
          *(PT_GLOBAL u32x4*)((PT_GLOBAL uint16_t*)a.dz + size_t(r) * a.pitch + c) = w;
          if (a.low) {
            float y[8];
            decode8<DT>(w, y);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = __builtin_fabsf(y[j]) < __builtin_inff() ? e[j] - y[j] : 0.0f;       // inf stays inf
            *(PT_GLOBAL u32x4*)((PT_GLOBAL uint16_t*)a.dz + size_t(r + LOW) * a.pitch + c) = encode8<DT>(y);
          }
        }
      }
    });
  if (!a.part) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) s_part[wave][lane * 8 + j] = sum[j];
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < 512; i += 256) {
    const uint32_t col = bx * 512 + i;
    if (col < a.pitch) ((PT_GLOBAL float*)a.part)[size_t(by) * a.pitch + col] = ((s_part[0][i] + s_part[1][i]) + s_part[2][i]) + s_part[3][i];
  }
}

__global__ void __launch_bounds__(256) k_linear_zero(uint16_t* __restrict__ out, uint64_t stride, uint32_t width) {
  for (uint32_t c = threadIdx.x; c < width; c += 256) out[blockIdx.x * stride + c] = 0;
}

// ---- host ------------------------------------------------------------------------------------------------------

enum Kind { BIG, MID, FEW };
struct Choice { Kind kind; Split split; uint64_t bytes; };

// Which tiles a product of m x n is soonest done in (of Big's the last of m may be a narrower one), and how they are split.  layer: with an epilogue, which in Big nothing
// else of its compute unit hides (8192 x 768 x 2304 57.7 us in Big, 50.1 in Mid; 4096 x 512 x 4096 28.1, 33.3).
Choice choose(uint32_t m, uint32_t n, uint32_t twos, bool layer) {
  const auto of = [&](auto c, Kind kind) {
    typedef decltype(c) C;
    const Split s = split<C>((m + C::BM - 1) / C::BM * ((n + C::BN - 1) / C::BN), twos, !layer ? 3000 : C::BM == 256 ? 12000 : 5000);
    return Choice{kind, s, 4ull * s.tail * s.n * C::BM * C::BN};
  };
  if (n <= uint32_t(Few::BN)) {
    Choice c = of(Few{}, FEW);
    // shared by so few workgroups that a quarter of the chip idles: by twice as many, two of which fit a compute unit (64 rows, once and twice as many: 4096 x 11008, 172,
    // 36.0 and 29.2 us; 4096 x 12288, 192, 37.3 and 30.9).  Where more run, twice as many cost their sums if the weight is short (1600 x 6400, 250, 13.7 and 13.7; 4096 x 5120,
    // 240, 16.8 and 17.9; 4096 x 4096, 15.5 and 17.0; 2048 x 8192, 15.6 and 17.1); of a long one they would pay too, which this rule leaves (5120 x 13824, 216, 51.9 and 45.6;
    // 4096 x 14336, 224, 41.7 and 34.5; 8192 x 8192, 44.0 and 38.8).
    if (layer && c.split.tail && !c.split.whole && c.split.tail * c.split.n <= 192 && c.split.n * 4 <= twos) {
      c.split.n *= 2;
      c.bytes *= 2;
    }
    return c;
  }
  const Choice big = of(Big{}, BIG), mid = of(Mid{}, MID);
  const uint32_t left = m % 256, tenths = m / 256 * 10 + (left == 0 ? 0 : left <= 64 ? 4 : left <= 128 ? 6 : 10);
  return mid.split.ns < big.split.ns * tenths / ((m + 255) / 256 * 10) ? mid : big;
}

bool direct(const void* at, uint64_t stride, uint32_t width, uint32_t bytes) {
  return uint64_t(width) * bytes % 128 == 0 && stride * bytes % 16 == 0 && (uintptr_t)at % 16 == 0 && stride <= (1u << 21);
}

// Where everything lies in the workspace.
struct Plan {
  bool x_direct, w_direct, slope;          // slope: the products need a dz that is not d_out
  bool both;                               // gradients in one launch
  bool low;                                // as in ProductArgs
  uint32_t rows;                           // of dz and the x that is multiplied with it
  uint32_t Kd, Np;                         // width and outs rounded up to whole steps (Kd in 16-bit words)
  Choice c, c_x, c_w;
  uint32_t rows_each, row_blocks;
  uint64_t x, w, dz, part, sums, sums_w, total;
};

bool in8(const pt_linear& l) { return l.x_scale != nullptr; }

struct Taker {
  uint64_t at = 0;
  uint64_t operator()(uint64_t bytes) { const uint64_t x = at; at += up(bytes, 256); return x; }
};

Plan plan_out(const pt_linear& l) {
  Plan p{};
  const uint32_t bytes = in8(l) ? 1 : 2;
  if (thin(l.rows, l.outs, uint64_t(l.width) * bytes)) return p;
  Taker take;
  p.Kd = uint32_t(up(uint64_t(l.width) * bytes, 2 * TWO) / 2);
  p.x_direct = direct(l.x, l.x_stride, l.width, bytes);
  p.w_direct = direct(l.weight, l.weight_stride, l.width, bytes);
  p.c = choose(l.outs, l.rows, p.Kd / TWO, true);
  p.x = take(p.x_direct ? 0 : 2ull * l.rows * p.Kd);
  p.w = take(p.w_direct ? 0 : 2ull * l.outs * p.Kd);
  p.sums = take(p.c.bytes);
  p.total = take.at;
  return p;
}

Plan plan_grads(const pt_linear& l) {
  Plan p{};
  Taker take;
  p.Kd = uint32_t(up(l.width, TWO));
  p.Np = uint32_t(up(l.outs, TWO));
  const bool rounds = l.act != PT_ACT_NONE || l.gate || l.drop.p > 0.0;
  p.low = rounds && l.rows <= LOW && (l.d_x || l.d_weight);
  p.rows = p.low ? 2 * LOW : l.rows;
  p.x_direct = !l.d_weight || (!p.low && direct(l.x, l.x_stride, l.width, 2));
  p.w_direct = !l.d_x || direct(l.weight, l.weight_stride, l.width, 2);
  p.slope = (l.d_x || l.d_weight) && (rounds || !direct(l.d_out, l.d_out_stride, l.outs, 2));
  p.x = take(p.x_direct ? 0 : 2ull * p.rows * p.Kd);
  p.w = take(p.w_direct ? 0 : 2ull * l.outs * p.Kd);
  p.dz = take(p.slope ? 2ull * p.rows * p.Np : 0);
  const uint32_t strips = (p.Np + 511) / 512;
  p.rows_each = std::max(16u, std::min(256u, uint32_t(uint64_t(l.rows) * strips / 2048)));
  p.rows_each = std::max(p.rows_each, (l.rows + 65534) / 65535);
  p.row_blocks = ((p.low ? LOW : l.rows) + p.rows_each - 1) / p.rows_each;
  p.part = take(l.d_bias ? 4ull * p.row_blocks * p.Np : 0);
  if (l.d_x) p.c_x = choose(l.width, p.rows, p.Np / TWO, false);
  if (l.d_weight) p.c_w = choose(l.width, l.outs, (p.rows + TWO - 1) / TWO, false);
  // of few rows both are a matter of reading the weight or writing its gradient: side by side (16 x 4096 x 11008 61.0 -> 53.6 us, 3 x 12796 x 2624 84.8 -> 66.2)
  if (l.d_x && l.d_weight && p.c_x.kind == FEW && p.c_w.kind == BIG)
    p.c_w = {MID, {(l.width + Mid::BM - 1) / Mid::BM * ((l.outs + Mid::BN - 1) / Mid::BN), 0, 1, 0}, 0};
  p.both = l.d_x && l.d_weight && p.c_x.kind != BIG && p.c_w.kind == MID;
  p.sums = take(p.both ? p.c_x.bytes : std::max(p.c_x.bytes, p.c_w.bytes));
  p.sums_w = p.both ? take(p.c_w.bytes) : p.sums;
  p.total = take.at;
  return p;
}

int check(const pt_linear* l, const char* who) {
  if (!l) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: layer is NULL", who);
  if (l->dtype != PT_BF16 && l->dtype != PT_FP16) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: dtype %d is neither PT_BF16 nor PT_FP16", who, l->dtype);
  if (l->act < PT_ACT_NONE || l->act > PT_ACT_SILU) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: act %d is none of pt_act", who, l->act);
  if (!l->outs || !l->width) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: outs and width must be > 0", who);
  if (!pt_random::valid(l->drop)) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: the dropout's p is not in [0, 1)", who);
  if (!l->x_scale != !l->weight_scale) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: scales of one operand only", who);
  const struct { const void* at; uint64_t stride; uint32_t width; } rows[] = {
    {l->x, l->x_stride, l->width}, {l->weight, l->weight_stride, l->width}, {l->gate, l->gate_stride, l->outs}, {l->residual, l->residual_stride, l->outs},
    {l->pre, l->pre_stride, l->outs}, {l->out, l->out_stride, l->outs}, {l->d_out, l->d_out_stride, l->outs}, {l->d_x, l->d_x_stride, l->width},
    {l->d_weight, l->d_weight_stride, l->width}, {l->d_gate, l->d_gate_stride, l->outs}};
  for (const auto& x : rows)
    if (x.at && x.stride < x.width) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: rows of width %u at a smaller stride", who, x.width);
  uintptr_t a = (uintptr_t)l->bias | (uintptr_t)l->gate | (uintptr_t)l->residual | (uintptr_t)l->pre | (uintptr_t)l->out | (uintptr_t)l->d_out |
                (uintptr_t)l->d_x | (uintptr_t)l->d_weight | (uintptr_t)l->d_bias | (uintptr_t)l->d_gate;
  if (!l->x_scale) a |= (uintptr_t)l->x | (uintptr_t)l->weight;
  if (a % 2 != 0 || ((uintptr_t)l->x_scale | (uintptr_t)l->weight_scale) % 4 != 0 || (uintptr_t)l->drop.step % 8 != 0)
    return pt_fail(nullptr, PT_ERR_ALIGNMENT, "%s: an array is not aligned to its elements", who);
  const auto tiles = [](uint64_t m, uint64_t n) { return ((m + 127) / 128) * ((n + 127) / 128); };
  if (l->rows > (1u << 25) || l->outs > (1u << 21) || l->width > (1u << 20) ||
      std::max({tiles(l->outs, l->rows), tiles(l->width, l->rows), tiles(l->width, l->outs)}) >= (1u << 24))
    return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "%s: more than 2^25 rows, 2^21 outs, a width over 2^20 or too many tiles", who);
  return PT_OK;
}
int check_workspace(uint64_t need, const void* workspace, uint64_t bytes, const char* who) {
  if (!need) return PT_OK;
  if (!workspace) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: workspace is NULL", who);
  if ((uintptr_t)workspace % 256 != 0) return pt_fail(nullptr, PT_ERR_ALIGNMENT, "%s: the workspace is not 256-byte aligned", who);
  if (need > bytes)
    return pt_fail(nullptr, PT_ERR_NOMEM, "%s: a workspace of %llu bytes is too small (pt_linear_workspace)", who, (unsigned long long)bytes);
  return PT_OK;
}

// Launches.
template <int MUL, int DT, class C, bool PK, bool QK, class E> int product_of(const ProductArgs& a, const E& e, hipStream_t st) {
  const auto launch = [&](auto act) {
    hipLaunchKernelGGL((k_linear_product<MUL, DT, act(), C, PK, QK, E>), dim3(split_grid(a.split)), dim3(C::THREADS), 0, st, a, e);
  };
  if constexpr (std::is_same_v<E, Layer> && C::BM == 256) with_act(e.act, launch);
  else launch(std::integral_constant<int, ANY>{});
  PT_LAUNCH_CHECK(nullptr, "k_linear_product");
  if (!a.split.tail) return PT_OK;
  hipLaunchKernelGGL((k_linear_join<DT, C, E>), dim3(joiners<C>(a.split.tail)), dim3(256), 0, st, a, e);
  PT_LAUNCH_CHECK(nullptr, "k_linear_join");
  return PT_OK;
}
template <int MUL, int DT, bool PK, bool QK, class E> int product(Kind k, const ProductArgs& a, const E& e, hipStream_t st) {
  return k == FEW ? product_of<MUL, DT, Few, PK, QK>(a, e, st) : k == MID ? product_of<MUL, DT, Mid, PK, QK>(a, e, st) : product_of<MUL, DT, Big, PK, QK>(a, e, st);
}

template <int DT, class C> int both(const ProductArgs& x, const Plain& ex, const ProductArgs& w, const Plain& ew, const BiasArgs& b, uint32_t bias_blocks, hipStream_t st) {
  const uint32_t grid = split_grid(x.split);
  hipLaunchKernelGGL((k_linear_both<DT, C>), dim3(grid + split_grid(w.split)), dim3(256), 0, st, x, ex, w, ew, grid);
  PT_LAUNCH_CHECK(nullptr, "k_linear_both");
  const uint32_t jx = joiners<C>(x.split.tail), jw = joiners<Mid>(w.split.tail);
  if (!(jx + jw + bias_blocks)) return PT_OK;
  hipLaunchKernelGGL((k_linear_ends<DT, C>), dim3(jx + jw + bias_blocks), dim3(256), 0, st, x, ex, w, ew, b, jx, jw);
  PT_LAUNCH_CHECK(nullptr, "k_linear_ends");
  return PT_OK;
}

// The operand of rows as they lie, or as they have been copied.
Operand rows_of(bool as_is, const void* at, uint64_t stride, uint32_t width, const void* copy, uint32_t pitch, uint32_t rows) {
  return as_is ? Operand{at, stride * 2, rows, width} : Operand{copy, 2ull * pitch, rows, pitch};
}
template <int BYTES> int copy(const CopyArgs& x, const CopyArgs& w, hipStream_t st) {
  if (!x.rows && !w.rows) return PT_OK;
  hipLaunchKernelGGL(k_linear_copy<BYTES>, dim3(copy_blocks(x) + copy_blocks(w)), dim3(256), 0, st, x, w);
  PT_LAUNCH_CHECK(nullptr, "k_linear_copy");
  return PT_OK;
}

template <int MUL, int DT, int MT, int RT, int U, int WAVES> int thin_of(const ThinArgs& a, const Layer& e, hipStream_t st) {
  hipLaunchKernelGGL((k_linear_thin<MUL, DT, MT, RT, U, WAVES>), dim3((a.outs + 16 * MT - 1) / (16 * MT)), dim3(WAVES * 64), 0, st, a, e);
  PT_LAUNCH_CHECK(nullptr, "k_linear_thin");
  return PT_OK;
}
template <int MUL, int DT> int run_thin(const ThinArgs& a, const Layer& e, hipStream_t st) {
  const uint32_t groups = (a.outs + 15) / 16;
  if (a.rows <= 16) {
    return groups >= 512 ? thin_of<MUL, DT, 1, 1, 2, 4>(a, e, st) : groups >= 256 ? thin_of<MUL, DT, 1, 1, 2, 8>(a, e, st) : thin_of<MUL, DT, 1, 1, 2, 16>(a, e, st);
  }
  return groups >= 640 ? thin_of<MUL, DT, 4, 2, 2, 8>(a, e, st) : groups >= 384 ? thin_of<MUL, DT, 2, 2, 2, 8>(a, e, st) : thin_of<MUL, DT, 1, 2, 2, 8>(a, e, st);
}

template <int DT> int run_out(const pt_linear& l, const Plan& p, char* ws, hipStream_t st) {
  const bool b8 = in8(l);
  // where a gate is not read and rows begin at multiples of 16 bytes (in pieces of lines: whole)
  const bool direct = !l.gate && ((uintptr_t)l.out | (uintptr_t)l.pre | (uintptr_t)l.residual) % 16 == 0 &&
                      ((l.out_stride | (l.pre ? l.pre_stride : 0) | (l.residual ? l.residual_stride : 0)) % 8 == 0);
  const Layer e = {(const uint16_t*)l.bias, (const uint16_t*)l.gate, (const uint16_t*)l.residual, (uint16_t*)l.pre, (uint16_t*)l.out, l.x_scale, l.weight_scale,
                   l.gate_stride, l.residual_stride, l.pre_stride, l.out_stride, l.outs, l.rows, l.act, pt_random::make(l.drop), (uint64_t(l.outs) + 3) / 4, direct};
  const uint32_t bytes = b8 ? 1 : 2;
  if (thin(l.rows, l.outs, uint64_t(l.width) * bytes)) {
    const ThinArgs a = {(const char*)l.x, (const char*)l.weight, l.x_stride * bytes, l.weight_stride * bytes, l.rows, l.outs, l.width * bytes};
    return b8 ? run_thin<PT_E4M3, DT>(a, e, st) : run_thin<DT, DT>(a, e, st);
  }
  const uint32_t pitch = 2 * p.Kd / bytes;
  const CopyArgs cx = {l.x, l.x_stride, p.x_direct ? 0 : l.rows, l.width, pitch, ws + p.x, 0, 0}, cw = {l.weight, l.weight_stride, p.w_direct ? 0 : l.outs, l.width, pitch, ws + p.w, 0, 0};
  if (int rc = b8 ? copy<1>(cx, cw, st) : copy<2>(cx, cw, st); rc != PT_OK) return rc;
  const uint32_t per = b8 ? 2 : 1;         // elements in a 16-bit word
  const ProductArgs a = {rows_of(p.w_direct, l.weight, l.weight_stride / per, l.width / per, ws + p.w, p.Kd, l.outs),
                         rows_of(p.x_direct, l.x, l.x_stride / per, l.width / per, ws + p.x, p.Kd, l.rows), l.outs, l.rows, p.Kd / TWO, (float*)(ws + p.sums),
                         p.c.split, false};
  return b8 ? product<PT_E4M3, DT, true, true>(p.c.kind, a, e, st) : product<DT, DT, true, true>(p.c.kind, a, e, st);
}

template <int DT> int run_grads(const pt_linear& l, const Plan& p, char* ws, hipStream_t st) {
  const CopyArgs cx = {l.x, l.x_stride, p.x_direct ? 0 : p.rows, l.width, p.Kd, ws + p.x, p.low ? l.rows : 0, DT == PT_BF16 ? 0x7f80u : 0x7c00u};
  const CopyArgs cw = {l.weight, l.weight_stride, p.w_direct ? 0 : l.outs, l.width, p.Kd, ws + p.w, 0, 0};
  if (p.slope || l.d_bias || l.d_gate) {
    const SlopeArgs a = {(const uint16_t*)l.d_out, l.act != PT_ACT_NONE || l.gate ? (const uint16_t*)l.pre : nullptr, (const uint16_t*)l.gate,
                         p.slope ? (uint16_t*)(ws + p.dz) : nullptr, (uint16_t*)l.d_gate, l.d_bias ? (float*)(ws + p.part) : nullptr, l.d_out_stride,
                         l.pre_stride, l.gate_stride, l.d_gate_stride, pt_random::make(l.drop), (uint64_t(l.outs) + 3) / 4, l.rows, l.outs, p.Np, p.rows_each,
                         (p.Np + 511) / 512, l.act, p.low};
    const uint32_t blocks = a.strips * p.row_blocks;
    hipLaunchKernelGGL(k_linear_slope<DT>, dim3(blocks + copy_blocks(cx) + copy_blocks(cw)), dim3(256), 0, st, a, cx, cw, blocks);
    PT_LAUNCH_CHECK(nullptr, "k_linear_slope");
  } else if (int rc = copy<2>(cx, cw, st); rc != PT_OK) {
    return rc;
  }
  const BiasArgs bias = {(const float*)(ws + p.part), p.row_blocks, p.Np, l.outs, (uint16_t*)l.d_bias};
  const uint32_t bias_blocks = l.d_bias ? column_blocks(l.outs) : 0;
  if (l.d_bias && !p.both) {
    hipLaunchKernelGGL(k_linear_bias<DT>, dim3(bias_blocks), dim3(256), 0, st, bias);
    PT_LAUNCH_CHECK(nullptr, "k_linear_bias");
  }
  const Operand dz = p.slope ? Operand{ws + p.dz, 2ull * p.Np, 0, 0} : Operand{l.d_out, 2 * l.d_out_stride, 0, 0};
  const uint32_t dz_width = p.slope ? p.Np : l.outs;
  // of weight and x, k are their rows
  const auto across = [](Operand o, uint32_t rows) { return Operand{o.at, o.pitch, o.k, rows}; };
  const ProductArgs ax = {across(rows_of(p.w_direct, l.weight, l.weight_stride, l.width, ws + p.w, p.Kd, 0), l.outs), {dz.at, dz.pitch, p.rows, dz_width}, l.width, p.rows,
                          p.Np / TWO, (float*)(ws + p.sums), p.c_x.split, p.low};
  const ProductArgs aw = {across(rows_of(p.x_direct, l.x, l.x_stride, l.width, ws + p.x, p.Kd, 0), p.rows), {dz.at, dz.pitch, dz_width, p.rows}, l.width, l.outs,
                          (p.rows + TWO - 1) / TWO, (float*)(ws + p.sums_w), p.c_w.split, false};
  const Plain ex = {(uint16_t*)l.d_x, l.d_x_stride, l.width, l.rows}, ew = {(uint16_t*)l.d_weight, l.d_weight_stride, l.width, l.outs};
  if (p.both) return p.c_x.kind == FEW ? both<DT, Few>(ax, ex, aw, ew, bias, bias_blocks, st) : both<DT, Mid>(ax, ex, aw, ew, bias, bias_blocks, st);
  if (l.d_x)
    if (int rc = product<DT, DT, false, true>(p.c_x.kind, ax, ex, st); rc != PT_OK) return rc;
  return l.d_weight ? product<DT, DT, false, false>(p.c_w.kind, aw, ew, st) : int(PT_OK);
}

}  // namespace

extern "C" int pt_linear_workspace(const pt_linear* layer, uint64_t* out_bytes, uint64_t* grads_bytes) {
  if (int rc = check(layer, "pt_linear_workspace"); rc != PT_OK) return rc;
  if (out_bytes) *out_bytes = layer->rows ? plan_out(*layer).total : 0;
  if (grads_bytes) *grads_bytes = layer->rows && !in8(*layer) ? plan_grads(*layer).total : 0;
  return PT_OK;
}

extern "C" int pt_linear_out(const pt_linear* l, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (int rc = check(l, "pt_linear_out"); rc != PT_OK) return rc;
  if (!l->rows) return PT_OK;
  if (!l->x || !l->weight || !l->out) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_linear_out: NULL array");
  const Plan p = plan_out(*l);
  if (int rc = check_workspace(p.total, workspace, workspace_bytes, "pt_linear_out"); rc != PT_OK) return rc;
  return l->dtype == PT_BF16 ? run_out<PT_BF16>(*l, p, (char*)workspace, (hipStream_t)stream) : run_out<PT_FP16>(*l, p, (char*)workspace, (hipStream_t)stream);
}

extern "C" int pt_linear_grads(const pt_linear* l, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (int rc = check(l, "pt_linear_grads"); rc != PT_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (in8(*l)) return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "pt_linear_grads: operands in 8 bits");
  if (l->d_gate && !l->gate) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_linear_grads: d_gate without a gate");
  if (!l->rows) {
    if (l->d_weight) {
      hipLaunchKernelGGL(k_linear_zero, dim3(l->outs), dim3(256), 0, st, (uint16_t*)l->d_weight, l->d_weight_stride, l->width);
      PT_LAUNCH_CHECK(nullptr, "k_linear_zero");
    }
    if (l->d_bias) {
      hipLaunchKernelGGL(k_linear_zero, dim3(1), dim3(256), 0, st, (uint16_t*)l->d_bias, 0, l->outs);
      PT_LAUNCH_CHECK(nullptr, "k_linear_zero");
    }
    return PT_OK;
  }
  if (!l->d_out || (l->d_weight && !l->x) || (l->d_x && !l->weight) || ((l->act != PT_ACT_NONE || l->gate) && !l->pre))
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_linear_grads: NULL array");
  const Plan p = plan_grads(*l);
  if (int rc = check_workspace(p.total, workspace, workspace_bytes, "pt_linear_grads"); rc != PT_OK) return rc;
  return l->dtype == PT_BF16 ? run_grads<PT_BF16>(*l, p, (char*)workspace, st) : run_grads<PT_FP16>(*l, p, (char*)workspace, st);
}
