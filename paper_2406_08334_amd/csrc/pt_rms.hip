// RMS norm with the residual's addition, its gradients, and rows in 8 bits.
//
//   norm    s = x + residual, rstd = 1 / sqrt(mean s^2 + eps), y = s rstd gain, in 16 bits or as e4m3 codes with the row's scale
//   grads   t = d_y gain, d_x = d_sum + rstd (t - s rstd^2 mean(t s)), d_gain = sum over rows of d_y s rstd
//   rows8   e4m3 codes of rows as they are
//
// Bound by memory: a row is held in registers between its sums and its results, so that every array is read or written once.  A row is a wave's, or that
// of several waves, so that a lane has 32 of its elements at most.  The gain's gradient is summed by lanes over the rows that their workgroup goes through, and
// from there by columns.  With the residual, bf16: norm of 8192 x 4096 45.7 us, 5.9 TB/s; in 8 bits 16384 x 5120 101 us, 5.8; gradients of 8192 x 4096 48 and 4 us, 5.6;
// rows8 of 13824 x 5120 in fp32 61 us, 5.8.
#include "pt_rows.h"

#include <cfloat>
#include <cmath>

using namespace pt_rows_ops;

namespace {

constexpr uint32_t MOST_WIDTH = 32768;
constexpr uint32_t MOST_ROWS = 1u << 21;   // of a launch: 2^32 lanes are more than a grid may have

// Sum of x, and largest of `big`, over the lanes that share a row.
template <int WAVES>
__device__ __forceinline__ float row_sum(float x, float* s) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x += s[w];
  }
  return x;
}
template <int WAVES>
__device__ __forceinline__ uint32_t row_max(uint32_t x, uint32_t* s) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = max(x, uint32_t(__shfl_xor(int(x), off, 64)));
  if constexpr (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x = max(x, s[w]);
  }
  return x;
}

// Which rows a workgroup's waves have and which elements a lane: pieces of eight, piece p at lane_at + p * step.
template <int WAVES> struct Rows {
  static constexpr int THREADS = WAVES >= 4 ? WAVES * 64 : 256, PER = THREADS / 64 / WAVES;
  static constexpr uint32_t STEP = WAVES * 64 * 8;
  static __device__ __forceinline__ uint32_t first() { return __builtin_amdgcn_readfirstlane(blockIdx.x * PER + (WAVES == 1 ? threadIdx.x >> 6 : 0)); }
  static __device__ __forceinline__ uint32_t lane_at() { return (WAVES == 1 ? threadIdx.x & 63 : threadIdx.x) * 8; }
};

struct NormArgs {
  const uint16_t *x, *residual, *gain;
  uint16_t* sum;
  float* rstd;
  void* y;
  float* y_scale;
  uint64_t x_stride, residual_stride, sum_stride, y_stride;
  float eps, inv_width;
  uint32_t rows, width;
};

// AHEAD: workgroups take rows one after the other, the next one's loads under way while one is worked on.  That is for 8 bits, whose second sum over the row
// leaves the memory idle otherwise (16384 x 5120 fp16 117 -> 106 us with two workgroups a compute unit, 111 with four; 16 bits 124 -> 127).
template <int DT, int WAVES, int PIECES, bool AHEAD>
__global__ void __launch_bounds__(Rows<WAVES>::THREADS) k_rms(const NormArgs a) {
  typedef Rows<WAVES> R;
  __shared__ float s_sum[2][WAVES];
  __shared__ uint32_t s_big[2][WAVES];
  const uint32_t first = R::first(), at = R::lane_at();
  u32x4 qg[PIECES];
  struct Row { u32x4 x[PIECES], r[PIECES]; } now, next;
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
    if (a.gain) qg[p] = fetch8((const PT_GLOBAL uint16_t*)a.gain, at + p * R::STEP, a.width);
  const auto load = [&](Row& to, uint32_t r) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      to.x[p] = fetch8((const PT_GLOBAL uint16_t*)a.x + r * a.x_stride, at + p * R::STEP, a.width);
      if (a.residual) to.r[p] = fetch8((const PT_GLOBAL uint16_t*)a.residual + r * a.residual_stride, at + p * R::STEP, a.width);
    }
  };
  if (first < a.rows) load(AHEAD ? next : now, first);
  uint32_t odd = 0;
  const uint32_t turn = gridDim.x * R::PER;
  for (uint32_t r = first; r < a.rows; r += turn, odd ^= 1) {
    if constexpr (AHEAD) {
      now = next;
      if (r + turn < a.rows) load(next, r + turn);
    }
    float v[PIECES][8], sq = 0.0f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      decode8<DT>(place8(now.x[p], at + p * R::STEP, a.width), v[p]);
      if (a.residual) {
        float b[8];
        decode8<DT>(place8(now.r[p], at + p * R::STEP, a.width), b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[p][j] += b[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sq = __builtin_fmaf(v[p][j], v[p][j], sq);
    }
    sq = row_sum<WAVES>(sq, s_sum[odd]);
    const float rstd = 1.0f / __builtin_sqrtf(__builtin_fmaf(sq, a.inv_width, a.eps));
    if (a.rstd && at == 0) ((PT_GLOBAL float*)a.rstd)[r] = rstd;
    uint32_t big = 0;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      if (a.sum) pass8((PT_GLOBAL uint16_t*)a.sum + r * a.sum_stride, at + p * R::STEP, a.width, encode8<DT>(v[p]));
      float g[8];
      if (a.gain) decode8<DT>(place8(qg[p], at + p * R::STEP, a.width), g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[p][j] *= rstd;
        if (a.gain) v[p][j] *= g[j];
        big = max(big, __float_as_uint(v[p][j]) & 0x7fffffffu);
      }
    }
    if (!a.y_scale) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p) pass8((PT_GLOBAL uint16_t*)a.y + r * a.y_stride, at + p * R::STEP, a.width, encode8<DT>(v[p]));
      if constexpr (AHEAD) continue;
      else return;
    }
    const Scale8 s = scale8(row_max<WAVES>(big, s_big[odd]));
#pragma unroll
    for (int p = 0; p < PIECES; ++p) pass8b((PT_GLOBAL uint8_t*)a.y + r * a.y_stride, at + p * R::STEP, a.width, codes8(v[p], s.inv));
    if (at == 0) ((PT_GLOBAL float*)a.y_scale)[r] = s.scale;
    if constexpr (!AHEAD) return;
  }
}

struct GradArgs {
  const uint16_t *sum, *gain, *d_y, *d_sum;
  const float* rstd;
  uint16_t* d_x;
  float* part;               // [gridDim.x * PER][pitch]: sums of the gain's gradient, or NULL
  uint64_t sum_stride, d_y_stride, d_sum_stride, d_x_stride, pitch;
  float inv_width;
  uint32_t rows, width, turn;            // turn: rows that all workgroups take at a time
};

// The rows of a workgroup one after the other; where registers allow it, the next one's loads are under way while one is worked on.  What is kept of a row
// over its sum is its words, and they are decoded once more: 24 registers for eight elements instead of 36.
template <int DT, int WAVES, int PIECES>
__global__ void __launch_bounds__(Rows<WAVES>::THREADS) k_rms_grads(const GradArgs a) {
  typedef Rows<WAVES> R;
  constexpr bool AHEAD = WAVES * PIECES <= 16;
  __shared__ float s_sum[2][WAVES];
  const uint32_t first = R::first(), at = R::lane_at();
  struct Row {
    u32x4 s[PIECES], d[PIECES], r[PIECES];
    float rstd;
  } now, next;
  u32x4 qg[PIECES];
  float dg[PIECES][8] = {};
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
    if (a.gain) qg[p] = fetch8((const PT_GLOBAL uint16_t*)a.gain, at + p * R::STEP, a.width);
  const auto load = [&](Row& to, uint32_t r) {
    to.rstd = ((const PT_GLOBAL float*)a.rstd)[r];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      to.s[p] = fetch8((const PT_GLOBAL uint16_t*)a.sum + r * a.sum_stride, at + p * R::STEP, a.width);
      to.d[p] = fetch8((const PT_GLOBAL uint16_t*)a.d_y + r * a.d_y_stride, at + p * R::STEP, a.width);
      if (a.d_sum) to.r[p] = fetch8((const PT_GLOBAL uint16_t*)a.d_sum + r * a.d_sum_stride, at + p * R::STEP, a.width);
    }
  };
  // s rstd and d_y of piece p
  const auto piece = [&](int p, float (&s)[8], float (&t)[8]) {
    decode8<DT>(place8(now.s[p], at + p * R::STEP, a.width), s);
    decode8<DT>(place8(now.d[p], at + p * R::STEP, a.width), t);
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] *= now.rstd;
  };
  const auto gained = [&](int p, float (&t)[8]) {
    if (!a.gain) return;
    float g[8];
    decode8<DT>(place8(qg[p], at + p * R::STEP, a.width), g);
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] *= g[j];
  };
  if (first < a.rows) load(AHEAD ? next : now, first);
  uint32_t odd = 0;
  for (uint32_t r = first; r < a.rows; r += a.turn, odd ^= 1) {
    if constexpr (AHEAD) {
      now = next;
      if (r + a.turn < a.rows) load(next, r + a.turn);
    } else if (r != first) {
      load(now, r);
    }
    float c = 0.0f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      __builtin_amdgcn_sched_barrier(0);
      float s[8], t[8];
      piece(p, s, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) dg[p][j] = __builtin_fmaf(t[j], s[j], dg[p][j]);
      gained(p, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) c = __builtin_fmaf(t[j], s[j], c);
    }
    c = row_sum<WAVES>(c, s_sum[odd]) * a.inv_width;       // two arrays in turn: the next row's sums don't wait for this one's readers
    if (!a.d_x) continue;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      __builtin_amdgcn_sched_barrier(0);                   // piece by piece: together they would take twice the registers
      asm volatile("" : "+v"(now.s[p]), "+v"(now.d[p]), "+v"(qg[p]));
      float s[8], t[8], d[8];
      piece(p, s, t);
      gained(p, t);
      if (a.d_sum) decode8<DT>(place8(now.r[p], at + p * R::STEP, a.width), d);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = now.rstd * __builtin_fmaf(-c, s[j], t[j]);
        d[j] = a.d_sum ? d[j] + x : x;
      }
      pass8((PT_GLOBAL uint16_t*)a.d_x + r * a.d_x_stride, at + p * R::STEP, a.width, encode8<DT>(d));
    }
  }
  if (!a.part) return;
  PT_GLOBAL float* part = (PT_GLOBAL float*)a.part + first * a.pitch;
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const uint32_t c = at + p * R::STEP;
    if (c < a.pitch) {                                     // pitch is a multiple of eight
      *(PT_GLOBAL f32x4*)(part + c) = f32x4{dg[p][0], dg[p][1], dg[p][2], dg[p][3]};
      *(PT_GLOBAL f32x4*)(part + c + 4) = f32x4{dg[p][4], dg[p][5], dg[p][6], dg[p][7]};
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(256) k_rms_gain(const float* part, uint32_t rows, uint64_t pitch, uint32_t width, uint16_t* out) {
  add_columns<DT>(part, rows, pitch, width, out, blockIdx.x);
}

struct Rows8Args {
  const void* x;
  uint8_t* codes;
  float* scale;
  uint64_t x_stride, codes_stride;
  uint32_t rows, width;
};

typedef f32x4 f32x4_a __attribute__((aligned(4)));

template <int TYPE, int WAVES, int PIECES>
__global__ void __launch_bounds__(Rows<WAVES>::THREADS) k_rows8(const Rows8Args a) {
  typedef Rows<WAVES> R;
  __shared__ uint32_t s_big[WAVES];
  const uint32_t r = R::first(), at = R::lane_at();
  if (r >= a.rows) return;
  float v[PIECES][8];
  if constexpr (TYPE == PT_FP32) {
    const PT_GLOBAL float* x = (const PT_GLOBAL float*)a.x + r * a.x_stride;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const uint32_t c = at + p * R::STEP;
      if (c + 8 <= a.width) {
        const f32x4 lo = *(const PT_GLOBAL f32x4_a*)(x + c), hi = *(const PT_GLOBAL f32x4_a*)(x + c + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[p][j] = lo[j]; v[p][4 + j] = hi[j]; }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[p][j] = c + j < a.width ? x[c + j] : 0.0f;
      }
    }
  } else {
    const PT_GLOBAL uint16_t* x = (const PT_GLOBAL uint16_t*)a.x + r * a.x_stride;
    u32x4 q[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) q[p] = fetch8(x, at + p * R::STEP, a.width);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) decode8<TYPE>(place8(q[p], at + p * R::STEP, a.width), v[p]);
  }
  uint32_t big = 0;
#pragma unroll
  for (int p = 0; p < PIECES; ++p)
#pragma unroll
    for (int j = 0; j < 8; ++j) big = max(big, __float_as_uint(v[p][j]) & 0x7fffffffu);
  const Scale8 s = scale8(row_max<WAVES>(big, s_big));
#pragma unroll
  for (int p = 0; p < PIECES; ++p) pass8b((PT_GLOBAL uint8_t*)a.codes + r * a.codes_stride, at + p * R::STEP, a.width, codes8(v[p], s.inv));
  if (at == 0) ((PT_GLOBAL float*)a.scale)[r] = s.scale;
}

// ---- host -----------------------------------------------------------------------------------------------

// f: called with the waves that share a row of `width` and a lane's pieces of it, as constants: as few waves as 32 elements a lane allow (by_width_grads, where
// sums over the rows are kept too: as the registers do), and no more idle lanes than that makes.
template <int W, int P, class F> int with(F&& f) { return f(std::integral_constant<int, W>{}, std::integral_constant<int, P>{}); }
template <class F> int by_width(uint32_t width, F&& f) {
  if (width <= 512) return with<1, 1>(f);
  if (width <= 1024) return with<1, 2>(f);
  if (width <= 1536) return with<1, 3>(f);
  if (width <= 2048) return with<1, 4>(f);
  if (width <= 4096) return with<4, 2>(f);
  if (width <= 6144) return with<4, 3>(f);
  if (width <= 8192) return with<4, 4>(f);
  if (width <= 16384) return with<16, 2>(f);
  return with<16, 4>(f);
}
template <class F> int by_width_grads(uint32_t width, F&& f) {
  if (width <= 512) return with<1, 1>(f);
  if (width <= 1024) return with<1, 2>(f);
  if (width <= 2048) return with<4, 1>(f);
  if (width <= 4096) return with<4, 2>(f);
  if (width <= 6144) return with<4, 3>(f);
  if (width <= 8192) return with<8, 2>(f);
  if (width <= 16384) return with<8, 4>(f);
  return with<16, 4>(f);
}
template <int WAVES> uint32_t grid_of(uint32_t rows) { return (rows + Rows<WAVES>::PER - 1) / Rows<WAVES>::PER; }

// Workgroups of the gradients: as many as run at a time, each with a row of partial sums of the gain's gradient for every row it works on at a time.  (8192 x 4096 by 512
// 53.2 us, 256 63.1, 768 61.8; 8192 x 1600 by 512 26.9, 256 40.3; 2048 x 16384 by 256 72.3, 512 82.9, 1024 104.5.)
template <int WAVES> uint32_t grads_grid(uint32_t rows, uint32_t width) { return std::min(grid_of<WAVES>(rows), width > 8192 ? 256u : 512u); }
uint64_t grads_bytes(const pt_rms& n) {
  uint64_t bytes = 0;
  if (n.d_gain && n.rows)
    by_width_grads(n.width, [&](auto w, auto) { bytes = 4ull * grads_grid<w()>(n.rows, n.width) * Rows<w()>::PER * up(n.width, 8); return PT_OK; });
  return bytes;
}

template <int DT> int norm_rows(const NormArgs& a, hipStream_t st) {
  return by_width(a.width, [&](auto w, auto p) {
    constexpr uint32_t TWO_A_UNIT = 512;
    const uint32_t grid = grid_of<w()>(a.rows);
    if constexpr (w() == 4) {
      if (a.y_scale && grid >= 8 * TWO_A_UNIT) {
        hipLaunchKernelGGL((k_rms<DT, w(), p(), true>), dim3(TWO_A_UNIT), dim3(Rows<w()>::THREADS), 0, st, a);
        PT_LAUNCH_CHECK(nullptr, "k_rms");
        return int(PT_OK);
      }
    }
    hipLaunchKernelGGL((k_rms<DT, w(), p(), false>), dim3(grid), dim3(Rows<w()>::THREADS), 0, st, a);
    PT_LAUNCH_CHECK(nullptr, "k_rms");
    return int(PT_OK);
  });
}

int check(const pt_rms* n, const char* who) {
  if (!n) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: norm is NULL", who);
  if (n->dtype != PT_BF16 && n->dtype != PT_FP16) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: dtype %d is neither PT_BF16 nor PT_FP16", who, n->dtype);
  if (!n->width) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: width must be > 0", who);
  if (!(n->eps >= 0.0 && n->eps <= double(FLT_MAX))) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: eps is not >= 0 and in fp32's range", who);
  const struct { const void* at; uint64_t stride; } rows[] = {{n->x, n->x_stride}, {n->residual, n->residual_stride}, {n->sum, n->sum_stride},
    {n->y, n->y_stride}, {n->d_y, n->d_y_stride}, {n->d_sum, n->d_sum_stride}, {n->d_x, n->d_x_stride}};
  for (const auto& x : rows)
    if (x.at && x.stride < n->width) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: rows of width %u at a smaller stride", who, n->width);
  if (((uintptr_t)n->x | (uintptr_t)n->residual | (uintptr_t)n->gain | (uintptr_t)n->sum | (uintptr_t)n->d_y | (uintptr_t)n->d_sum | (uintptr_t)n->d_x |
       (uintptr_t)n->d_gain | (n->y_scale ? 0 : (uintptr_t)n->y)) % 2 != 0 || ((uintptr_t)n->rstd | (uintptr_t)n->y_scale) % 4 != 0)
    return pt_fail(nullptr, PT_ERR_ALIGNMENT, "%s: an array is not aligned to its elements", who);
  if (n->width > MOST_WIDTH || n->rows > (1u << 30)) return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "%s: a width over %u or more than 2^30 rows", who, MOST_WIDTH);
  return PT_OK;
}

}  // namespace

extern "C" int pt_rms_workspace(const pt_rms* norm, uint64_t* bytes) {
  if (int rc = check(norm, "pt_rms_workspace"); rc != PT_OK) return rc;
  if (bytes) *bytes = grads_bytes(*norm);
  return PT_OK;
}

extern "C" int pt_rms_norm(const pt_rms* n, void* stream) {
  if (int rc = check(n, "pt_rms_norm"); rc != PT_OK) return rc;
  if (!n->rows) return PT_OK;
  if (!n->x || !n->y) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rms_norm: NULL array");
  const float eps = n->eps > 0.0 ? std::max(float(n->eps), FLT_TRUE_MIN) : 0.0f;       // above 0 stays above 0: rows of zeros
  for (uint64_t r = 0; r < n->rows; r += MOST_ROWS) {
    const auto row = [&](const void* x, uint64_t stride) { return x ? (uint16_t*)x + r * stride : nullptr; };
    const NormArgs a = {row(n->x, n->x_stride), row(n->residual, n->residual_stride), (const uint16_t*)n->gain, row(n->sum, n->sum_stride),
                        n->rstd ? n->rstd + r : nullptr, n->y_scale ? (void*)((uint8_t*)n->y + r * n->y_stride) : row(n->y, n->y_stride),
                        n->y_scale ? n->y_scale + r : nullptr, n->x_stride, n->residual_stride, n->sum_stride, n->y_stride, eps,
                        1.0f / float(n->width), uint32_t(std::min<uint64_t>(MOST_ROWS, n->rows - r)), n->width};
    if (int rc = n->dtype == PT_BF16 ? norm_rows<PT_BF16>(a, (hipStream_t)stream) : norm_rows<PT_FP16>(a, (hipStream_t)stream); rc != PT_OK) return rc;
  }
  return PT_OK;
}

extern "C" int pt_rms_grads(const pt_rms* n, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (int rc = check(n, "pt_rms_grads"); rc != PT_OK) return rc;
  const void* sum = n->sum ? n->sum : n->x;
  if (n->rows && (!sum || !n->rstd || !n->d_y)) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rms_grads: NULL array");
  if (n->rows && !n->sum && n->residual) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rms_grads: with a residual the sum is needed");
  if (!n->d_x && !n->d_gain) return PT_OK;
  const uint64_t bytes = grads_bytes(*n);
  if (bytes && !workspace) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rms_grads: workspace is NULL");
  if (bytes && (uintptr_t)workspace % 256 != 0) return pt_fail(nullptr, PT_ERR_ALIGNMENT, "pt_rms_grads: the workspace is not 256-byte aligned");
  if (bytes > workspace_bytes)
    return pt_fail(nullptr, PT_ERR_NOMEM, "pt_rms_grads: a workspace of %llu bytes is too small (pt_rms_workspace)", (unsigned long long)workspace_bytes);
  hipStream_t st = (hipStream_t)stream;
  return by_width_grads(n->width, [&](auto w, auto p) {
    typedef Rows<w()> R;
    const uint32_t grid = grads_grid<w()>(n->rows, n->width), part_rows = grid * R::PER;
    const uint64_t pitch = up(n->width, 8);
    const GradArgs a = {(const uint16_t*)sum, (const uint16_t*)n->gain, (const uint16_t*)n->d_y, (const uint16_t*)n->d_sum, n->rstd, (uint16_t*)n->d_x,
                        n->d_gain ? (float*)workspace : nullptr, n->sum ? n->sum_stride : n->x_stride, n->d_y_stride, n->d_sum_stride, n->d_x_stride, pitch,
                        1.0f / float(n->width), n->rows, n->width, part_rows};
    if (grid) {
      if (n->dtype == PT_BF16) hipLaunchKernelGGL((k_rms_grads<PT_BF16, w(), p()>), dim3(grid), dim3(R::THREADS), 0, st, a);
      else hipLaunchKernelGGL((k_rms_grads<PT_FP16, w(), p()>), dim3(grid), dim3(R::THREADS), 0, st, a);
      PT_LAUNCH_CHECK(nullptr, "k_rms_grads");
    }
    if (!n->d_gain) return int(PT_OK);
    const dim3 columns(column_blocks(n->width));
    if (n->dtype == PT_BF16) hipLaunchKernelGGL(k_rms_gain<PT_BF16>, columns, dim3(256), 0, st, a.part, part_rows, pitch, n->width, (uint16_t*)n->d_gain);
    else hipLaunchKernelGGL(k_rms_gain<PT_FP16>, columns, dim3(256), 0, st, a.part, part_rows, pitch, n->width, (uint16_t*)n->d_gain);
    PT_LAUNCH_CHECK(nullptr, "k_rms_gain");
    return int(PT_OK);
  });
}

extern "C" int pt_rows8(const pt_rows* d, void* stream) {
  if (!d) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rows8: rows is NULL");
  if (d->type != PT_BF16 && d->type != PT_FP16 && d->type != PT_FP32)
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rows8: type %d is none of PT_BF16, PT_FP16, PT_FP32", d->type);
  if (!d->width) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rows8: width must be > 0");
  if (d->rows && (!d->x || !d->codes || !d->scale)) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rows8: NULL array");
  if (d->x_stride < d->width || d->codes_stride < d->width)
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_rows8: rows of width %u at a smaller stride", d->width);
  if ((uintptr_t)d->x % (d->type == PT_FP32 ? 4 : 2) != 0 || (uintptr_t)d->scale % 4 != 0)
    return pt_fail(nullptr, PT_ERR_ALIGNMENT, "pt_rows8: an array is not aligned to its elements");
  if (d->width > MOST_WIDTH || d->rows > (1u << 30)) return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "pt_rows8: a width over %u or more than 2^30 rows", MOST_WIDTH);
  if (!d->rows) return PT_OK;
  for (uint64_t r = 0; r < d->rows; r += MOST_ROWS) {
    const Rows8Args a = {(const char*)d->x + r * d->x_stride * (d->type == PT_FP32 ? 4 : 2), (uint8_t*)d->codes + r * d->codes_stride, d->scale + r, d->x_stride,
                         d->codes_stride, uint32_t(std::min<uint64_t>(MOST_ROWS, d->rows - r)), d->width};
    const int rc = by_width(d->width, [&](auto w, auto p) {
      const dim3 grid(grid_of<w()>(a.rows)), block(Rows<w()>::THREADS);
      if (d->type == PT_BF16) hipLaunchKernelGGL((k_rows8<PT_BF16, w(), p()>), grid, block, 0, (hipStream_t)stream, a);
      else if (d->type == PT_FP16) hipLaunchKernelGGL((k_rows8<PT_FP16, w(), p()>), grid, block, 0, (hipStream_t)stream, a);
      else hipLaunchKernelGGL((k_rows8<PT_FP32, w(), p()>), grid, block, 0, (hipStream_t)stream, a);
      PT_LAUNCH_CHECK(nullptr, "k_rows8");
      return int(PT_OK);
    });
    if (rc != PT_OK) return rc;
  }
  return PT_OK;
}
