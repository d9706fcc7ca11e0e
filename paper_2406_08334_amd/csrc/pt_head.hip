// Loss of a language model's head: softmax cross entropy from hidden states and weight, with gradients, logits of a piece of the rows at a time.
//
//   rows     the rows with a target, counted and listed on the device (ignored ones take no part in anything that follows)
//   gather   their hidden states next to each other, zero-padded to whole steps of the products
//   logits   z = W h^T on the matrix cores, tile by tile; of each tile the largest z and the sum of exp(z - that) of every row, and, for gradients, z in fp32
//   soft     from the tiles' sums lse and loss of a row; G = s (exp(z - lse) - [target]) in 16 bits over the row's z, in place
//   d_hidden = G W, d_weight = G^T h on the matrix cores
//
// Three products of 2 rows vocab width operations each are what it costs.  Gradients want lse of a whole row before the first of them: pieces of the
// vocabulary would take the first product twice, so the pieces are rows, of which as many are taken at a time as the workspace has room for.
// The loss alone never stores a logit.
#include "pt_common.h"
#include "pt_mfma.h"
#include "pt_update.h"

#include <algorithm>

using namespace pt_mfma;

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a __attribute__((aligned(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t PIECE_STEP = 256;       // pieces are multiples of this many rows
constexpr uint32_t PIECE_BEST = 8192;
constexpr float LOG2E = 1.44269504088896340736f;

// What the device finds out about the rows.
struct Meta {
  uint32_t count;            // rows with a target
  float up, down;            // a power of two that G is multiplied by before it is rounded to 16 bits, and 1 / it: the largest |G| becomes 2^13 to 2^14
};

struct Shape {
  uint32_t R, V, d;
  uint32_t Kd, Vp;           // width and vocabulary rounded up to whole steps and tiles
};

// ---- rows ---------------------------------------------------------------------------------------------

// One workgroup lists the rows that have a target, in order.
__global__ void __launch_bounds__(1024) k_head_rows(const int64_t* __restrict__ target, const float* __restrict__ scale, Shape s, Meta* __restrict__ meta,
                                                    uint32_t* __restrict__ row_of, uint32_t* __restrict__ target_of) {
  __shared__ uint32_t s_n[16];
  __shared__ float s_big[16];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t n = 0;
  float big = 0.0f;
  for (uint32_t r0 = 0; r0 < s.R; r0 += 1024) {
    const uint32_t r = r0 + threadIdx.x;
    const int64_t y = r < s.R ? target[r] : -1;
    const bool has = uint64_t(y) < s.V;
    if (has) big = fmaxf(big, scale ? __builtin_fabsf(scale[r]) : 1.0f);
    const uint64_t mask = __ballot(has);
    if (lane == 0) s_n[wave] = uint32_t(__popcll(mask));
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (uint32_t w = 0; w < 16; ++w) { const uint32_t k = s_n[w]; before += w < wave ? k : 0; all += k; }
    if (has) {
      const uint32_t at = n + before + uint32_t(__popcll(mask & ((uint64_t(1) << lane) - 1)));
      row_of[at] = r;
      target_of[at] = uint32_t(y);
    }
    n += all;
    __syncthreads();
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) big = fmaxf(big, __shfl_xor(big, off, 64));
  if (lane == 0) s_big[wave] = big;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int w = 1; w < 16; ++w) big = fmaxf(big, s_big[w]);
  int e = 0;
  if (big > 0.0f && big < 3.4e38f) (void)frexpf(big, &e);       // big < 2^e
  e = max(-100, min(100, 14 - e));
  *meta = {n, ldexpf(1.0f, e), ldexpf(1.0f, -e)};
}

// One row of 16-bit words, at any address, into one of Kd words that begins at a multiple of 16 bytes; zero behind its end.
__device__ __forceinline__ void copy_row(const PT_GLOBAL uint16_t* from, PT_GLOBAL uint16_t* to, uint32_t d, uint32_t Kd, uint32_t lane, uint32_t lanes) {
  for (uint32_t c = lane * 8; c < Kd; c += lanes * 8) {
    u32x4 q = {0, 0, 0, 0};
    if (c + 8 <= d) q = *(const PT_GLOBAL u32x4_a*)(from + c);
    else
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j)
        if (c + j < d) q[j / 2] |= uint32_t(from[c + j]) << (16 * (j & 1));
    *(PT_GLOBAL u32x4*)(to + c) = q;
  }
}

// A wave a row: the hidden states of the rows with a target, zero rows up to a whole step behind them, and nothing for those without one.
__global__ void __launch_bounds__(256) k_head_gather(const uint16_t* __restrict__ hidden, uint64_t stride, const int64_t* __restrict__ target, Shape s,
                                                     const Meta* __restrict__ meta, const uint32_t* __restrict__ row_of, uint16_t* __restrict__ packed,
                                                     float* __restrict__ loss, uint16_t* __restrict__ d_hidden, uint64_t d_stride) {
  const uint32_t r = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const uint32_t n = meta->count;
  PT_GLOBAL uint16_t* to = (PT_GLOBAL uint16_t*)packed + size_t(r) * s.Kd;
  if (r < n) copy_row((const PT_GLOBAL uint16_t*)hidden + row_of[r] * stride, to, s.d, s.Kd, lane, 64);
  else if (r < (n + TWO - 1) / TWO * TWO) {
    for (uint32_t c = lane * 8; c < s.Kd; c += 512) *(PT_GLOBAL u32x4*)(to + c) = u32x4{0, 0, 0, 0};
  }
  if (r < s.R && uint64_t(target[r]) >= s.V) {
    if (lane == 0) loss[r] = 0.0f;
    if (d_hidden)
      for (uint32_t c = lane; c < s.d; c += 64) d_hidden[r * d_stride + c] = 0;
  }
}

// A weight whose rows do not all begin at multiples of 16 bytes.
__global__ void __launch_bounds__(256) k_head_weight(const uint16_t* __restrict__ weight, uint64_t stride, Shape s, uint16_t* __restrict__ padded) {
  const uint32_t v = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (v < s.V)
    copy_row((const PT_GLOBAL uint16_t*)weight + v * stride, (PT_GLOBAL uint16_t*)padded + size_t(v) * s.Kd, s.d, s.Kd, threadIdx.x & 63, 64);
}

__global__ void __launch_bounds__(256) k_head_zero(uint16_t* __restrict__ d_weight, uint64_t stride, Shape s) {
  for (uint32_t c = threadIdx.x; c < s.d; c += 256) d_weight[blockIdx.x * stride + c] = 0;
}

// ---- products ------------------------------------------------------------------------------------------

// Tile `id` of tm x tn: the XCDs, which workgroups go to in turn, get tiles next to each other, in patches of a few n.
__device__ __forceinline__ bool tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t& m, uint32_t& n) {
  constexpr uint32_t GROUP = 8;
  const uint32_t total = tm * tn, per = (total + 7) / 8, at = (id >> 3), i = (id & 7) * per + at;
  if (at >= per || i >= total) return false;
  const uint32_t g = i / (GROUP * tm), n0 = g * GROUP, gn = min(GROUP, tn - n0), r = i - g * GROUP * tm;
  n = n0 + r % gn;
  m = r / gn;
  return true;
}
inline uint32_t tile_grid(uint64_t tm, uint64_t tn) { return uint32_t((tm * tn + 7) / 8 * 8); }

// Rows of piece [first, first + rows) that have a target.
__device__ __forceinline__ uint32_t piece_rows(const Meta* meta, uint32_t first, uint32_t rows) {
  const uint32_t n = meta->count;
  return n > first ? min(rows, n - first) : 0;
}

struct LogitArgs {
  Shape s;
  Operand w, h;              // h: of the piece
  const Meta* meta;
  uint32_t first, rows;
  const uint32_t* target_of; // of the piece
  f32x2* part;               // [rows][parts] of the piece: largest z, sum of exp(z - largest)
  uint32_t parts;
  float* at_target;          // [rows]
  float* z;                  // [rows][Vp], or NULL
};

template <int DT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) k_head_logits(const LogitArgs a) {
  typedef Tile<DT, true, true, BM, BN, WM, WN> T;
  __shared__ __attribute__((aligned(16))) char even[T::BYTES], odd[T::BYTES];
  const uint32_t n_rows = piece_rows(a.meta, a.first, a.rows);
  uint32_t tm, tn;
  if (!tile_of(blockIdx.x, (a.s.V + BM - 1) / BM, (n_rows + BN - 1) / BN, tm, tn)) return;
  const uint32_t m0 = tm * BM, n0 = tn * BN;
  Operand h = a.h;
  h.extent = n_rows;
  T t;
  t.run((lds_char*)even, (lds_char*)odd, a.w, h, m0, n0, 0, a.s.Kd / TWO);
  const uint32_t lane = threadIdx.x & 63, mb = m0 + t.wave_m() + (lane >> 4) * 4;
  // of rows m behind the vocabulary there is nothing to sum
  if (m0 + BM > a.s.V) {
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (mb + i * 16 + q >= a.s.V)
#pragma unroll
          for (int j = 0; j < T::FN; ++j) t.acc[i][j][q] = -__builtin_inff();
  }
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const uint32_t n = n0 + t.wave_n() + j * 16 + (lane & 15);
    const bool live = n < n_rows;
    float big = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) big = fmaxf(big, t.acc[i][j][q]);
    big = fmaxf(big, __shfl_xor(big, 16, 64));
    big = fmaxf(big, __shfl_xor(big, 32, 64));
    const float top = big == -__builtin_inff() ? 0.0f : big;          // of nothing but -inf the sum is 0
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) sum += __builtin_amdgcn_exp2f((t.acc[i][j][q] - top) * LOG2E);
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (live && lane < 16) a.part[size_t(n) * a.parts + tm * WM + t.wave_m() / T::TM] = f32x2{big, sum};
    const uint32_t y = live ? a.target_of[n] - mb : ~0u;              // the lane's z are mb + 16 i + q
    float zy = 0.0f;
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) zy = y == uint32_t(i * 16 + q) ? t.acc[i][j][q] : zy;
    if (y < uint32_t(T::TM) && (y & 15) < 4) a.at_target[n] = zy;
    if (a.z && live)
#pragma unroll
      for (int i = 0; i < T::FM; ++i) *(PT_GLOBAL f32x4*)((PT_GLOBAL float*)a.z + size_t(n) * a.s.Vp + mb + i * 16) = t.acc[i][j];
  }
}

// lse of a row from its tiles' sums, by `lanes` lanes of which this is `lane`; in all of them.
__device__ __forceinline__ f32x2 join(f32x2 a, f32x2 b) {
  const float top = fmaxf(a[0], b[0]);
  if (top == -__builtin_inff()) return f32x2{top, a[1] + b[1]};
  return f32x2{top, a[1] * __builtin_amdgcn_exp2f((a[0] - top) * LOG2E) + b[1] * __builtin_amdgcn_exp2f((b[0] - top) * LOG2E)};
}
__device__ __forceinline__ f32x2 join_wave(f32x2 x) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) x = join(x, f32x2{__shfl_xor(x[0], off, 64), __shfl_xor(x[1], off, 64)});
  return x;
}

struct SoftArgs {
  Shape s;
  const Meta* meta;
  uint32_t first, rows;
  const uint32_t *row_of, *target_of;      // of the piece
  const f32x2* part;
  uint32_t parts;
  const float* at_target;
  const float* scale;
  float* loss;
  float* z;
};

// The loss alone: a wave a row.
__global__ void __launch_bounds__(256) k_head_loss(const SoftArgs a) {
  const uint32_t r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= piece_rows(a.meta, a.first, a.rows)) return;
  f32x2 x = {-__builtin_inff(), 0.0f};
  for (uint32_t i = lane; i < a.parts; i += 64) x = join(x, a.part[size_t(r) * a.parts + i]);
  x = join_wave(x);
  if (lane == 0) a.loss[a.row_of[r]] = x[0] + logf(x[1]) - a.at_target[r];
}

// Loss and G of a row by a workgroup: the row's z lie where its G goes, which is half as long.
template <int DT>
__global__ void __launch_bounds__(256) k_head_soft(const SoftArgs a) {
  const uint32_t r = blockIdx.x, tid = threadIdx.x, n = piece_rows(a.meta, a.first, a.rows);
  if (r >= (n + TWO - 1) / TWO * TWO) return;
  PT_GLOBAL float* z = (PT_GLOBAL float*)a.z + size_t(r) * a.s.Vp;
  PT_GLOBAL uint16_t* g = (PT_GLOBAL uint16_t*)z;
  if (r >= n) {                                            // rows up to a whole step: zero
    for (uint32_t c = tid * 8; c < a.s.Vp; c += 2048) *(PT_GLOBAL u32x4*)(g + c) = u32x4{0, 0, 0, 0};
    return;
  }
  __shared__ f32x2 s_x[4];
  f32x2 x = {-__builtin_inff(), 0.0f};
  for (uint32_t i = tid; i < a.parts; i += 256) x = join(x, a.part[size_t(r) * a.parts + i]);
  x = join_wave(x);
  if ((tid & 63) == 0) s_x[tid >> 6] = x;
  __syncthreads();
  x = join(join(s_x[0], s_x[1]), join(s_x[2], s_x[3]));
  const uint32_t row = a.row_of[r], y = a.target_of[r];
  const float zy = a.at_target[r], lse = x[0] + logf(x[1]), s = (a.scale ? a.scale[row] : 1.0f) * a.meta->up;
  if (tid == 0) a.loss[row] = lse - zy;
  const float off = lse * LOG2E, gy = s * expm1f(zy - lse);
  for (uint32_t c0 = 0; c0 < a.s.Vp; c0 += 2048) {
    const uint32_t c = c0 + tid * 8;
    f32x4 q[2] = {};
    if (c < a.s.Vp) { q[0] = *(PT_GLOBAL f32x4*)(z + c); q[1] = *(PT_GLOBAL f32x4*)(z + c + 4); }
    uint32_t w[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      float p = s * __builtin_amdgcn_exp2f(__builtin_fmaf(q[j / 4][j % 4], LOG2E, -off));
      if (c + j == y) p = gy;
      w[j] = c + j < a.s.V ? encode16<DT>(p) : 0u;
    }
    __syncthreads();                                       // every lane has its z of this round and of those before
    if (c < a.s.Vp) *(PT_GLOBAL u32x4*)(g + c) = u32x4{w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16};
  }
}

// Four values of consecutive m of a row that has d of them.
template <int DT>
__device__ __forceinline__ void store4(PT_GLOBAL uint16_t* row, uint32_t m, uint32_t d, bool wide, f32x4 x) {
  const uint32_t w[4] = {encode16<DT>(x[0]), encode16<DT>(x[1]), encode16<DT>(x[2]), encode16<DT>(x[3])};
  if (wide && m + 4 <= d) *(PT_GLOBAL u32x2*)(row + m) = u32x2{w[0] | w[1] << 16, w[2] | w[3] << 16};
  else
#pragma unroll
    for (uint32_t q = 0; q < 4; ++q)
      if (m + q < d) row[m + q] = uint16_t(w[q]);
}

struct GradArgs {
  Shape s;
  Operand p, q;
  const Meta* meta;
  uint32_t first, rows;
  const uint32_t* row_of;    // of the piece
  uint16_t* out;
  uint64_t stride;
  bool wide;                 // four results may be stored at once
  float* acc;                // d_weight over several pieces: sums so far [V][pitch]
  uint32_t pitch;
  bool read_acc, write_acc;
};

// d_hidden of a piece: m runs over the width, n over rows, k over the vocabulary.
template <int DT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) k_head_d_hidden(const GradArgs a) {
  typedef Tile<DT, false, true, BM, BN, WM, WN> T;
  __shared__ __attribute__((aligned(16))) char even[T::BYTES], odd[T::BYTES];
  const uint32_t n_rows = piece_rows(a.meta, a.first, a.rows);
  uint32_t tm, tn;
  if (!tile_of(blockIdx.x, (a.s.d + BM - 1) / BM, (n_rows + BN - 1) / BN, tm, tn)) return;
  Operand q = a.q;
  q.extent = n_rows;
  T t;
  t.run((lds_char*)even, (lds_char*)odd, a.p, q, tm * BM, tn * BN, 0, a.s.Vp / TWO);
  const uint32_t lane = threadIdx.x & 63, mb = tm * BM + t.wave_m() + (lane >> 4) * 4;
  const float down = a.meta->down;
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const uint32_t n = tn * BN + t.wave_n() + j * 16 + (lane & 15);
    if (n >= n_rows) continue;
    PT_GLOBAL uint16_t* row = (PT_GLOBAL uint16_t*)a.out + a.row_of[n] * a.stride;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) store4<DT>(row, mb + i * 16, a.s.d, a.wide, t.acc[i][j] * down);
  }
}

// d_weight: m runs over the width, n over the vocabulary, k over the piece's rows.
template <int DT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN) k_head_d_weight(const GradArgs a) {
  typedef Tile<DT, false, false, BM, BN, WM, WN> T;
  __shared__ __attribute__((aligned(16))) char even[T::BYTES], odd[T::BYTES];
  const uint32_t n_rows = piece_rows(a.meta, a.first, a.rows);
  if (!n_rows && a.read_acc && a.write_acc) return;
  uint32_t tm, tn;
  if (!tile_of(blockIdx.x, (a.s.d + BM - 1) / BM, (a.s.V + BN - 1) / BN, tm, tn)) return;
  Operand p = a.p, q = a.q;
  p.k = q.k = (n_rows + TWO - 1) / TWO * TWO;
  T t;
  t.run((lds_char*)even, (lds_char*)odd, p, q, tm * BM, tn * BN, 0, p.k / TWO);
  const uint32_t lane = threadIdx.x & 63, mb = tm * BM + t.wave_m() + (lane >> 4) * 4;
  const float down = a.meta->down;
#pragma unroll
  for (int j = 0; j < T::FN; ++j) {
    const uint32_t n = tn * BN + t.wave_n() + j * 16 + (lane & 15);
    if (n >= a.s.V) continue;
    PT_GLOBAL uint16_t* row = (PT_GLOBAL uint16_t*)a.out + n * a.stride;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) {
      const uint32_t m = mb + i * 16;
      if (m >= a.s.d) continue;
      f32x4 x = t.acc[i][j] * down;
      PT_GLOBAL f32x4* sum = (PT_GLOBAL f32x4*)((PT_GLOBAL float*)a.acc + size_t(n) * a.pitch + m);
      if (a.read_acc) x += *sum;
      if (a.write_acc) *sum = x;
      else store4<DT>(row, m, a.s.d, a.wide, x);
    }
  }
}

// ---- host -----------------------------------------------------------------------------------------------

constexpr uint32_t BM = 256, BN = 256, WM = 2, WN = 4, THREADS = 64 * WM * WN;

uint64_t up(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }

// Where everything lies in the workspace, for pieces of `rows` rows.
struct Plan {
  Shape s;
  uint32_t parts, pitch, pieces, rows;
  bool grads, direct;                      // direct: the weight is taken where it lies
  uint64_t meta, row_of, target_of, at_target, packed, weight, part, z, acc, total;
};

Plan make_plan(const pt_head& h, uint64_t rows) {
  Plan p{};
  p.s = {h.rows, h.vocab, h.width, uint32_t(up(h.width, TWO)), uint32_t(up(h.vocab, BM))};
  p.grads = h.d_hidden || h.d_weight;
  p.direct = h.width % BK == 0 && h.weight_stride % 8 == 0 && (uintptr_t)h.weight % 16 == 0;
  p.parts = p.s.Vp / BM * WM;
  p.pitch = uint32_t(up(h.width, 4));
  p.rows = uint32_t(std::min<uint64_t>(rows, up(h.rows, PIECE_STEP)));
  p.pieces = (h.rows + p.rows - 1) / p.rows;
  p.rows = uint32_t(up((h.rows + p.pieces - 1) / p.pieces, PIECE_STEP));       // of one size
  p.pieces = (h.rows + p.rows - 1) / p.rows;
  uint64_t at = 0;
  const auto take = [&](uint64_t bytes) { const uint64_t x = at; at += up(bytes, 256); return x; };
  p.meta = take(sizeof(Meta));
  p.row_of = take(4ull * h.rows);
  p.target_of = take(4ull * h.rows);
  p.at_target = take(4ull * p.rows);
  p.packed = take(2ull * up(h.rows, TWO) * p.s.Kd);
  p.weight = take(p.direct ? 0 : 2ull * h.vocab * p.s.Kd);
  p.part = take(8ull * p.rows * p.parts);
  p.z = take(p.grads ? 4ull * p.rows * p.s.Vp : 0);
  p.acc = take(h.d_weight && p.pieces > 1 ? 4ull * h.vocab * p.pitch : 0);
  p.total = at;
  return p;
}

int check(const pt_head* h, const char* who) {
  if (!h) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: head is NULL", who);
  if (h->dtype != PT_BF16 && h->dtype != PT_FP16)
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: dtype %d is neither PT_BF16 nor PT_FP16", who, h->dtype);
  if (!h->vocab || !h->width) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: vocab and width must be > 0", who);
  if (!h->weight || (h->rows && (!h->hidden || !h->target || !h->loss))) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: NULL array", who);
  if (h->hidden_stride < h->width || h->weight_stride < h->width || (h->d_hidden && h->d_hidden_stride < h->width) ||
      (h->d_weight && h->d_weight_stride < h->width))
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: rows of width %u at a smaller stride", who, h->width);
  if (((uintptr_t)h->hidden | (uintptr_t)h->weight | (uintptr_t)h->d_hidden | (uintptr_t)h->d_weight) % 2 != 0 ||
      ((uintptr_t)h->row_scale | (uintptr_t)h->loss) % 4 != 0 || (uintptr_t)h->target % 8 != 0)
    return pt_fail(nullptr, PT_ERR_ALIGNMENT, "%s: an array is not aligned to its elements", who);
  // a step's loads reach 256 rows or 64 from a 64-bit address on by 32-bit offsets
  if (h->rows > (1u << 30) || h->vocab > (1u << 21) || h->width > (1u << 20) || h->weight_stride > (1u << 21))
    return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "%s: more than 2^30 rows, 2^21 words, a width over 2^20 or a weight stride over 2^21", who);
  return PT_OK;
}

template <int DT>
int run(const pt_head& h, const Plan& p, char* ws, hipStream_t st) {
  const Shape& s = p.s;
  Meta* meta = (Meta*)(ws + p.meta);
  uint32_t *row_of = (uint32_t*)(ws + p.row_of), *target_of = (uint32_t*)(ws + p.target_of);
  uint16_t* packed = (uint16_t*)(ws + p.packed);
  hipLaunchKernelGGL(k_head_rows, dim3(1), dim3(1024), 0, st, h.target, h.row_scale, s, meta, row_of, target_of);
  PT_LAUNCH_CHECK(nullptr, "k_head_rows");
  hipLaunchKernelGGL(k_head_gather, dim3(uint32_t(up(s.R, TWO) / 4)), dim3(256), 0, st, (const uint16_t*)h.hidden, h.hidden_stride, h.target, s, meta,
                     row_of, packed, h.loss, (uint16_t*)h.d_hidden, h.d_hidden_stride);
  PT_LAUNCH_CHECK(nullptr, "k_head_gather");
  Operand w = {h.weight, h.weight_stride * 2, 0, 0};
  if (!p.direct) {
    hipLaunchKernelGGL(k_head_weight, dim3((s.V + 3) / 4), dim3(256), 0, st, (const uint16_t*)h.weight, h.weight_stride, s, (uint16_t*)(ws + p.weight));
    PT_LAUNCH_CHECK(nullptr, "k_head_weight");
    w.at = ws + p.weight;
    w.pitch = 2ull * s.Kd;
  }
  const uint32_t wide_k = p.direct ? s.d : s.Kd;            // of a row of the weight that may be read
  for (uint32_t i = 0; i < p.pieces; ++i) {
    const uint32_t first = i * p.rows, rows = std::min(p.rows, s.R - first);
    const Operand hid = {packed + size_t(first) * s.Kd, 2ull * s.Kd, 0, s.Kd};
    Operand wk = w;
    wk.extent = s.V;
    wk.k = wide_k;
    const LogitArgs la = {s, wk, hid, meta, first, rows, target_of + first, (f32x2*)(ws + p.part), p.parts, (float*)(ws + p.at_target),
                          p.grads ? (float*)(ws + p.z) : nullptr};
    hipLaunchKernelGGL((k_head_logits<DT, BM, BN, WM, WN>), dim3(tile_grid((s.V + BM - 1) / BM, (rows + BN - 1) / BN)), dim3(THREADS), 0, st, la);
    PT_LAUNCH_CHECK(nullptr, "k_head_logits");
    const SoftArgs sa = {s, meta, first, rows, row_of + first, target_of + first, (const f32x2*)(ws + p.part), p.parts,
                         (const float*)(ws + p.at_target), h.row_scale, h.loss, (float*)(ws + p.z)};
    if (!p.grads) {
      hipLaunchKernelGGL(k_head_loss, dim3((rows + 3) / 4), dim3(256), 0, st, sa);
      PT_LAUNCH_CHECK(nullptr, "k_head_loss");
      continue;
    }
    hipLaunchKernelGGL(k_head_soft<DT>, dim3(uint32_t(up(rows, TWO))), dim3(256), 0, st, sa);
    PT_LAUNCH_CHECK(nullptr, "k_head_soft");
    const uint64_t z_pitch = 4ull * s.Vp;
    if (h.d_hidden) {
      Operand wm = w;
      wm.extent = wide_k;
      wm.k = s.V;
      const GradArgs ga = {s, wm, {ws + p.z, z_pitch, 0, s.Vp}, meta, first, rows, row_of + first, (uint16_t*)h.d_hidden, h.d_hidden_stride,
                           (uintptr_t)h.d_hidden % 8 == 0 && h.d_hidden_stride % 4 == 0, nullptr, 0, false, false};
      hipLaunchKernelGGL((k_head_d_hidden<DT, BM, BN, WM, WN>), dim3(tile_grid((s.d + BM - 1) / BM, (rows + BN - 1) / BN)), dim3(THREADS), 0, st, ga);
      PT_LAUNCH_CHECK(nullptr, "k_head_d_hidden");
    }
    if (h.d_weight) {
      Operand hm = hid;
      hm.extent = s.Kd;
      const GradArgs ga = {s, hm, {ws + p.z, z_pitch, s.Vp, 0}, meta, first, rows, nullptr, (uint16_t*)h.d_weight, h.d_weight_stride,
                           (uintptr_t)h.d_weight % 8 == 0 && h.d_weight_stride % 4 == 0, (float*)(ws + p.acc), p.pitch, i > 0, i + 1 < p.pieces};
      hipLaunchKernelGGL((k_head_d_weight<DT, BM, BN, WM, WN>), dim3(tile_grid((s.d + BM - 1) / BM, (s.V + BN - 1) / BN)), dim3(THREADS), 0, st, ga);
      PT_LAUNCH_CHECK(nullptr, "k_head_d_weight");
    }
  }
  return PT_OK;
}

}  // namespace

extern "C" int pt_head_workspace(const pt_head* head, uint64_t* least_bytes, uint64_t* best_bytes) {
  if (int rc = check(head, "pt_head_workspace"); rc != PT_OK) return rc;
  if (least_bytes) *least_bytes = head->rows ? make_plan(*head, PIECE_STEP).total : 0;
  if (best_bytes) *best_bytes = head->rows ? make_plan(*head, PIECE_BEST).total : 0;
  return PT_OK;
}

extern "C" int pt_head_loss(const pt_head* head, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (int rc = check(head, "pt_head_loss"); rc != PT_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (!head->rows) {
    if (!head->d_weight) return PT_OK;
    hipLaunchKernelGGL(k_head_zero, dim3(head->vocab), dim3(256), 0, st, (uint16_t*)head->d_weight, head->d_weight_stride,
                       Shape{0, head->vocab, head->width, 0, 0});
    PT_LAUNCH_CHECK(nullptr, "k_head_zero");
    return PT_OK;
  }
  if (!workspace) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_head_loss: workspace is NULL");
  if ((uintptr_t)workspace % 256 != 0) return pt_fail(nullptr, PT_ERR_ALIGNMENT, "pt_head_loss: the workspace is not 256-byte aligned");
  // the largest pieces that fit
  uint64_t rows = PIECE_BEST;
  while (rows > PIECE_STEP && make_plan(*head, rows).total > workspace_bytes) rows -= PIECE_STEP;
  const Plan p = make_plan(*head, rows);
  if (p.total > workspace_bytes)
    return pt_fail(nullptr, PT_ERR_NOMEM, "pt_head_loss: a workspace of %llu bytes, at least %llu are needed", (unsigned long long)workspace_bytes,
                   (unsigned long long)p.total);
  return head->dtype == PT_BF16 ? run<PT_BF16>(*head, p, (char*)workspace, st) : run<PT_FP16>(*head, p, (char*)workspace, st);
}
