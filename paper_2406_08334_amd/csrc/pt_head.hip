// Loss of a language model's head: softmax cross entropy from hidden states and weight, with gradients, logits of a piece of the rows at a time.
//
//   rows     the rows with a target, counted and listed on the device (ignored ones take no part in anything that follows); for the gradient of the
//            weight in the order of their targets, 128 words at a time
//   gather   their hidden states next to each other, zero-padded to whole steps of the products
//   logits   z = W h^T on the matrix cores, tile by tile; of each wave's part of a tile the largest z and the sum of exp(z - that) of every row, and, for
//            gradients, exp(z - that) (fp16 inputs: z in fp32)
//   soft     from those largest z, log of the sum (lse in two parts) and loss of a row; G = s (exp(z - lse) - [target]) in 16 bits, in place
//   d_hidden = G W, d_weight = G^T h on the matrix cores, and with them what rounding G has left at the targets
//
// Three products of 2 rows vocab width operations each are what it costs.  Gradients want lse of a whole row before the first of them: pieces of the
// vocabulary would take the first product twice, so the pieces are rows, of which as many are taken at a time as the workspace has room for.
// The loss alone never stores a logit.
//
// 8192 rows, width 1600, vocabulary 50257, bf16: 3.7 - 3.8 ms, of which the products 3.4 (1.21, 1.14, 1.03; 3.95 TFLOP: 1160 TFLOP/s, where a large library
// product reaches 1270 at this width) and soft 0.35; 6144 of 8192 rows, width 4096, vocabulary 32000: 3.85 - 4.0 ms, 1200 - 1250 TFLOP/s.
#include "pt_common.h"
#include "pt_mfma.h"
#include "pt_update.h"

#include <algorithm>

using namespace pt_mfma;

namespace {

typedef u32x4 u32x4_a __attribute__((aligned(2)));
typedef u32x2 u32x2_a __attribute__((aligned(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t PIECE_STEP = 256;       // pieces are multiples of this many rows
// Of a piece at best: this many rows, or, of a small vocabulary, as many as keep this many bytes of logits (16384 x 256 x 600 in one piece of 16384 rows
// instead of two: d_weight, which then needs no sums of pieces, and may be shared, 2 x 86 -> 17 + 5 us).
constexpr uint64_t PIECE_BEST = 8192, PIECE_BYTES = 1ull << 30, PIECE_MOST = 32768;
constexpr float LOG2E = 1.44269504088896340736f;

// What is kept of the logits of a piece.  bf16 inputs: exp(z - the largest of the wave's part of the row) as an fp16 number, 2^15 being 1: a rounding of up to
// 2^-11 ahead of G's own of up to 2^-8.  fp16 inputs, whose G is rounded by up to 2^-11 itself: z in fp32 (exponentials in fp16 would save a tenth of the
// time at most, and round every word but the target twice by as much).
template <int DT> constexpr bool KEEP_EXP = DT == PT_BF16;
template <int DT> constexpr uint32_t KEPT_BYTES = KEEP_EXP<DT> ? 2 : 4;
constexpr float ONE_EXP = 15.0f;

// What the device finds out about the rows.
struct Meta {
  uint32_t count;            // rows with a target
  float up, down;            // a power of two that G is multiplied by before it is rounded to 16 bits, and 1 / it: the largest |G| becomes 2^13 to 2^14
};

struct Shape {
  uint32_t R, V, d;
  uint32_t Kd, Vp;           // width and vocabulary rounded up to whole steps and tiles
  uint32_t low;              // 0, or, of few rows, how far behind a row of G what its rounding has left lies (and h once more)
  uint32_t groups;           // of GROUP words, which the rows are ordered by; 1: they are in the call's order
};
constexpr uint32_t GROUP = 128;            // what the smaller tiles of d_weight have of the vocabulary

// ---- rows ---------------------------------------------------------------------------------------------

constexpr uint32_t NO_TARGET = ~0u;

// big: the largest scale.
__device__ __forceinline__ Meta found_rows(uint32_t n, float big) {
  int e = 0;
  if (big > 0.0f && big < __builtin_inff()) (void)frexpf(big, &e);       // big < 2^e, e up to 128
  e = min(100, 14 - e);                                        // no less than -114: the power and 1 / it are numbers of normal size
  return {n, ldexpf(1.0f, e), ldexpf(1.0f, -e)};
}

struct RowArgs {
  const int64_t* target;
  const float* scale;
  Shape s;
  Meta* meta;
  uint32_t *row_of, *target_of;
  uint32_t* starts;          // [groups + 1]: where the rows of a group begin
};

// How many rows have a target below `word`, by a workgroup of THREADS.
template <int THREADS>
__device__ __forceinline__ uint32_t rows_below(const RowArgs& a, uint32_t word) {
  constexpr uint32_t WAVES = THREADS / 64, TURN = 8;
  __shared__ uint32_t s_below[WAVES];
  uint32_t n = 0;
  for (uint32_t r0 = 0; r0 < a.s.R; r0 += TURN * THREADS) {
    int64_t y[TURN];
#pragma unroll
    for (uint32_t q = 0; q < TURN; ++q) {
      const uint32_t r = r0 + q * THREADS + threadIdx.x;
      y[q] = r < a.s.R ? a.target[r] : -1;
    }
#pragma unroll
    for (uint32_t q = 0; q < TURN; ++q) n += uint64_t(y[q]) < word ? 1u : 0u;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off, 64);
  if ((threadIdx.x & 63) == 0) s_below[threadIdx.x >> 6] = n;
  __syncthreads();
  n = 0;
#pragma unroll
  for (uint32_t w = 0; w < WAVES; ++w) n += s_below[w];
  return n;
}

// The rows whose target is one of `words` from `word` on, in order, by a workgroup of THREADS; n: how many lie before them.  found: of all rows up to those.
template <int THREADS, class F>
__device__ __forceinline__ void list_rows(const RowArgs& a, uint32_t word, uint32_t words, uint32_t n, Meta& found, F&& each) {
  constexpr uint32_t WAVES = THREADS / 64, TURN = 4;       // rows of a lane at a time: their loads are under way together
  __shared__ uint32_t s_n[TURN * WAVES];
  __shared__ float s_big[WAVES];
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float big = 0.0f;
  for (uint32_t r0 = 0; r0 < a.s.R; r0 += TURN * THREADS) {
    int64_t y[TURN];
    float scale[TURN];
    uint64_t mask[TURN];
#pragma unroll
    for (uint32_t q = 0; q < TURN; ++q) {
      const uint32_t r = r0 + q * THREADS + threadIdx.x;
      y[q] = r < a.s.R ? a.target[r] : -1;
      scale[q] = r < a.s.R && a.scale ? __builtin_fabsf(a.scale[r]) : 1.0f;
    }
#pragma unroll
    for (uint32_t q = 0; q < TURN; ++q) {
      if (uint64_t(y[q]) < a.s.V) big = fmaxf(big, scale[q]);
      mask[q] = __ballot(uint64_t(y[q]) - word < words);
      if (lane == 0) s_n[q * WAVES + wave] = uint32_t(__popcll(mask[q]));
    }
    __syncthreads();
#pragma unroll
    for (uint32_t q = 0; q < TURN; ++q) {
      uint32_t before = 0, all = 0;
#pragma unroll
      for (uint32_t w = 0; w < WAVES; ++w) { const uint32_t k = s_n[q * WAVES + w]; before += w < wave ? k : 0; all += k; }
      if (uint64_t(y[q]) - word < words)
        each(n + before + uint32_t(__popcll(mask[q] & ((uint64_t(1) << lane) - 1))), r0 + q * THREADS + threadIdx.x, uint32_t(y[q]));
      n += all;
    }
    __syncthreads();
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) big = fmaxf(big, __shfl_xor(big, off, 64));
  if (lane == 0) s_big[wave] = big;
  __syncthreads();
#pragma unroll
  for (uint32_t w = 0; w < WAVES; ++w) big = fmaxf(big, s_big[w]);
  found = found_rows(n, big);
}

// A workgroup lists the rows of a group: each goes through all targets, twice, so that no count of another has to be waited for.  Bound by the round trips
// of its turns: 8192 rows in 11 us by 8 workgroups (1000 words), 13 by 393 (50257 words), 22 by 1024 (131072, two rounds of them); in the call's order, by
// one that goes through them once, 10.
__global__ void __launch_bounds__(1024) k_head_rows(const RowArgs a) {
  const uint32_t g = blockIdx.x, word = a.s.groups > 1 ? g * GROUP : 0, n = g ? rows_below<1024>(a, word) : 0;
  Meta m;
  list_rows<1024>(a, word, a.s.groups > 1 ? min(GROUP, a.s.V - word) : a.s.V, n, m, [&](uint32_t at, uint32_t r, uint32_t y) { a.row_of[at] = r; a.target_of[at] = y; });
  if (threadIdx.x != 0) return;
  a.starts[g] = n;
  if (g + 1 < a.s.groups) return;
  a.starts[g + 1] = m.count;
  *a.meta = m;
}

// One row of 16-bit words, at any address, into one of Kd words that begins at a multiple of 16 bytes; zero behind its end.
__device__ __forceinline__ void copy_row(const PT_GLOBAL uint16_t* from, PT_GLOBAL uint16_t* to, uint32_t d, uint32_t Kd, uint32_t lane, uint32_t lanes) {
#pragma unroll 4
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
// LIST: every workgroup lists the rows by itself, of which there are LISTED at most: a launch less (1000 x 1024 x 8000 105 -> 101 us); a wave counts the rows
// that its own comes behind.
// Bound by memory: 8192 rows of 4096 in 22 us, 5.2 TB/s.
constexpr uint32_t LISTED = 1024;
template <bool LIST>
__global__ void __launch_bounds__(256) k_head_gather(const RowArgs a, const uint16_t* __restrict__ hidden, uint64_t stride, uint16_t* __restrict__ packed,
                                                     float* __restrict__ loss, uint16_t* __restrict__ d_hidden, uint64_t d_stride) {
  __shared__ uint32_t s_row[LIST ? LISTED : 1], s_target[LIST ? LISTED : 1];
  const uint32_t r = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const Shape& s = a.s;
  uint32_t n, from = 0, place = r;
  if constexpr (LIST) {
    Meta m;
    list_rows<256>(a, 0, s.V, 0, m, [&](uint32_t at, uint32_t row, uint32_t y) { s_row[at] = row; s_target[at] = y; });
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.meta = m;
    n = m.count;
    if (r < n) {
      from = s_row[r];
      const uint32_t y = s_target[r];
      if (s.groups > 1) {
        const uint32_t g = y / GROUP;
        uint32_t begun = 0;                                // the groups up to that of the row before
        place = 0;
        for (uint32_t i = lane; i < n; i += 64) {
          const uint32_t h = s_target[i] / GROUP;
          const bool before = h < g || (h == g && i < r);
          place += before ? 1 : 0;
          begun = max(begun, before ? h + 1 : 0);
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) { place += __shfl_xor(place, off, 64); begun = max(begun, uint32_t(__shfl_xor(begun, off, 64))); }
        place = __builtin_amdgcn_readfirstlane(place);
        for (uint32_t i = begun + lane; i <= g; i += 64) a.starts[i] = place;
        if (place + 1 == n)
          for (uint32_t i = g + 1 + lane; i <= s.groups; i += 64) a.starts[i] = n;
      }
      if (lane == 0) { a.row_of[place] = from; a.target_of[place] = y; }
    } else if (n == 0 && r == 0) {
      for (uint32_t i = lane; i <= s.groups; i += 64) a.starts[i] = 0;
    }
  } else {
    n = a.meta->count;
    if (r < n) from = a.row_of[r];
  }
  const uint32_t zeros = s.low ? s.low : (n + TWO - 1) / TWO * TWO;
  for (uint32_t at = place; at < zeros + s.low && r < zeros; at += s.low) {      // once, or twice
    PT_GLOBAL uint16_t* to = (PT_GLOBAL uint16_t*)packed + size_t(at) * s.Kd;
    if (r < n) copy_row((const PT_GLOBAL uint16_t*)hidden + from * stride, to, s.d, s.Kd, lane, 64);
    else
      for (uint32_t c = lane * 8; c < s.Kd; c += 512) *(PT_GLOBAL u32x4*)(to + c) = u32x4{0, 0, 0, 0};
    if (!s.low) break;
  }
  if (r < s.R && uint64_t(a.target[r]) >= s.V) {
    if (lane == 0) loss[r] = 0.0f;
    if (d_hidden)
      for (uint32_t c = lane; c < s.d; c += 64) d_hidden[r * d_stride + c] = 0;
  }
}

// A weight whose rows do not all begin at multiples of 16 bytes, or end inside a step: the products load 16 bytes a lane past registers, which want that.
// Bound by memory: 50257 rows of 771 in 34 us, 4.9 TB/s.
__global__ void __launch_bounds__(256) k_head_weight(const uint16_t* __restrict__ weight, uint64_t stride, Shape s, uint16_t* __restrict__ padded) {
  const uint32_t v = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (v < s.V)
    copy_row((const PT_GLOBAL uint16_t*)weight + v * stride, (PT_GLOBAL uint16_t*)padded + size_t(v) * s.Kd, s.d, s.Kd, threadIdx.x & 63, 64);
}

__global__ void __launch_bounds__(256) k_head_zero(uint16_t* __restrict__ d_weight, uint64_t stride, Shape s) {
  for (uint32_t c = threadIdx.x; c < s.d; c += 256) d_weight[blockIdx.x * stride + c] = 0;
}

// ---- products ------------------------------------------------------------------------------------------

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
template <class C> __host__ __device__ inline Split split(uint32_t tiles, uint32_t twos) {
  const uint64_t round = uint64_t(twos) * C::TWO_NS + 3000;
  Split best = {tiles, 0, 1, (tiles + C::SLOTS - 1) / C::SLOTS * round};
  const uint32_t tail = tiles % C::SLOTS, whole = tiles - tail;
  if (!tail) return best;
  for (uint32_t n : {2u, 3u, 4u, 6u, 8u, 12u, 16u, 24u, 32u, std::min(32u, uint32_t(C::SLOTS) / tail)}) {
    if (n < 2 || n * 2 > twos) continue;
    const uint64_t ns = whole / C::SLOTS * round + (tail * n + C::SLOTS - 1) / C::SLOTS * (uint64_t((twos + n - 1) / n) * C::TWO_NS + 3000) +
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
  const int64_t* target;     // the call's own rows instead, those without a target among them (then there are no gradients); or NULL
  f32x2* part;               // [rows][parts] of the piece: largest z, sum of exp(z - largest)
  uint32_t parts;
  float* at_target;          // [rows]
  void* z;                   // [rows][Vp], or NULL: what is kept of the logits
};

// z of a tile and what becomes of it (above).  m runs over the vocabulary, so that a lane has four z of a row next to each other, n over the rows.
// Products bound it: 8192 x 1600 x 50257 1.2 ms, 1100 TFLOP/s, what is kept being written (0.8 GB) while other workgroups multiply; the loss alone of
// 4096 x 4096 x 32000 0.79 ms, 1360 TFLOP/s.  Of few rows reading the weight: one of 1600 x 50257 26 us, 6.2 TB/s.
template <int DT, class C>
__global__ void __launch_bounds__(C::THREADS) k_head_logits(const LogitArgs a) {
  typedef typename C::template Of<DT, true, true> T;
  __shared__ __attribute__((aligned(16))) char even[T::BYTES], odd[T::BYTES];
  const uint32_t n_rows = a.target ? a.rows : piece_rows(a.meta, a.first, a.rows);
  uint32_t tm, tn;
  if (!tile_of(blockIdx.x, (a.s.V + C::BM - 1) / C::BM, (n_rows + C::BN - 1) / C::BN, tm, tn)) return;
  const uint32_t m0 = tm * C::BM, n0 = tn * C::BN;
  Operand h = a.h;
  h.extent = n_rows;
  T t;
  t.run((lds_char*)even, (lds_char*)odd, a.w, h, m0, n0, 0, a.s.Kd / TWO);
  const uint32_t lane = threadIdx.x & 63, mb = m0 + t.wave_m() + (lane >> 4) * 4;
  // of rows m behind the vocabulary there is nothing to sum
  if (m0 + C::BM > a.s.V) {
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
    // The difference first: the largest adds 1 exactly, so no sum is below 1 and no loss below 0.  Of nothing but -inf the sum is 0.
    const float top = big == -__builtin_inff() ? 0.0f : big;
    float sum = 0.0f;
    if (KEEP_EXP<DT> && a.z) {
      typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
      PT_GLOBAL uint16_t* row = (PT_GLOBAL uint16_t*)a.z + size_t(n) * a.s.Vp + m0 + t.wave_m() + eight_at();
#pragma unroll
      for (int i = 0; i < T::FM; i += 2) {
        u32x2 w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f32x4 e;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            e[q] = __builtin_amdgcn_exp2f(__builtin_fmaf(t.acc[i + h][j][q] - top, LOG2E, ONE_EXP));
            sum += e[q];
          }
          w[h] = __builtin_bit_cast(u32x2, __builtin_convertvector(e, f16x4));
        }
        const u32x4 x = eight(w[0], w[1]);
        if (live) *(PT_GLOBAL u32x4*)(row + i * 16) = x;
      }
    } else {
#pragma unroll
      for (int i = 0; i < T::FM; ++i) {
        if (a.z && live) *(PT_GLOBAL f32x4*)((PT_GLOBAL float*)a.z + size_t(n) * a.s.Vp + mb + i * 16) = t.acc[i][j];
#pragma unroll
        for (int q = 0; q < 4; ++q) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(t.acc[i][j][q] - top, LOG2E, ONE_EXP));
      }
    }
    sum *= 0x1p-15f;
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (live && lane < 16) a.part[size_t(n) * a.parts + tm * C::WM + t.wave_m() / T::TM] = f32x2{big, sum};
    uint32_t y = ~0u;                                                 // the lane's z are mb + 16 i + q
    if (live) y = a.target ? (uint64_t(a.target[n]) < a.s.V ? uint32_t(a.target[n]) - mb : ~0u) : a.target_of[n] - mb;
    const bool mine = y < uint32_t(T::TM) && (y & 15) < 4;
    if (__any(mine)) {
      float zy = 0.0f;
#pragma unroll
      for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) zy = y == uint32_t(i * 16 + q) ? t.acc[i][j][q] : zy;
      if (mine) a.at_target[n] = zy;
    }
  }
}

// Largest z and sum of two parts of a row together; lse of a row from all of them.
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
  Meta* meta;
  uint32_t first, rows;
  uint32_t *row_of, *target_of;            // of the piece
  const int64_t* target;                   // as in LogitArgs
  const uint16_t* hidden;                  // of such rows, and where they go
  uint64_t hidden_stride;
  uint16_t* packed;
  const f32x2* part;
  uint32_t parts, part_width;
  const float* at_target;
  const float* scale;
  float* loss;
  void* z;
  uint16_t* g;               // G; where z lies, or, of few rows, elsewhere
  uint64_t g_pitch;          // bytes
  float* rest;               // [rows]: of G at the target, what its rounding has left
  uint16_t* rests;           // [rows][2 GROUP]: the same as a row of a matrix over two groups of words, zero at all others; or NULL
};

// Of the workgroup, in all its lanes.
__device__ __forceinline__ f32x2 join_row(const f32x2* part, uint32_t parts) {
  __shared__ f32x2 s_x[4];
  f32x2 x = {-__builtin_inff(), 0.0f};
  for (uint32_t i = threadIdx.x; i < parts; i += 256) x = join(x, part[i]);
  x = join_wave(x);
  if ((threadIdx.x & 63) == 0) s_x[threadIdx.x >> 6] = x;
  __syncthreads();
  return join(join(s_x[0], s_x[1]), join(s_x[2], s_x[3]));
}

// A row's loss from its largest z, the sum of exp(z - that) and the target's z.  The difference of two z first: lse as one number would be rounded at the
// size of the logits, and a small loss beside large ones is less than that (z of 4000: 1e-4).
__device__ __forceinline__ float loss_of(f32x2 x, float zy) { return (x[0] - zy) + logf(x[1]); }

// The loss alone: a workgroup a row.  4096 rows, 250 parts each: 9 us.
__global__ void __launch_bounds__(256) k_head_loss(const SoftArgs a) {
  const uint32_t r = blockIdx.x;
  if (r >= (a.target ? a.rows : piece_rows(a.meta, a.first, a.rows))) return;
  const f32x2 x = join_row(a.part + size_t(r) * a.parts, a.parts);
  if (threadIdx.x != 0) return;
  if (a.target) a.loss[r] = uint64_t(a.target[r]) < a.s.V ? loss_of(x, a.at_target[r]) : 0.0f;
  else a.loss[a.row_of[r]] = loss_of(x, a.at_target[r]);
}

// Eight numbers in 16 bits, and what is left of them.
template <int DT>
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  const u32x2 a = encode16x4<DT>(f32x4{x[0], x[1], x[2], x[3]}), b = encode16x4<DT>(f32x4{x[4], x[5], x[6], x[7]});
  return u32x4{a.x, a.y, b.x, b.y};
}
template <int DT>
__device__ __forceinline__ u32x4 pack8_rest(const float (&x)[8], const u32x4& q) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = x[j] - decode16<DT>((q[j / 2] >> (16 * (j & 1))) & 0xffffu);
  return pack8<DT>(y);
}

// Loss and G of a row by a workgroup, G where what is kept of the row's logits lies.  Of few rows G has a place of its own, and several workgroups
// (gridDim.y) share a row.  Bound by memory: 6144 x 32000 bf16 in 132 us, 6.0 TB/s; 8192 x 50257 bf16 338 us, 4.9; 8192 x 32000 fp16 348, 4.5.
// Of z in fp32, which are twice as long, a round takes 2048: a lane has its own of the next round under way while it stores those of this one,
// and stores when every lane has this round's.
// Rows as they are (few; SoftArgs::target): every one has its place, those without a target a G of zero, and the workgroups behind those of G do what
// gathering does before otherwise.
template <int DT>
__global__ void __launch_bounds__(256) k_head_soft(const SoftArgs a) {
  uint32_t r = blockIdx.x, n, y = NO_TARGET;
  const uint32_t tid = threadIdx.x;
  float up;
  if (a.target) {
    if (r >= TWO) {
      if (blockIdx.y) return;
      r -= TWO;
      const bool has = r < a.rows && uint64_t(a.target[r]) < a.s.V;
      for (uint32_t at = r; at <= r + a.s.low; at += a.s.low) {
        PT_GLOBAL uint16_t* to = (PT_GLOBAL uint16_t*)a.packed + size_t(at) * a.s.Kd;
        if (has) copy_row((const PT_GLOBAL uint16_t*)a.hidden + r * a.hidden_stride, to, a.s.d, a.s.Kd, tid, 256);
        else
          for (uint32_t c = tid * 8; c < a.s.Kd; c += 2048) *(PT_GLOBAL u32x4*)(to + c) = u32x4{0, 0, 0, 0};
      }
      return;
    }
    // a wave sees all rows
    const uint32_t lane = tid & 63;
    const int64_t t = lane < a.rows ? a.target[lane] : -1;
    const bool has = uint64_t(t) < a.s.V;
    float big = has ? (a.scale ? __builtin_fabsf(a.scale[lane]) : 1.0f) : 0.0f;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) big = fmaxf(big, __shfl_xor(big, off, 64));
    const Meta m = found_rows(a.rows, big);
    if (blockIdx.x == 0 && blockIdx.y == 0 && tid < a.rows) {
      a.row_of[tid] = tid;
      a.target_of[tid] = has ? uint32_t(t) : NO_TARGET;
      if (!has) { a.loss[tid] = 0.0f; a.rest[tid] = 0.0f; }
      if (tid == 0) *a.meta = m;
    }
    up = m.up;
    n = a.rows;
    if (r < n) {
      const int64_t own = a.target[r];
      if (uint64_t(own) < a.s.V) y = uint32_t(own);
    }
  } else {
    n = piece_rows(a.meta, a.first, a.rows);
    up = a.meta->up;
    if (r < n) y = a.target_of[r];
  }
  if (r >= (a.s.low ? a.s.low : (n + TWO - 1) / TWO * TWO)) return;
  PT_GLOBAL uint16_t* g = (PT_GLOBAL uint16_t*)((PT_GLOBAL char*)a.g + r * a.g_pitch);
  PT_GLOBAL uint16_t* g_low = (PT_GLOBAL uint16_t*)((PT_GLOBAL char*)g + a.s.low * a.g_pitch);
  const uint32_t first = blockIdx.y * 2048 + tid * 8, turn = gridDim.y * 2048;
  if (y == NO_TARGET) {                                    // rows up to a whole step too: zero
    for (uint32_t c = first; c < a.s.Vp; c += turn) {
      *(PT_GLOBAL u32x4*)(g + c) = u32x4{0, 0, 0, 0};
      if (a.s.low) *(PT_GLOBAL u32x4*)(g_low + c) = u32x4{0, 0, 0, 0};
    }
    return;
  }
  const f32x2 x = join_row(a.part + size_t(r) * a.parts, a.parts);
  const uint32_t row = a.target ? r : a.row_of[r];
  const float top = x[0], log_sum = logf(x[1]), s = (a.scale ? a.scale[row] : 1.0f) * up, loss = loss_of(x, a.at_target[r]);
  const float gy = s * expm1f(-loss);
  if (tid == 0 && blockIdx.y == 0) {
    a.loss[row] = loss;
    a.rest[r] = gy - decode16<DT>(encode16<DT>(gy));
  }
  if (a.rests && tid < 2 * GROUP / 8) {
    const uint32_t rest = encode16<DT>(gy - decode16<DT>(encode16<DT>(gy))), at = y % (2 * GROUP);
    u32x4 w = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) w[j] = at / 2 == tid * 4 + j ? rest << (16 * (at & 1)) : 0;
    *(PT_GLOBAL u32x4*)((PT_GLOBAL uint16_t*)a.rests + size_t(r) * (2 * GROUP) + tid * 8) = w;
  }
  if constexpr (KEEP_EXP<DT>) {
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    const PT_GLOBAL f32x2* part = (const PT_GLOBAL f32x2*)a.part + size_t(r) * a.parts;
#pragma unroll 4
    for (uint32_t c = first; c < a.s.Vp; c += turn) {
      const f16x8 e = __builtin_bit_cast(f16x8, *(const PT_GLOBAL u32x4*)((const PT_GLOBAL uint16_t*)a.z + size_t(r) * a.s.Vp + c));
      const float f = s * __builtin_amdgcn_exp2f(__builtin_fmaf((part[min(c / a.part_width, a.parts - 1)][0] - top) - log_sum, LOG2E, -ONE_EXP));
      float p[8];
#pragma unroll
      for (uint32_t j = 0; j < 8; ++j) {
        p[j] = f * float(e[j]);
        if (c + j == y) p[j] = gy;
        if (c + j >= a.s.V) p[j] = 0.0f;
      }
      const u32x4 w = pack8<DT>(p);
      *(PT_GLOBAL u32x4*)(g + c) = w;
      if (a.s.low) *(PT_GLOBAL u32x4*)(g_low + c) = pack8_rest<DT>(p, w);
    }
    return;
  }
  const PT_GLOBAL float* z = (const PT_GLOBAL float*)a.z + size_t(r) * a.s.Vp;
  const uint32_t last = a.s.Vp - 8;                        // lanes behind the row's end load its last ones, and store nothing
  f32x4 q[2], next[2];
  uint32_t c = first, at = min(c, last);
  q[0] = *(const PT_GLOBAL f32x4*)(z + at); q[1] = *(const PT_GLOBAL f32x4*)(z + at + 4);
  for (; c < a.s.Vp + tid * 8; c += turn) {
    at = min(c + turn, last);
    next[0] = *(const PT_GLOBAL f32x4*)(z + at); next[1] = *(const PT_GLOBAL f32x4*)(z + at + 4);
    float p[8];
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
      p[j] = s * __builtin_amdgcn_exp2f(((q[j / 4][j % 4] - top) - log_sum) * LOG2E);
      if (c + j == y) p[j] = gy;
      if (c + j >= a.s.V) p[j] = 0.0f;
    }
    const u32x4 w = pack8<DT>(p);
    asm volatile("" : : "v"(w) : "memory");                // this round's z are in registers
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (c < a.s.Vp) {
      *(PT_GLOBAL u32x4*)(g + c) = w;
      if (a.s.low) *(PT_GLOBAL u32x4*)(g_low + c) = pack8_rest<DT>(p, w);
    }
    q[0] = next[0]; q[1] = next[1];
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

struct GradArgs {
  Shape s;
  Operand p, q;
  const Meta* meta;
  uint32_t first, rows;
  const uint32_t *row_of, *target_of;      // of the piece
  uint16_t* out;
  uint64_t stride;
  float* part;               // sums of several workgroups a tile: [n][tail][BN][BM]
  Split split;               // of d_weight
  const float* rest;
  const uint16_t* rests;     // of the piece, for d_weight, and where the groups' rows begin; or NULL
  const uint32_t* starts;
  const uint16_t* weight;
  uint64_t weight_stride;
  float* acc;                // d_weight over several pieces: sums so far [V][pitch]
  uint32_t pitch;
  bool read_acc, write_acc;
};

// G at the target has been rounded like the rest of its row, of which it can be the only number that counts: what that has left, times the target's
// row of the weight, goes into the sum in fp32.  (Into d_weight: d_weight_tile.)
template <int DT>
__device__ __forceinline__ f32x4 add_rest(f32x4 x, float rest, const PT_GLOBAL uint16_t* w, uint32_t m, uint32_t d) {
  if (m >= d) return x;
  const u32x2 q = *(const PT_GLOBAL u32x2*)(w + m);        // the rows that the products take are whole pieces of 16 bytes
  const float v[4] = {decode16<DT>(q.x & 0xffffu), decode16<DT>(q.x >> 16), decode16<DT>(q.y & 0xffffu), decode16<DT>(q.y >> 16)};
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = __builtin_fmaf(rest, v[j], x[j]);
  return x;
}

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

// d_hidden of a piece: m runs over the width, n over rows, k over the vocabulary.  Products bound it: 6144 x 4096 x 32000 1.23 ms, 1310 TFLOP/s;
// 8192 x 1600 x 50257 1.15 ms, 1150: 224 tiles, a round that leaves 32 compute units idle (by eight workgroups each they would be 1792, seven rounds of an
// eighth, but their sums cost more than the idle units).
template <int DT, class C>
__device__ __forceinline__ void d_hidden_tile(const GradArgs& a, lds_char* even, lds_char* odd, uint32_t block) {
  const uint32_t n_rows = piece_rows(a.meta, a.first, a.rows);
  const uint32_t tiles_m = (a.s.d + C::BM - 1) / C::BM, tiles_n = (n_rows + C::BN - 1) / C::BN, twos = a.s.Vp / TWO;
  const Split sp = split<C>(tiles_m * tiles_n, twos);
  uint32_t tm, tn, part;
  PT_GLOBAL float* sums;
  if (!part_of<C>(sp, block, tiles_m, tiles_n, a.part, tm, tn, part, sums)) return;
  const uint32_t t0 = sums ? uint32_t(uint64_t(twos) * part / sp.n) : 0, t1 = sums ? uint32_t(uint64_t(twos) * (part + 1) / sp.n) : twos;
  Operand q = a.q;
  q.extent = n_rows;
  const float down = a.meta->down;
  with_tile<DT, C, false, true>(a.s.d - tm * C::BM, [&](auto t) {
    typedef decltype(t) T;
    t.run(even, odd, a.p, q, tm * C::BM, tn * C::BN, t0 * TWO, t1 - t0);
    const uint32_t lane = threadIdx.x & 63, mw = tm * C::BM + t.wave_m(), mb = mw + (lane >> 4) * 4;
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const uint32_t n = tn * C::BN + t.wave_n() + j * 16 + (lane & 15);
      const bool live = n < n_rows;
      if (sums) {
        leave<C>(t, j, sums);
        continue;
      }
      const uint32_t at = live ? n : 0;                    // lanes without a row take part in the exchange
      PT_GLOBAL uint16_t* row = (PT_GLOBAL uint16_t*)a.out + a.row_of[at] * a.stride;
      const uint32_t y = a.target_of[at];
      const PT_GLOBAL uint16_t* w = (const PT_GLOBAL uint16_t*)a.weight + (y == NO_TARGET ? 0 : y) * a.weight_stride;
      const float rest = a.rest[at];
#pragma unroll
      for (int i = 0; i < T::FM; i += 2) {
        const uint32_t m = mb + i * 16;
        u32x4 x = eight(encode16x4<DT>(add_rest<DT>(t.acc[i][j], rest, w, m, a.s.d) * down),
                        encode16x4<DT>(add_rest<DT>(t.acc[i + 1][j], rest, w, m + 16, a.s.d) * down));
        if (y == NO_TARGET) x = u32x4{0, 0, 0, 0};         // whatever the weight holds
        if (live) store8(row, mw + i * 16 + eight_at(), a.s.d, x);
      }
    }
  });
}

template <int DT, class C>
__global__ void __launch_bounds__(C::THREADS) k_head_d_hidden(const GradArgs a) {
  constexpr int BYTES = C::template Of<DT, false, true>::BYTES;
  __shared__ __attribute__((aligned(16))) char even[BYTES], odd[BYTES];
  d_hidden_tile<DT, C>(a, (lds_char*)even, (lds_char*)odd, blockIdx.x);
}

// Adds up what several workgroups a tile have left, four results of a row at a time, by JOINERS workgroups at most: that many at once, and few if the rows
// turn out to need none.  f: called with place (m, n) and sum.
constexpr uint32_t JOINERS = 2048;
template <class C> uint32_t joiners(uint32_t tail) { return std::min<uint32_t>(JOINERS, tail * (C::BM * C::BN / 1024)); }
template <class C, class F>
__device__ __forceinline__ void join_tiles(const float* room, const Split& s, uint32_t tm, uint32_t tn, F&& f) {
  constexpr uint32_t TILE = C::BM * C::BN;
  const size_t next = size_t(s.tail) * TILE;
  for (uint32_t i = blockIdx.x; i < s.tail * (TILE / 1024); i += gridDim.x) {
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

template <int DT, class C>
__global__ void __launch_bounds__(256) k_head_join(const GradArgs a) {
  const uint32_t n_rows = piece_rows(a.meta, a.first, a.rows), tiles_m = (a.s.d + C::BM - 1) / C::BM, tiles_n = (n_rows + C::BN - 1) / C::BN;
  const float down = a.meta->down;
  join_tiles<C>(a.part, split<C>(tiles_m * tiles_n, a.s.Vp / TWO), tiles_m, tiles_n, [&](uint32_t m, uint32_t n, f32x4 x) {
    if (n >= n_rows || m >= a.s.d) return;
    const uint32_t target = a.target_of[n];
    u32x2 y = {0, 0};
    if (target != NO_TARGET) {
      const PT_GLOBAL uint16_t* w = (const PT_GLOBAL uint16_t*)a.weight + target * a.weight_stride;
      y = encode16x4<DT>(add_rest<DT>(x, a.rest[n], w, m, a.s.d) * down);
    }
    store4((PT_GLOBAL uint16_t*)a.out + a.row_of[n] * a.stride, m, a.s.d, y);
  });
}

// d_weight: m runs over the width, n over the vocabulary, k over the piece's rows, and once more over those whose target is a word of the tile: what is left
// of their G there, a matrix with one number a row, so that a word with a thousand rows takes no longer than a thousand with one.  A tile's rows lie next to
// each other, as they are ordered by target: of 8192 rows and 50257 words 42, one round of two steps behind 64.  (8192 x 1600 x 50257 3.66 -> 3.69 ms for the whole
// call, 1531 x 771 x 50257 604 -> 619 us, 8192 x 512 x 1000 97 -> 104; the error against 64 bits of 6144 x 4096 x 32000, bf16: 2.2e-3 to 2.4e-3 -> 1.66e-3, what
// rounding the result costs.)
// Products bound it: 6144 x 4096 x 32000 1.21 ms, 1330 TFLOP/s; 8192 x 1600 x 50257 1.05 ms, 1250.
template <int DT, class C>
__device__ __forceinline__ void d_weight_tile(const GradArgs& a, lds_char* even, lds_char* odd, uint32_t block) {
  const uint32_t n_rows = piece_rows(a.meta, a.first, a.rows);
  if (!n_rows && a.read_acc && a.write_acc) return;
  uint32_t tm, tn, part;
  PT_GLOBAL float* left;
  if (!part_of<C>(a.split, block, (a.s.d + C::BM - 1) / C::BM, (a.s.V + C::BN - 1) / C::BN, a.part, tm, tn, part, left)) return;
  Operand p = a.p, q = a.q;
  p.k = q.k = !n_rows ? 0 : a.s.low ? 2 * a.s.low : (n_rows + TWO - 1) / TWO * TWO;
  const uint32_t twos = p.k / TWO, t0 = left ? twos * part / a.split.n : 0, t1 = left ? twos * (part + 1) / a.split.n : twos;
  const float down = a.meta->down;
  with_tile<DT, C, false, false>(a.s.d - tm * C::BM, [&](auto t) {
    typedef decltype(t) T;
    t.run(even, odd, p, q, tm * C::BM, tn * C::BN, t0 * TWO, t1 - t0);
    if (a.rests) {
      const uint32_t g = tn * (C::BN / GROUP), end = a.first + piece_rows(a.meta, a.first, a.rows);
      const uint32_t r0 = max(a.starts[g], a.first) - a.first, r1 = min(max(a.starts[min(g + C::BN / GROUP, a.s.groups)], a.first), end) - a.first;
      if (r0 < r1) {
        const uint32_t more = (r1 - r0 + TWO - 1) / TWO, m0 = left ? more * part / a.split.n : 0, m1 = left ? more * (part + 1) / a.split.n : more;
        __builtin_amdgcn_s_barrier();
        Operand h = a.p;
        h.k = min(r0 + m1 * TWO, r1);
        t.add(even, odd, h, {a.rests + tn * C::BN % (2 * GROUP), 2 * (2 * GROUP), C::BN, h.k}, tm * C::BM, 0, r0 + m0 * TWO, m1 - m0);
      }
    }
    const uint32_t lane = threadIdx.x & 63, mw = tm * C::BM + t.wave_m(), mb = mw + (lane >> 4) * 4;
#pragma unroll
    for (int j = 0; j < T::FN; ++j) {
      const uint32_t n = tn * C::BN + t.wave_n() + j * 16 + (lane & 15);
      const bool live = n < a.s.V;
      if (left) {
        leave<C>(t, j, left);
        continue;
      }
      const uint32_t at = live ? n : 0;                    // lanes without a row take part in the exchange
      PT_GLOBAL uint16_t* row = (PT_GLOBAL uint16_t*)a.out + at * a.stride;
      PT_GLOBAL float* sums = (PT_GLOBAL float*)a.acc + size_t(at) * a.pitch;          // of the pieces before, in fp32
#pragma unroll
      for (int i = 0; i < T::FM; i += 2) {
        u32x2 w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t m = mb + (i + h) * 16;
          f32x4 x = t.acc[i + h][j] * down;
          if (a.read_acc && m < a.s.d) x += *(const PT_GLOBAL f32x4*)(sums + m);
          if (a.write_acc && m < a.s.d && live) *(PT_GLOBAL f32x4*)(sums + m) = x;
          w[h] = encode16x4<DT>(x);
        }
        const u32x4 x = eight(w[0], w[1]);
        if (live && !a.write_acc) store8(row, mw + i * 16 + eight_at(), a.s.d, x);
      }
    }
  });
}

template <int DT, class C>
__global__ void __launch_bounds__(C::THREADS) k_head_d_weight(const GradArgs a) {
  constexpr int BYTES = C::template Of<DT, false, false>::BYTES;
  __shared__ __attribute__((aligned(16))) char even[BYTES], odd[BYTES];
  d_weight_tile<DT, C>(a, (lds_char*)even, (lds_char*)odd, blockIdx.x);
}

template <int DT, class C>
__global__ void __launch_bounds__(256) k_head_join_weight(const GradArgs a) {
  const float down = a.meta->down;
  join_tiles<C>(a.part, a.split, (a.s.d + C::BM - 1) / C::BM, (a.s.V + C::BN - 1) / C::BN, [&](uint32_t m, uint32_t n, f32x4 x) {
    if (n < a.s.V && m < a.s.d) store4((PT_GLOBAL uint16_t*)a.out + n * a.stride, m, a.s.d, encode16x4<DT>(x * down));
  });
}

// Both gradients of few rows in one launch: neither fills the chip for long.  Bound by memory, which the weight is read from and its gradient written to:
// 64 x 1600 x 50257 in 87 us, 3.7 TB/s (d_weight in tiles of 128 x 64 89, of 64 x 128 91, of 64 x 64 114).
template <int DT>
__global__ void __launch_bounds__(256) k_head_few_grads(const GradArgs h, const GradArgs w, uint32_t blocks_h) {
  static_assert(Few::THREADS == 256 && Mid::THREADS == 256, "one launch");
  constexpr int BYTES = std::max(Few::Of<DT, false, true>::BYTES, Mid::Of<DT, false, false>::BYTES);
  __shared__ __attribute__((aligned(16))) char even[BYTES], odd[BYTES];
  if (blockIdx.x < blocks_h) d_hidden_tile<DT, Few>(h, (lds_char*)even, (lds_char*)odd, blockIdx.x);
  else d_weight_tile<DT, Mid>(w, (lds_char*)even, (lds_char*)odd, blockIdx.x - blocks_h);
}

// ---- host -----------------------------------------------------------------------------------------------

// Up to LOW_ROWS rows the gradient of the weight is a matter of writing it: what rounding G has left is multiplied as well, as rows of its own.  It is of few
// rows that a result has few terms whose roundings could cancel.  (100 x 1600 x 50257: 168 us without, 180 with; 256 x 4096 x 32000: 330, 379.)
constexpr uint32_t LOW_ROWS = 128, FEW_ROWS = 64;

// Whether a product of m x n is sooner done in tiles of Mid.
inline bool mid_tiles(uint64_t m, uint64_t n) {
  const auto rounds = [&](uint64_t bm, uint64_t bn, uint64_t slots) { return ((m + bm - 1) / bm * ((n + bn - 1) / bn) + slots - 1) / slots; };
  return rounds(Mid::BM, Mid::BN, Mid::SLOTS) * Mid::TWO_NS < rounds(Big::BM, Big::BN, Big::SLOTS) * Big::TWO_NS;
}
uint64_t up(uint64_t x, uint64_t to) { return (x + to - 1) / to * to; }

// Of d_hidden of any number of rows up to `rows` that turns out to have a target: the most workgroups, tiles that several share, and bytes of their sums.
struct Most { uint32_t grid, tail; uint64_t bytes; };

// Where everything lies in the workspace, for pieces of `rows` rows.
struct Plan {
  Shape s;
  uint32_t parts, pitch, pieces, rows;
  bool grads, direct, as_is;               // direct: the weight is taken where it lies; as_is: so are the hidden states
  bool ordered;                            // rows by target, for d_weight
  Most hidden;                             // of a whole piece
  uint64_t meta, row_of, target_of, starts, at_target, rest, rests, packed, weight, part, z, g, g_pitch, sums, acc, total;
};

// Partial sums of a row's exponentials.
template <class C> uint32_t parts(uint32_t vocab) { return (vocab + C::BM - 1) / C::BM * C::WM; }

template <class C> Most most(const Shape& s, uint32_t rows) {
  Most x = {0, 0, 0};
  const uint32_t tm = (s.d + C::BM - 1) / C::BM;
  for (uint32_t tn = 1; tn <= (rows + C::BN - 1) / C::BN; ++tn) {
    const Split sp = split<C>(tm * tn, s.Vp / TWO);
    x.grid = std::max(x.grid, split_grid(sp));
    x.tail = std::max(x.tail, sp.tail);
    x.bytes = std::max<uint64_t>(x.bytes, 4ull * sp.tail * sp.n * C::BM * C::BN);
  }
  return x;
}

// Whether d_hidden is sooner done in tiles of Mid.
inline bool mid_hidden(const Shape& s, uint32_t rows) {
  const auto ns = [&](auto c) {
    typedef decltype(c) C;
    return split<C>((s.d + C::BM - 1) / C::BM * ((rows + C::BN - 1) / C::BN), s.Vp / TWO).ns;
  };
  return ns(Mid{}) < ns(Big{});
}

// d_weight of `rows` rows: whether it is sooner done in tiles of Mid, whose width ends at multiples of 128 (of Big's the last tile may be a narrower one),
// and how they are split; in one piece alone, which needs no sums of pieces.
struct WeightTiles { bool mid; Split split; uint64_t bytes; };
inline WeightTiles weight_tiles(const Shape& s, uint32_t rows, bool one_piece) {
  const uint32_t twos = (rows + TWO - 1) / TWO, left = s.d % 256, tenths = s.d / 256 * 10 + (left == 0 ? 0 : left <= 64 ? 4 : left <= 128 ? 6 : 10);
  const auto tiles = [&](auto c) {
    typedef decltype(c) C;
    const uint32_t n = (s.d + C::BM - 1) / C::BM * ((s.V + C::BN - 1) / C::BN);
    const Split sp = split<C>(n, one_piece ? twos : 1);
    return WeightTiles{C::BM == Mid::BM, sp, 4ull * sp.tail * sp.n * C::BM * C::BN};
  };
  const WeightTiles big = tiles(Big{}), mid = tiles(Mid{});
  const uint64_t big_ns = big.split.ns * tenths / ((s.d + 255) / 256 * 10);
  return mid.split.ns < big_ns ? mid : big;
}

Most most_hidden(const Shape& s, uint32_t rows) {
  return rows <= FEW_ROWS ? most<Few>(s, rows) : mid_hidden(s, rows) ? most<Mid>(s, rows) : most<Big>(s, rows);
}

Plan make_plan(const pt_head& h, uint64_t rows) {
  Plan p{};
  p.s = {h.rows, h.vocab, h.width, uint32_t(up(h.width, TWO)), uint32_t(up(h.vocab, 256)), 0, 1};
  if (h.d_weight && h.rows <= LOW_ROWS) p.s.low = uint32_t(up(h.rows, BK));
  p.ordered = h.d_weight && h.rows > LOW_ROWS;
  if (p.ordered) p.s.groups = (h.vocab + GROUP - 1) / GROUP;
  p.grads = h.d_hidden || h.d_weight;
  p.direct = h.width % BK == 0 && h.weight_stride % 8 == 0 && (uintptr_t)h.weight % 16 == 0;
  p.as_is = p.direct && h.rows <= FEW_ROWS && h.hidden_stride % 8 == 0 && h.hidden_stride <= (1u << 21) && (uintptr_t)h.hidden % 16 == 0;
  p.parts = std::max({parts<Few>(h.vocab), parts<Mid>(h.vocab), parts<Big>(h.vocab)});
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
  p.starts = take(4ull * (p.s.groups + 1));
  p.at_target = take(4ull * p.rows);
  p.rest = take(p.grads ? 4ull * p.rows : 0);
  p.rests = take(p.ordered ? 2ull * (2 * GROUP) * p.rows : 0);
  p.packed = take(2ull * (up(h.rows, TWO) + p.s.low) * p.s.Kd);
  p.weight = take(p.direct ? 0 : 2ull * h.vocab * p.s.Kd);
  p.part = take(8ull * p.rows * p.parts);
  const uint64_t kept = h.dtype == PT_BF16 ? KEPT_BYTES<PT_BF16> : KEPT_BYTES<PT_FP16>;
  p.z = take(p.grads ? kept * p.rows * p.s.Vp : 0);
  p.g = p.z;
  p.g_pitch = kept * p.s.Vp;
  if (p.grads && h.rows <= LOW_ROWS) {
    p.g_pitch = 2ull * p.s.Vp;
    p.g = take(p.g_pitch * (up(h.rows, TWO) + p.s.low));
  }
  uint64_t sums = 0;                       // of the gradients, which come one after the other
  if (h.d_hidden) {
    p.hidden = most_hidden(p.s, std::min(p.rows, h.rows));
    sums = p.hidden.bytes;
    if (p.pieces > 1) sums = std::max(sums, most_hidden(p.s, h.rows - (p.pieces - 1) * p.rows).bytes);
  }
  if (h.d_weight && p.pieces == 1 && h.rows > FEW_ROWS) sums = std::max(sums, weight_tiles(p.s, h.rows, true).bytes);
  p.sums = take(sums);
  p.acc = take(h.d_weight && p.pieces > 1 ? 4ull * h.vocab * p.pitch : 0);
  p.total = at;
  return p;
}

uint64_t best_rows(const pt_head& h) {
  const uint64_t row = up(h.vocab, 256) * (h.dtype == PT_BF16 ? KEPT_BYTES<PT_BF16> : KEPT_BYTES<PT_FP16>);
  return std::min({std::max(PIECE_BEST, PIECE_BYTES / row / PIECE_STEP * PIECE_STEP), PIECE_MOST, up(h.rows, PIECE_STEP)});
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
  if (h->rows > (1u << 25) || h->vocab > (1u << 21) || h->width > (1u << 20) || h->weight_stride > (1u << 21))
    return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "%s: more than 2^25 rows, 2^21 words, a width over 2^20 or a weight stride over 2^21", who);
  return PT_OK;
}

// Launches.
template <int DT, class C> int logits(const LogitArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_head_logits<DT, C>), dim3(tile_grid((a.s.V + C::BM - 1) / C::BM, (a.rows + C::BN - 1) / C::BN)), dim3(C::THREADS), 0, st, a);
  PT_LAUNCH_CHECK(nullptr, "k_head_logits");
  return PT_OK;
}
template <int DT, class C> int join_hidden(const GradArgs& a, const Most& x, hipStream_t st) {
  if (!x.tail) return PT_OK;
  hipLaunchKernelGGL((k_head_join<DT, C>), dim3(joiners<C>(x.tail)), dim3(256), 0, st, a);
  PT_LAUNCH_CHECK(nullptr, "k_head_join");
  return PT_OK;
}
template <int DT, class C> int d_hidden(const GradArgs& a, const Most& x, hipStream_t st) {
  hipLaunchKernelGGL((k_head_d_hidden<DT, C>), dim3(x.grid), dim3(C::THREADS), 0, st, a);
  PT_LAUNCH_CHECK(nullptr, "k_head_d_hidden");
  return join_hidden<DT, C>(a, x, st);
}
template <int DT> int few_grads(const GradArgs& h, const GradArgs& w, const Most& x, hipStream_t st) {
  hipLaunchKernelGGL(k_head_few_grads<DT>, dim3(x.grid + split_grid(w.split)), dim3(256), 0, st, h, w, x.grid);
  PT_LAUNCH_CHECK(nullptr, "k_head_few_grads");
  return join_hidden<DT, Few>(h, x, st);
}
template <int DT, class C> int d_weight(const GradArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_head_d_weight<DT, C>), dim3(split_grid(a.split)), dim3(C::THREADS), 0, st, a);
  PT_LAUNCH_CHECK(nullptr, "k_head_d_weight");
  if (!a.split.tail) return PT_OK;
  hipLaunchKernelGGL((k_head_join_weight<DT, C>), dim3(joiners<C>(a.split.tail)), dim3(256), 0, st, a);
  PT_LAUNCH_CHECK(nullptr, "k_head_join_weight");
  return PT_OK;
}

template <int DT>
int run(const pt_head& h, const Plan& p, char* ws, hipStream_t st) {
  const Shape& s = p.s;
  Meta* meta = (Meta*)(ws + p.meta);
  uint32_t *row_of = (uint32_t*)(ws + p.row_of), *target_of = (uint32_t*)(ws + p.target_of);
  uint16_t* packed = (uint16_t*)(ws + p.packed);
  const RowArgs ra = {h.target, h.row_scale, s, meta, row_of, target_of, (uint32_t*)(ws + p.starts)};
  const dim3 gather(uint32_t(up(s.R, TWO) / 4));
  if (p.as_is) {
    // few rows: those without a target are multiplied too, and what else gathering does is done with G
  } else if (s.R <= LISTED) {
    hipLaunchKernelGGL(k_head_gather<true>, gather, dim3(256), 0, st, ra, (const uint16_t*)h.hidden, h.hidden_stride, packed, h.loss, (uint16_t*)h.d_hidden,
                       h.d_hidden_stride);
  } else {
    hipLaunchKernelGGL(k_head_rows, dim3(s.groups), dim3(1024), 0, st, ra);
    PT_LAUNCH_CHECK(nullptr, "k_head_rows");
    hipLaunchKernelGGL(k_head_gather<false>, gather, dim3(256), 0, st, ra, (const uint16_t*)h.hidden, h.hidden_stride, packed, h.loss,
                       (uint16_t*)h.d_hidden, h.d_hidden_stride);
  }
  PT_LAUNCH_CHECK(nullptr, "k_head_gather");
  // the weight: k (of the logits) next to each other in rows of `width` elements
  uint32_t width = s.d;
  const uint16_t* weight = (const uint16_t*)h.weight;
  uint64_t stride = h.weight_stride;
  if (!p.direct) {
    hipLaunchKernelGGL(k_head_weight, dim3((s.V + 3) / 4), dim3(256), 0, st, weight, stride, s, (uint16_t*)(ws + p.weight));
    PT_LAUNCH_CHECK(nullptr, "k_head_weight");
    weight = (const uint16_t*)(ws + p.weight);
    stride = width = s.Kd;
  }
  int rc = PT_OK;
  for (uint32_t i = 0; i < p.pieces && rc == PT_OK; ++i) {
    const uint32_t first = i * p.rows, rows = std::min(p.rows, s.R - first);
    uint16_t* hid = packed + size_t(first) * s.Kd;
    const bool few = rows <= FEW_ROWS, mid = mid_tiles(s.V, rows);
    WeightTiles wt = weight_tiles(s, rows, p.pieces == 1);
    if (few) wt = {true, {(s.d + Mid::BM - 1) / Mid::BM * ((s.V + Mid::BN - 1) / Mid::BN), 0, 1, 0}, 0};          // together with d_hidden
    const Operand hidden = p.as_is ? Operand{h.hidden, h.hidden_stride * 2, 0, s.d} : Operand{hid, 2ull * s.Kd, 0, s.Kd};
    const LogitArgs la = {s, {weight, stride * 2, s.V, width}, hidden, meta, first, rows, target_of + first, p.as_is ? h.target : nullptr, (f32x2*)(ws + p.part),
                          few ? parts<Few>(s.V) : mid ? parts<Mid>(s.V) : parts<Big>(s.V), (float*)(ws + p.at_target),
                          p.grads ? ws + p.z : nullptr};
    rc = few ? logits<DT, Few>(la, st) : mid ? logits<DT, Mid>(la, st) : logits<DT, Big>(la, st);
    if (rc != PT_OK) return rc;
    const SoftArgs sa = {s, meta, first, rows, row_of + first, target_of + first, la.target, (const uint16_t*)h.hidden,
                         h.hidden_stride, packed, la.part, la.parts,
                         uint32_t(few ? Few::BM / Few::WM : mid ? Mid::BM / Mid::WM : Big::BM / Big::WM), la.at_target, h.row_scale, h.loss, ws + p.z,
                         (uint16_t*)(ws + p.g), p.g_pitch, (float*)(ws + p.rest), p.ordered ? (uint16_t*)(ws + p.rests) : nullptr};
    if (!p.grads) {
      hipLaunchKernelGGL(k_head_loss, dim3(rows), dim3(256), 0, st, sa);
      PT_LAUNCH_CHECK(nullptr, "k_head_loss");
      continue;
    }
    const uint32_t slices = p.g == p.z ? 1 : std::max(1u, std::min((s.Vp + 2047) / 2048, 512 / rows));
    hipLaunchKernelGGL(k_head_soft<DT>, dim3(uint32_t(up(rows, TWO)) + (p.as_is ? s.low : 0), slices), dim3(256), 0, st, sa);
    PT_LAUNCH_CHECK(nullptr, "k_head_soft");
    const GradArgs ga = {s, {weight, stride * 2, width, s.V}, {ws + p.g, p.g_pitch, 0, s.Vp}, meta, first, rows, row_of + first, target_of + first,
                   (uint16_t*)h.d_hidden, h.d_hidden_stride, (float*)(ws + p.sums), wt.split, sa.rest, sa.rests, ra.starts, weight, stride, (float*)(ws + p.acc), p.pitch,
                   i > 0, i + 1 < p.pieces};
    GradArgs gw = ga;
    gw.p = {hid, 2ull * s.Kd, s.Kd, 0};
    gw.q = {ws + p.g, p.g_pitch, s.Vp, 0};
    gw.out = (uint16_t*)h.d_weight;
    gw.stride = h.d_weight_stride;
    const Most most = h.d_hidden && rows != std::min(p.rows, s.R) ? most_hidden(s, rows) : p.hidden;          // a shorter last piece
    if (few && h.d_hidden && h.d_weight) {
      rc = few_grads<DT>(ga, gw, most, st);
      continue;
    }
    if (h.d_hidden)
      rc = few                  ? d_hidden<DT, Few>(ga, most, st)
           : mid_hidden(s, rows) ? d_hidden<DT, Mid>(ga, most, st)
                                 : d_hidden<DT, Big>(ga, most, st);
    if (h.d_weight && rc == PT_OK) rc = wt.mid ? d_weight<DT, Mid>(gw, st) : d_weight<DT, Big>(gw, st);
  }
  return rc;
}

}  // namespace

extern "C" int pt_head_workspace(const pt_head* head, uint64_t* least_bytes, uint64_t* best_bytes) {
  if (int rc = check(head, "pt_head_workspace"); rc != PT_OK) return rc;
  if (least_bytes) {
    // the smallest pieces as a rule, but one piece needs no sums of pieces
    uint64_t least = head->rows ? ~0ull : 0;
    for (uint64_t rows = PIECE_STEP; head->rows && rows <= best_rows(*head); rows += PIECE_STEP) least = std::min(least, make_plan(*head, rows).total);
    *least_bytes = least;
  }
  if (best_bytes) *best_bytes = head->rows ? make_plan(*head, best_rows(*head)).total : 0;
  return PT_OK;
}

extern "C" int pt_head_loss(const pt_head* head, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (int rc = check(head, "pt_head_loss"); rc != PT_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  if (!head->rows) {
    if (!head->d_weight) return PT_OK;
    hipLaunchKernelGGL(k_head_zero, dim3(head->vocab), dim3(256), 0, st, (uint16_t*)head->d_weight, head->d_weight_stride,
                       Shape{0, head->vocab, head->width, 0, 0, 0, 1});
    PT_LAUNCH_CHECK(nullptr, "k_head_zero");
    return PT_OK;
  }
  if (!workspace) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_head_loss: workspace is NULL");
  if ((uintptr_t)workspace % 256 != 0) return pt_fail(nullptr, PT_ERR_ALIGNMENT, "pt_head_loss: the workspace is not 256-byte aligned");
  // the largest pieces that fit
  uint64_t rows = best_rows(*head);
  Plan p = make_plan(*head, rows);
  while (p.total > workspace_bytes && rows > PIECE_STEP) p = make_plan(*head, rows -= PIECE_STEP);
  if (p.total > workspace_bytes)
    return pt_fail(nullptr, PT_ERR_NOMEM, "pt_head_loss: a workspace of %llu bytes is too small (pt_head_workspace)", (unsigned long long)workspace_bytes);
  return head->dtype == PT_BF16 ? run<PT_BF16>(*head, p, (char*)workspace, st) : run<PT_FP16>(*head, p, (char*)workspace, st);
}
