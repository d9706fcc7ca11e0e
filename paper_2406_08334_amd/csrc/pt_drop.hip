// Dropout with the residual's addition; no mask is stored: it is a function of seed, step and place.
//
//   out = residual + x m / (1 - p)
//
// Bound by memory: 4 bytes an element, 6 with a residual (32768 x 1600 in 53 us, 5.9 TB/s); a 64-bit word of random bits for four elements costs two products of 64
// bits, which hide behind that.  Rows of an odd width, a division a lane and lines in pieces: 32768 x 771 36 us, 4.2 TB/s.
#include "pt_random.h"
#include "pt_rows.h"

using namespace pt_rows_ops;

namespace {

struct DropArgs {
  const uint16_t *x, *residual;
  uint16_t* out;
  uint64_t x_stride, residual_stride, out_stride;
  pt_random::Drop drop;
  uint64_t n;                // pieces of eight elements, of all rows
  uint32_t width, pieces;    // of a row; pieces 0: the elements of all rows lie back to back, `flat` of them, and no word is shared by two rows
  uint64_t flat;
};

template <int DT>
__device__ __forceinline__ void drop8(const DropArgs& a, uint64_t key, uint64_t word, u32x4 x, u32x4 r, float (&y)[8]) {
  decode8<DT>(x, y);
  if (a.drop.off) {
#pragma unroll
    for (int h = 0; h < 2; ++h) a.drop.apply(key + (word + h + 1) * pt_random::PHI, y + 4 * h);
  }
  if (a.residual) {
    float b[8];
    decode8<DT>(r, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] += b[j];
  }
}

template <int DT>
__global__ void __launch_bounds__(256) k_dropout(const DropArgs a) {
  const uint64_t key = a.drop.key();
  const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.n) return;
  uint64_t row = 0, word;
  uint32_t c, left;
  if (a.pieces) {
    row = uint32_t(i) / a.pieces;
    c = (uint32_t(i) - uint32_t(row) * a.pieces) * 8;
    left = a.width - c;
    word = row * ((a.width - 1) / 4 + 1) + c / 4;
  } else {
    c = 0;
    left = uint32_t(a.flat - i * 8 < 8 ? a.flat - i * 8 : 8);
    word = i * 2;
  }
  const uint64_t at = a.pieces ? c : i * 8;
  const PT_GLOBAL uint16_t* x = (const PT_GLOBAL uint16_t*)a.x + row * a.x_stride + at;
  const u32x4 q = fetch8(x, 0, left);
  u32x4 r = {0, 0, 0, 0};
  if (a.residual) r = load8((const PT_GLOBAL uint16_t*)a.residual + row * a.residual_stride + at, 0, left);
  float y[8];
  drop8<DT>(a, key, word, q, r, y);
  pass8((PT_GLOBAL uint16_t*)a.out + row * a.out_stride + at, 0, left, encode8<DT>(y));
}

}  // namespace

extern "C" int pt_dropout(const pt_dropped* d, void* stream) {
  if (!d) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_dropout: dropped is NULL");
  if (d->dtype != PT_BF16 && d->dtype != PT_FP16) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_dropout: dtype %d is neither PT_BF16 nor PT_FP16", d->dtype);
  if (!d->width) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_dropout: width must be > 0");
  if (!pt_random::valid(d->drop)) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_dropout: p is not in [0, 1)");
  if (d->rows && (!d->x || !d->out)) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_dropout: NULL array");
  if (d->x_stride < d->width || d->out_stride < d->width || (d->residual && d->residual_stride < d->width))
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_dropout: rows of width %u at a smaller stride", d->width);
  if (((uintptr_t)d->x | (uintptr_t)d->out | (uintptr_t)d->residual) % 2 != 0 || (uintptr_t)d->drop.step % 8 != 0)
    return pt_fail(nullptr, PT_ERR_ALIGNMENT, "pt_dropout: an array is not aligned to its elements");
  const uint64_t pieces = (uint64_t(d->width) + 7) / 8;
  if (d->rows * pieces > 0xfffffc00ull)     // a lane each, of which a grid has less than 2^32
    return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "pt_dropout: more than 2^32 - 1024 pieces of eight elements");
  if (!d->rows) return PT_OK;
  DropArgs a = {(const uint16_t*)d->x, (const uint16_t*)d->residual, (uint16_t*)d->out, d->x_stride, d->residual_stride, d->out_stride,
                pt_random::make(d->drop), d->rows * pieces, d->width, uint32_t(pieces), 0};
  if (d->width % 4 == 0 && d->x_stride == d->width && d->out_stride == d->width && (!d->residual || d->residual_stride == d->width)) {
    a.flat = uint64_t(d->rows) * d->width;
    a.n = (a.flat + 7) / 8;
    a.pieces = 0;
  }
  const dim3 grid(uint32_t((a.n + 255) / 256));
  if (d->dtype == PT_BF16) hipLaunchKernelGGL(k_dropout<PT_BF16>, grid, dim3(256), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(k_dropout<PT_FP16>, grid, dim3(256), 0, (hipStream_t)stream, a);
  PT_LAUNCH_CHECK(nullptr, "k_dropout");
  return PT_OK;
}
