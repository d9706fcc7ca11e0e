// AdamW over a list of tensors at once, with states in 32 or in 8 bits: one launch for the norm of all gradients, one for the update.
//
// The update is that of the chunks (pt_update.h), bit for bit where the states have 32 bits.  States in 8 bits are blocks of 256 consecutive
// elements of a tensor: m and r = sqrt(v) as OCP e4m3 numbers times an fp32 scale, the block's largest magnitude / 448.  r, because its
// range is half of v's in powers of two: e4m3 numbers reach from 448 down to 2^-9, and an r 2^-18 below its block's largest is as good as
// the smallest code.  A wave holds a block, four elements a lane, so the largest magnitude is a tree over lanes and the state is read and
// written once: 16.06 bytes an element (gradient 2, master 8, parameter 2, states 4, scales 0.06) instead of 28.
//
// States are rounded up or down at random with the odds that keep their mean.  To the nearest, an average that moves by less than half a
// code's distance (6 %) a step, all of them with beta near 1, would stay where it is for good.  The 16 random bits of a state are a function of the
// list's seed, the number of the update and the element's place (splitmix64 of a counter: Steele, Lea, Flood, 2014), so a run can be repeated.
// What is not zero keeps an r of one code at least: an m beside an r of zero would be divided by eps alone.
#include "pt_common.h"
#include "pt_scalars.h"
#include "pt_update.h"

#include <algorithm>
#include <memory>

#pragma clang fp contract(off)

namespace {

typedef pt_f32x4 f32x4;
typedef pt_u32x2 u32x2;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// global memory takes these at any address of an element
typedef f32x4 f32x4_a __attribute__((aligned(4)));
typedef u32x2 u32x2_a __attribute__((aligned(2)));
typedef u32x4 u32x4_a __attribute__((aligned(2)));

constexpr uint32_t BLOCK = 256;              // elements of a block: a wave's, and those that share a scale
constexpr uint32_t UNIT = 4096;              // elements a wave of the norm takes at a time
constexpr uint32_t COARSE = 16;              // blocks / units per entry of the look-up tables
constexpr uint32_t NORM_THREADS = 256, NORM_BLOCKS = 512, NORM_WAVES = NORM_THREADS / 64;

constexpr uint32_t ALIGNED = 1u << 31;       // of Desc::flags: a block's arrays begin at multiples of what a lane stores

// One tensor as the kernels read it.  With states in 32 bits its blocks lie on the 128-byte lines of the master array, the first one up to 31 elements
// early: the addresses are those of that block's beginning, and `elems` counts the `early` ones in.  (4 blocks of width 771 back to back in flat
// buffers, 6.7e7 parameters: 360 -> 330 us.)
struct Desc {
  uint64_t grad, master, param, m, v, ms, vs, elems;
  uint32_t flags, early;
};

struct ListState {
  PtDevState s;
  // of the update in flight: 1 - beta1^t and its reciprocal, 1 / sqrt(1 - beta2^t), norm + 1e-6 and 1 / it, 1 / loss scale
  double bc1, inv_bc1, norm_eps, inv_norm, inv_scale;
  float rsb2;
  uint64_t key;          // of its random numbers
  uint32_t applied;      // the update of the norm before has been enqueued: the next norm ends its step first
};

// Which tensor owns block or unit i: a table entry per COARSE of them says where to begin.
// Tables and descriptions are written before the first launch: loads of the scalar cache, which no store of the update holds up.
struct Index { const PT_SCALAR uint32_t* first; const PT_SCALAR uint32_t* coarse; uint32_t n; };
__device__ __forceinline__ uint32_t owner(const Index& x, uint32_t i) {
  uint32_t t = x.coarse[i / COARSE];
  while (i >= x.first[t + 1]) ++t;
  return t;
}
__device__ __forceinline__ Desc describe(const PT_SCALAR Desc* at) {
  return {at->grad, at->master, at->param, at->m, at->v, at->ms, at->vs, at->elems, at->flags, at->early};
}

__device__ __forceinline__ uint64_t mix64(uint64_t x) {
  x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9ull;
  x = (x ^ (x >> 27)) * 0x94D049BB133111EBull;
  return x ^ (x >> 31);
}
constexpr uint64_t PHI = 0x9E3779B97F4A7C15ull;

// ---- norm --------------------------------------------------------------------------------------------

template <int DT>
__device__ __forceinline__ void take8(const u32x4& q, double& a0, double& a1) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const double x = decode16<DT>(q[k] & 0xffffu), y = decode16<DT>(q[k] >> 16);
    a0 = fma(x, x, a0);
    a1 = fma(y, y, a1);
  }
}

struct NormArgs {
  Index units;
  const PT_SCALAR Desc* desc;
  ListState* st;
  double* part;
  double beta1, beta2;
  uint64_t seed;
};

// Sum of squares of every gradient in a fixed order: waves take units in turn, the last workgroup to finish adds the workgroups' sums up in
// order, ends the step before and opens this one.  Reading bounds it (667e6 fp16 gradients: 205 us, 6.5 TB/s), of short lists the round trips of the hand-over
// (0.8e6: 6.7 us).  Two workgroups a compute unit: with one, or four, a step of 667e6 takes 3.12 - 3.25 or 3.07 - 3.20 ms instead of 3.05, of 67e6 334 or 333 us
// instead of 326; that many sums are also all the last one adds up.
template <int DT>
__global__ void __launch_bounds__(NORM_THREADS) k_list_norm(const NormArgs a) {
  const uint32_t lane = threadIdx.x & 63;
  double a0 = 0.0, a1 = 0.0;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * NORM_WAVES + (threadIdx.x >> 6));
  for (uint32_t i = wave; i < a.units.n; i += gridDim.x * NORM_WAVES) {
    const uint32_t u = a.units.n - 1 - i;           // from the far end: the update, which begins at the near one, finds that in the cache
    const uint32_t t = owner(a.units, u);
    const Desc d = describe(a.desc + t);
    const uint64_t at = uint64_t(u - a.units.first[t]) * UNIT;
    const uint32_t len = uint32_t(min(uint64_t(UNIT), d.elems - d.early - at));
    if (d.flags & PT_TENSOR_GRAD_F32) {
      const PT_GLOBAL float* g = (const PT_GLOBAL float*)d.grad + d.early + at;
      const uint32_t whole = len / 4;
#pragma unroll 8
      for (uint32_t k = lane; k < whole; k += 64) {
        const f32x4 q = *(const PT_GLOBAL f32x4_a*)(g + 4 * k);
#pragma unroll
        for (int j = 0; j < 4; ++j) { const double x = q[j]; if (j & 1) a1 = fma(x, x, a1); else a0 = fma(x, x, a0); }
      }
      if (4 * whole + lane < len) { const double x = g[4 * whole + lane]; a0 = fma(x, x, a0); }
    } else {
      const PT_GLOBAL uint16_t* g = (const PT_GLOBAL uint16_t*)d.grad + d.early + at;
      const uint32_t whole = len / 8;
      if (len == UNIT) {
        u32x4 q[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = *(const PT_GLOBAL u32x4_a*)(g + 8 * (lane + 64 * k));
#pragma unroll
        for (int k = 0; k < 8; ++k) take8<DT>(q[k], a0, a1);
      } else {
        for (uint32_t k = lane; k < whole; k += 64) {
          const u32x4 q = *(const PT_GLOBAL u32x4_a*)(g + 8 * k);
          take8<DT>(q, a0, a1);
        }
        if (8 * whole + lane < len) { const double x = decode16<DT>(g[8 * whole + lane]); a0 = fma(x, x, a0); }
      }
    }
  }
  double sum = a0 + a1;
  uint32_t none = 0;
  __shared__ uint32_t s_last;
  pt_block_sum(sum, none);
  if (threadIdx.x == 0) {
    st_agent(a.part + blockIdx.x, sum);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    s_last = __hip_atomic_fetch_add(&a.st->s.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1 ? 1u : 0u;
  }
  __syncthreads();
  if (!s_last) return;
  PtDevState s = a.st->s;
  if (a.st->applied) pt_advance(s, s.found_inf != 0);
  // the powers of beta while the sums are on their way
  const double bc = threadIdx.x < 2 ? 1.0 - pow(threadIdx.x ? a.beta2 : a.beta1, double(s.step + 1)) : 0.0;
  sum = 0.0;
  for (uint32_t k = threadIdx.x; k < gridDim.x; k += NORM_THREADS) sum += ld_agent(a.part + k);
  pt_block_sum(sum, none);
  if (threadIdx.x == 1) a.st->rsb2 = float(1.0 / sqrt(bc));
  if (threadIdx.x != 0) return;
  uint32_t inf;
  double sq;
  pt_close_sum(sum, 1.0 / s.loss_scale, sq, inf);
  s.sqnorm = sq;
  s.norm = sqrt(sq);
  s.found_inf = inf ? 1 : 0;
  s.skip = s.found_inf;
  s.ticket = 0;
  a.st->s = s;
  a.st->bc1 = bc;
  a.st->inv_bc1 = 1.0 / bc;
  a.st->norm_eps = s.norm + 1e-6;
  a.st->inv_norm = 1.0 / (s.norm + 1e-6);
  a.st->inv_scale = 1.0 / s.loss_scale;
  a.st->key = mix64(a.seed + uint64_t(uint32_t(s.step) + 1u) * PHI);
  a.st->applied = 0;
}

// The powers for an update whose betas are not those the norm was taken with.
__global__ void k_list_betas(ListState* st, double beta1, double beta2) {
  if (threadIdx.x > 1) return;
  const double bc = 1.0 - pow(threadIdx.x ? beta2 : beta1, double(st->s.step + 1));
  if (threadIdx.x) st->rsb2 = float(1.0 / sqrt(bc));
  else { st->bc1 = bc; st->inv_bc1 = 1.0 / bc; }
}

__global__ void k_list_set(ListState* st, int32_t step, double loss_scale, int32_t good_steps) {
  st->s.step = step; st->s.loss_scale = loss_scale; st->s.good_steps = good_steps;
  st->applied = 0;
}

// ---- update ------------------------------------------------------------------------------------------

struct UpdateArgs {
  Index blocks;
  const PT_SCALAR Desc* desc;
  ListState* st;
  double lr, max_norm;
  float c[8];                // the constants that neither norm nor counter enter; [5], [6]: not used
};

// a / b, correctly rounded, from inv = 1 / b correctly rounded (Markstein: one step on the remainder).
__device__ __forceinline__ double quotient(double a, double b, double inv) {
  const double q = a * inv;
  return fma(fma(-q, b, a), inv, q);
}

// The nine constants of the update, in every wave, from the few numbers that the norm has left.
__device__ __forceinline__ Consts list_consts(const UpdateArgs& a, double& clip) {
  const PT_SCALAR ListState& st = *(const PT_SCALAR ListState*)a.st;       // the norm's launch has written all that is read here
  clip = 1.0;
  if (a.max_norm > 0.0) {
    const double q = quotient(a.max_norm, st.norm_eps, st.inv_norm);
    clip = q < 1.0 ? q : 1.0;
  }
  return {a.c[0], a.c[1], a.c[2], a.c[3], a.c[4], float(quotient(a.lr, st.bc1, st.inv_bc1)), st.rsb2, a.c[7],
          float(quotient(clip, st.s.loss_scale, st.inv_scale))};
}

constexpr float TOP8 = 448.0f, TINY8 = 0x1p-100f, LOW8 = 0x1p-9f;        // largest and smallest number of the format; blocks of less than TINY8 are zero
// An r is kept up to here: its square, a last place or two off by its scale, is an fp32 number still.  Were it inf, its block's others, one code at least
// of a scale as large, would have squares of inf too, for good.
constexpr float MOST_R = 0x1.ffffp63f;

// Largest of x over the wave (of numbers >= 0), in every lane: in four steps over the 16 lanes of a row, then over the rows.
template <int CTRL> __device__ __forceinline__ float dpp_max(float x) {
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false)));
}
__device__ __forceinline__ float wave_max(float x) {
  x = dpp_max<0xb1>(x);          // lane ^ 1
  x = dpp_max<0x4e>(x);          // lane ^ 2
  x = dpp_max<0x141>(x);         // mirrored in eight
  x = dpp_max<0x140>(x);         // mirrored in 16
  const int i = __float_as_int(x);
  const float a = __int_as_float(__builtin_amdgcn_readlane(i, 0)), b = __int_as_float(__builtin_amdgcn_readlane(i, 16));
  const float c = __int_as_float(__builtin_amdgcn_readlane(i, 32)), d = __int_as_float(__builtin_amdgcn_readlane(i, 48));
  return fmaxf(fmaxf(a, b), fmaxf(c, d));
}

// sqrt of a number >= 0, rounded to the nearest but for one in some millions (x of normal size): the reciprocal root is right to its last
// place, one step on the remainder.  Of inf, a variance that no fp32 number holds, inf: the step would have inf times 0 in it.
__device__ __forceinline__ float root(float x) {
  const float y = __builtin_amdgcn_rsqf(x), s = x * y;
  const float r = __builtin_fmaf(__builtin_fmaf(-s, s, x), 0.5f * y, s);
  return x > 0x1p-100f ? (x < __builtin_inff() ? r : x) : __builtin_sqrtf(x);
}

// The update with states in 8 bits: as update_element, but every product is rounded before it is added.  A code is a threshold on m and r, and a
// difference in their last bit turns over one in a million of them, each by 6 % or more; so the two averages are what any plain evaluation
// in fp32 gives.  The quotient is good to two units in the last place: nothing but w depends on it.
__device__ __forceinline__ void update_element8(const Consts& k, float decay, float g, float& w, float& m, float& v, float& s) {
  g = g * k.gm;
  const float m1 = k.b1 * m, m2 = k.omb1 * g;
  m = m1 + m2;
  float v2 = k.omb2 * g;
  v2 = v2 * g;
  const float v1 = k.b2 * v;
  v = v1 + v2;
  s = root(v);
  const float d = __builtin_fmaf(s, k.rsb2, k.eps);
  const float u = m * __builtin_amdgcn_rcpf(d);
  w = __builtin_fmaf(-k.step_size, u, w * decay);
}

// A lane's four codes; policy as pt_store.
__device__ __forceinline__ void store_word(PT_GLOBAL uint8_t* base, uint32_t x) {
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(uintptr_t)base, 0, 0xffffffffu, 0x27000);
  __builtin_amdgcn_raw_buffer_store_b32(x, r, 4 * threadIdx.x, 0, PT_NT_THROUGH);
}

// Four e4m3 numbers.
__device__ __forceinline__ f32x4 decode8(uint32_t codes, float scale) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(codes), true);
  return f32x4{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
}

// A block of 256 elements, four a lane, as they lie in memory.
template <int DT, int BITS>
struct Block {
  Desc d;
  uint32_t nb, lo, len;      // number of the block in its tensor; its elements: from lo to len
  f32x4 w, m, v, g32;        // m, v: of states in 32 bits; g32 or g16, as the tensor's gradient is
  u32x2 g16;
  uint32_t cm, cv;           // codes
  float ms, vs;

  __device__ __forceinline__ bool whole() const { return len == BLOCK && lo == 0; }
  template <class P> __device__ __forceinline__ P at(uint64_t base) const { return (P)base + uint64_t(nb) * BLOCK + threadIdx.x * 4; }

  // Loads block b, with hints but for the gradient, which the norm has just read.
  __device__ __forceinline__ void load(const UpdateArgs& a, uint32_t b) {
    const uint32_t t = owner(a.blocks, b);
    d = describe(a.desc + t);
    nb = b - a.blocks.first[t];
    const uint64_t left = d.elems - uint64_t(nb) * BLOCK;
    len = left < BLOCK ? uint32_t(left) : BLOCK;
    lo = BITS == 32 && nb == 0 ? d.early : 0;
    const auto pw = at<const PT_GLOBAL float*>(d.master);
    const auto pg = at<const PT_GLOBAL uint16_t*>(d.grad);
    const auto pg32 = at<const PT_GLOBAL float*>(d.grad);
    const auto pm = at<const PT_GLOBAL float*>(d.m), pv = at<const PT_GLOBAL float*>(d.v);
    const auto pm8 = at<const PT_GLOBAL uint8_t*>(d.m), pv8 = at<const PT_GLOBAL uint8_t*>(d.v);
    if (whole()) {
      if (d.flags & PT_TENSOR_GRAD_F32) g32 = *(const PT_GLOBAL f32x4_a*)pg32;
      else g16 = *(const PT_GLOBAL u32x2_a*)pg;
      w = __builtin_nontemporal_load((const PT_GLOBAL f32x4_a*)pw);
      if constexpr (BITS == 8) {
        cm = __builtin_nontemporal_load((const PT_GLOBAL uint32_t*)pm8);
        cv = __builtin_nontemporal_load((const PT_GLOBAL uint32_t*)pv8);
      } else {
        m = __builtin_nontemporal_load((const PT_GLOBAL f32x4_a*)pm);
        v = __builtin_nontemporal_load((const PT_GLOBAL f32x4_a*)pv);
      }
    } else {
      w = m = v = g32 = f32x4{};
      g16 = u32x2{};
      cm = cv = 0;
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j)
        if (threadIdx.x * 4 + j >= lo && threadIdx.x * 4 + j < len) {
          if (d.flags & PT_TENSOR_GRAD_F32) g32[j] = pg32[j];
          else g16[j / 2] |= uint32_t(pg[j]) << (16 * (j & 1));
          w[j] = pw[j];
          if constexpr (BITS == 8) { cm |= uint32_t(pm8[j]) << (8 * j); cv |= uint32_t(pv8[j]) << (8 * j); }
          else { m[j] = pm[j]; v[j] = pv[j]; }
        }
    }
    if constexpr (BITS == 8) { ms = ((const PT_GLOBAL float*)d.ms)[nb]; vs = ((const PT_GLOBAL float*)d.vs)[nb]; }
  }

  // Updates and stores it.  counter: of the random numbers of the lane's first pair of elements.
  __device__ __forceinline__ void finish(const Consts& k, uint64_t counter) {
    const float decay = d.flags & PT_TENSOR_NO_DECAY ? 1.0f : k.decay;
    f32x4 g;
    if (d.flags & PT_TENSOR_GRAD_F32) g = g32;
    else g = f32x4{decode16<DT>(g16.x & 0xffffu), decode16<DT>(g16.x >> 16), decode16<DT>(g16.y & 0xffffu), decode16<DT>(g16.y >> 16)};
    if constexpr (BITS == 8) {
      m = decode8(cm, ms);
      v = decode8(cv, vs);
      v = v * v;
    }
    float r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float wj = w[j], mj = m[j], vj = v[j];
      if constexpr (BITS == 8) update_element8(k, decay, g[j], wj, mj, vj, r[j]);
      else update_element(k, decay, g[j], wj, mj, vj, r[j]);
      w[j] = wj; m[j] = mj; v[j] = vj;
    }
    const u32x2 p2 = encode16x4<DT>(w);
    if constexpr (BITS == 8) {
      const float bm = fminf(wave_max(fmaxf(fmaxf(__builtin_fabsf(m[0]), __builtin_fabsf(m[1])), fmaxf(__builtin_fabsf(m[2]), __builtin_fabsf(m[3])))),
                             3.402823466e38f);
      const float bv = fminf(wave_max(fmaxf(fmaxf(r[0], r[1]), fmaxf(r[2], r[3]))), MOST_R);
      // the reciprocal first, and the scale by a product: what an elementwise evaluation of top / largest and largest / top makes of them
      const bool hm = bm >= TINY8, hv = bv >= TINY8;
      const float im = hm ? 1.0f / bm * TOP8 : 0.0f, iv = hv ? 1.0f / bv * TOP8 : 0.0f;
      uint32_t z[4];
      {
        const uint64_t z0 = mix64(counter), z1 = mix64(counter + PHI);
        z[0] = uint32_t(z0); z[1] = uint32_t(z0 >> 32); z[2] = uint32_t(z1); z[3] = uint32_t(z1 >> 32);
      }
      int qm = 0, qv = 0;
#define PT_CODE(j)                                                                                                                  \
      {                                                                                                                             \
        const float ym = __builtin_amdgcn_fmed3f(m[j] * im, -TOP8, TOP8), y = r[j] * iv;                                            \
        const float yv = __builtin_amdgcn_fmed3f(y, y > 0.0f ? LOW8 : 0.0f, TOP8);                                                  \
        qm = __builtin_amdgcn_cvt_sr_fp8_f32(ym, int(z[j] << 16 | 0x8000u), qm, j);                                                 \
        qv = __builtin_amdgcn_cvt_sr_fp8_f32(yv, int((z[j] & 0xffff0000u) | 0x8000u), qv, j);                                       \
      }
      PT_CODE(0) PT_CODE(1) PT_CODE(2) PT_CODE(3)
#undef PT_CODE
      cm = uint32_t(qm); cv = uint32_t(qv);
      if (threadIdx.x == 0) {
        ((PT_GLOBAL float*)d.ms)[nb] = hm ? bm * (1.0f / TOP8) : 0.0f;
        ((PT_GLOBAL float*)d.vs)[nb] = hv ? bv * (1.0f / TOP8) : 0.0f;
      }
    }
    const auto pw = at<PT_GLOBAL float*>(d.master);
    const auto pp = at<PT_GLOBAL uint16_t*>(d.param);
    const auto pm = at<PT_GLOBAL float*>(d.m), pv = at<PT_GLOBAL float*>(d.v);
    const auto pm8 = at<PT_GLOBAL uint8_t*>(d.m), pv8 = at<PT_GLOBAL uint8_t*>(d.v);
    if (whole() && (d.flags & ALIGNED)) {
      const uint64_t e = uint64_t(nb) * BLOCK;
      pt_store<PT_NT_THROUGH>(w, (PT_GLOBAL float*)d.master + e, 16 * threadIdx.x);
      if (d.param) pt_store<PT_NT_THROUGH>(p2, (PT_GLOBAL uint16_t*)d.param + e, 8 * threadIdx.x);
      if constexpr (BITS == 8) {
        store_word((PT_GLOBAL uint8_t*)d.m + e, cm);
        store_word((PT_GLOBAL uint8_t*)d.v + e, cv);
      } else {
        pt_store<PT_NT_THROUGH>(m, (PT_GLOBAL float*)d.m + e, 16 * threadIdx.x);
        pt_store<PT_NT_THROUGH>(v, (PT_GLOBAL float*)d.v + e, 16 * threadIdx.x);
      }
      return;
    }
    if (whole()) {
      __builtin_nontemporal_store(w, (PT_GLOBAL f32x4_a*)pw);
      if (d.param) __builtin_nontemporal_store(p2, (PT_GLOBAL u32x2_a*)pp);
      if constexpr (BITS == 8) {
        __builtin_nontemporal_store(cm, (PT_GLOBAL uint32_t*)pm8);
        __builtin_nontemporal_store(cv, (PT_GLOBAL uint32_t*)pv8);
      } else {
        __builtin_nontemporal_store(m, (PT_GLOBAL f32x4_a*)pm);
        __builtin_nontemporal_store(v, (PT_GLOBAL f32x4_a*)pv);
      }
      return;
    }
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
      if (threadIdx.x * 4 + j >= lo && threadIdx.x * 4 + j < len) {
        pw[j] = w[j];
        if (d.param) pp[j] = uint16_t(p2[j / 2] >> (16 * (j & 1)));
        if constexpr (BITS == 8) { pm8[j] = uint8_t(cm >> (8 * j)); pv8[j] = uint8_t(cv >> (8 * j)); }
        else { pm[j] = m[j]; pv[j] = v[j]; }
      }
  }
};

// Blocks along x of a launch at most: its threads along x have to be less than 2^32.  More lie in rows of one length: workgroups without a block cost too.
constexpr uint32_t LAUNCH = 1u << 22;

// A wave a block, in the order of the list.  The bytes of memory bound it: 667e6 parameters, fp16, states in 32 bits 2.86 - 2.98 ms, 6.3 - 6.5 TB/s; 1.56e9,
// bf16, states in 8 bits 4.0 ms, 6.2 TB/s.  States in 32 bits: as for the chunks, few bytes in flight that lie next to each other are moved fastest, so
// unused LDS keeps a compute unit to 11 waves (2.46e8 parameters 1183 -> 1156 us, 6.3e6 42.2 -> 41.0) but for a short list, most of which is under way
// at once (without: 0.8e6 13.6 -> 12.5 us, 3.1e6 25.5 -> 24.8).  States in 8 bits have little more than half the bytes to an update and their own
// arithmetic: as many waves as there is room for (1.56e9, step with its norm: 4.47 ms; kept to 11 waves 7.0).
constexpr uint32_t SHORT = 16384;
template <int DT, int BITS>
__global__ void __launch_bounds__(64) k_list_adamw(const UpdateArgs a) {
  const PT_SCALAR ListState* st = (const PT_SCALAR ListState*)a.st;
  Block<DT, BITS> x;
  const uint32_t b = blockIdx.y * gridDim.x + blockIdx.x;
  if (b >= a.blocks.n) return;
  x.load(a, b);                                // a skipped step reads in vain
  asm volatile("" ::: "memory");
  double clip;
  const Consts k = list_consts(a, clip);
  if (b == 0 && threadIdx.x == 0) {            // what no other workgroup reads
    a.st->applied = 1;
    a.st->s.clip_coef = clip;
    const float c[9] = {k.b1, k.b2, k.omb1, k.omb2, k.decay, k.step_size, k.rsb2, k.eps, k.gm};
#pragma unroll
    for (int j = 0; j < 9; ++j) a.st->s.c[j] = c[j];
  }
  if (st->s.skip) return;
  x.finish(k, st->key + PHI * (uint64_t(b) * (BLOCK / 2) + 2 * threadIdx.x + 1));
}

// The update of a list without an element: its step has happened.
__global__ void k_list_applied(ListState* st) { st->applied = 1; st->s.clip_coef = 1.0; }

// Tables of an Index over `counts` pieces of every tensor.
void build_index(const std::vector<uint64_t>& counts, std::vector<uint32_t>& first, std::vector<uint32_t>& coarse) {
  first.assign(1, 0);
  for (uint64_t c : counts) first.push_back(uint32_t(first.back() + c));
  coarse.assign(size_t(first.back() / COARSE) + 1, 0);
  uint32_t t = 0;
  for (uint32_t i = 0; i < first.back(); i += COARSE) {
    while (i >= first[t + 1]) ++t;
    coarse[i / COARSE] = t;
  }
}

}  // namespace

struct pt_tensors {
  int dtype = PT_BF16, bits = 32;
  bool scaler = false;
  int device = 0;
  uint64_t seed = 0;
  Index units{}, blocks{};
  uint32_t norm_grid = 0;
  bool open = false;                      // a norm has been taken that no update has used
  double beta1 = 0.9, beta2 = 0.95;       // those whose powers the device has
  double next_beta1 = 0.9, next_beta2 = 0.95;
  uint8_t* mem = nullptr;                 // everything below lies in it
  ListState* st = nullptr;
  double* part = nullptr;
  const PT_SCALAR Desc* desc = nullptr;
};

namespace {

int create(pt_tensors* l, const pt_tensor* list, uint32_t n, const pt_scaler_cfg* cfg) {
  const char* who = "pt_tensors_create";
  const bool q = l->bits == 8;
  std::vector<Desc> desc;
  std::vector<uint64_t> nb, nu;
  uint64_t blocks = 0;
  for (uint32_t i = 0; i < n; ++i) {
    const pt_tensor& t = list[i];
    if (t.flags & ~(PT_TENSOR_NO_DECAY | PT_TENSOR_GRAD_F32))
      return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: tensor %u has unknown flags", who, i);
    if (!t.elems) continue;                             // owns no block; its pointers are not looked at
    if (!t.grad || !t.master || !t.m || !t.v || (q && (!t.m_scale || !t.v_scale)))
      return pt_fail(nullptr, PT_ERR_INVALID_ARG, "%s: NULL array of tensor %u", who, i);
    const uintptr_t at32 = (uintptr_t)t.master | (uintptr_t)t.m | (uintptr_t)t.v |
                           (q ? (uintptr_t)t.m_scale | (uintptr_t)t.v_scale : 0) | (t.flags & PT_TENSOR_GRAD_F32 ? (uintptr_t)t.grad : 0);
    if (at32 % 4 != 0 || ((uintptr_t)t.grad | (uintptr_t)t.param16) % 2 != 0)
      return pt_fail(nullptr, PT_ERR_ALIGNMENT, "%s: tensor %u: 16-bit arrays need 2-byte, all others 4-byte alignment", who, i);
    const uint32_t early = q ? 0 : uint32_t((uintptr_t)t.master >> 2) & 31;
    const uint64_t e4 = 4ull * early, e2 = 2ull * early, master = (uint64_t)t.master - e4, m = (uint64_t)t.m - e4, v = (uint64_t)t.v - e4;
    const uint64_t param = t.param16 ? (uint64_t)t.param16 - e2 : 0;
    const bool aligned = (master | (q ? 0 : m | v)) % 16 == 0 && param % 8 == 0;
    desc.push_back({(uint64_t)t.grad - (t.flags & PT_TENSOR_GRAD_F32 ? e4 : e2), master, param, m, v, (uint64_t)t.m_scale, (uint64_t)t.v_scale,
                    t.elems + early, t.flags | (aligned ? ALIGNED : 0), early});
    if (t.elems > (uint64_t(1) << 40)) return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "%s: tensor %u has more than 2^40 elements", who, i);
    nb.push_back((t.elems + early + BLOCK - 1) / BLOCK);
    nu.push_back((t.elems + UNIT - 1) / UNIT);
    blocks += nb.back();
    if (blocks > 0x7fffffffu) return pt_fail(nullptr, PT_ERR_UNSUPPORTED, "%s: more than 2^31 blocks of 256 elements", who);
  }
  std::vector<uint32_t> bf, bc, uf, uc;
  build_index(nb, bf, bc);
  build_index(nu, uf, uc);
  l->blocks.n = bf.back();
  l->units.n = uf.back();
  l->norm_grid = std::min(NORM_BLOCKS, std::max(1u, (l->units.n + NORM_WAVES - 1) / NORM_WAVES));
  // one allocation: state, partial sums, descriptions, tables
  const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  const size_t o_part = up(sizeof(ListState)), o_desc = o_part + up(NORM_BLOCKS * sizeof(double)), o_bf = o_desc + up(desc.size() * sizeof(Desc)),
               o_bc = o_bf + up(bf.size() * 4), o_uf = o_bc + up(bc.size() * 4), o_uc = o_uf + up(uf.size() * 4), total = o_uc + up(uc.size() * 4);
  std::vector<uint8_t> host(total, 0);
  ListState st{};
  st.s.clip_coef = 1.0;
  st.s.loss_scale = cfg ? cfg->init_scale : 1.0;
  st.s.growth = cfg ? cfg->growth : 1.0;
  st.s.backoff = cfg ? cfg->backoff : 1.0;
  st.s.growth_interval = cfg ? cfg->growth_interval : 1;
  st.s.scaler_enabled = cfg ? 1 : 0;
  std::memcpy(host.data(), &st, sizeof st);
  if (!desc.empty()) std::memcpy(host.data() + o_desc, desc.data(), desc.size() * sizeof(Desc));
  std::memcpy(host.data() + o_bf, bf.data(), bf.size() * 4);
  std::memcpy(host.data() + o_bc, bc.data(), bc.size() * 4);
  std::memcpy(host.data() + o_uf, uf.data(), uf.size() * 4);
  std::memcpy(host.data() + o_uc, uc.data(), uc.size() * 4);
  PT_HIP(nullptr, hipGetDevice(&l->device));
  PT_HIP(nullptr, hipMalloc((void**)&l->mem, total));
  PT_HIP(nullptr, hipMemcpy(l->mem, host.data(), total, hipMemcpyHostToDevice));
  l->st = (ListState*)l->mem;
  l->part = (double*)(l->mem + o_part);
  l->desc = (const PT_SCALAR Desc*)(l->mem + o_desc);
  l->blocks.first = (const PT_SCALAR uint32_t*)(l->mem + o_bf);
  l->blocks.coarse = (const PT_SCALAR uint32_t*)(l->mem + o_bc);
  l->units.first = (const PT_SCALAR uint32_t*)(l->mem + o_uf);
  l->units.coarse = (const PT_SCALAR uint32_t*)(l->mem + o_uc);
  return PT_OK;
}

}  // namespace

extern "C" int pt_tensors_create(pt_tensors** out, int dtype, const pt_tensor* list, uint32_t n_tensors, int state_bits,
                                 const pt_scaler_cfg* scaler, uint64_t seed) {
  if (!out) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_create: out is NULL");
  *out = nullptr;
  if (dtype != PT_BF16 && dtype != PT_FP16)
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_create: dtype %d is neither PT_BF16 nor PT_FP16", dtype);
  if (state_bits != 8 && state_bits != 32)
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_create: states have 8 or 32 bits, not %d", state_bits);
  if (!list && n_tensors) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_create: list is NULL");
  if (scaler && (!(scaler->init_scale >= 1.0) || !(scaler->growth >= 1.0) || !(scaler->backoff > 0.0) || !(scaler->backoff <= 1.0) ||
                 scaler->growth_interval < 1))
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_create: scaler needs init_scale >= 1, growth >= 1, 0 < backoff <= 1, "
                   "growth_interval >= 1");
  return pt_guarded(nullptr, "pt_tensors_create", [&] {
    std::unique_ptr<pt_tensors> l(new pt_tensors());
    l->dtype = dtype;
    l->bits = state_bits;
    l->scaler = scaler != nullptr;
    l->seed = seed;
    const int rc = create(l.get(), list, n_tensors, scaler);
    if (rc != PT_OK) {
      if (l->mem) (void)hipFree(l->mem);
      return rc;
    }
    *out = l.release();
    return int(PT_OK);
  });
}

extern "C" int pt_tensors_destroy(pt_tensors* l) {
  if (!l) return PT_OK;
  // its own device's work, whichever is current
  int current = l->device;
  (void)hipGetDevice(&current);
  if (current != l->device) (void)hipSetDevice(l->device);
  (void)hipDeviceSynchronize();
  if (l->mem) (void)hipFree(l->mem);
  if (current != l->device) (void)hipSetDevice(current);
  delete l;
  return PT_OK;
}

extern "C" int pt_tensors_set_state(pt_tensors* l, int32_t step, double loss_scale, int32_t good_steps, void* stream) {
  if (!l) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_set_state: NULL list");
  if (step < 0 || good_steps < 0 || !(loss_scale >= 1.0))
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_set_state: step, good_steps >= 0 and loss_scale >= 1 required");
  if (!l->scaler && loss_scale != 1.0)
    return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_set_state: list has no scaler, loss_scale must be 1");
  hipLaunchKernelGGL(k_list_set, dim3(1), dim3(1), 0, (hipStream_t)stream, l->st, step, loss_scale, good_steps);
  PT_LAUNCH_CHECK(nullptr, "k_list_set");
  l->open = false;                        // a norm was taken under the old loss scale
  return PT_OK;
}

extern "C" int pt_tensors_grad_sqnorm(pt_tensors* l, void* stream) {
  if (!l) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_grad_sqnorm: NULL list");
  l->beta1 = l->next_beta1;
  l->beta2 = l->next_beta2;
  const NormArgs a = {l->units, l->desc, l->st, l->part, l->beta1, l->beta2, l->seed};
  hipLaunchKernelGGL(l->dtype == PT_BF16 ? k_list_norm<PT_BF16> : k_list_norm<PT_FP16>, dim3(l->norm_grid), dim3(NORM_THREADS), 0,
                     (hipStream_t)stream, a);
  PT_LAUNCH_CHECK(nullptr, "k_list_norm");
  l->open = true;
  return PT_OK;
}

extern "C" int pt_tensors_adamw_step(pt_tensors* l, const pt_hparams* hp, void* stream) {
  if (!l || !hp) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_adamw_step: NULL argument");
  if (!l->open)
    return pt_fail(nullptr, PT_ERR_STATE, "pt_tensors_adamw_step: no norm has been taken since the last update (pt_tensors_grad_sqnorm)");
  if (hp->beta1 != l->beta1 || hp->beta2 != l->beta2) {
    hipLaunchKernelGGL(k_list_betas, dim3(1), dim3(64), 0, (hipStream_t)stream, l->st, hp->beta1, hp->beta2);
    PT_LAUNCH_CHECK(nullptr, "k_list_betas");
    l->beta1 = l->next_beta1 = hp->beta1;
    l->beta2 = l->next_beta2 = hp->beta2;
  }
  const UpdateArgs a = {l->blocks, l->desc, l->st, hp->lr, hp->max_norm,
                        {float(hp->beta1), float(hp->beta2), float(1.0 - hp->beta1), float(1.0 - hp->beta2),
                         float(1.0 - hp->lr * hp->weight_decay), 0.0f, 0.0f, float(hp->eps)}};
  const auto kernel = l->dtype == PT_BF16 ? (l->bits == 8 ? k_list_adamw<PT_BF16, 8> : k_list_adamw<PT_BF16, 32>)
                                          : (l->bits == 8 ? k_list_adamw<PT_FP16, 8> : k_list_adamw<PT_FP16, 32>);
  const uint32_t rows = (l->blocks.n + LAUNCH - 1) / LAUNCH;
  const uint32_t lds = l->bits == 8 || l->blocks.n <= SHORT ? 0 : PT_ADAMW_LDS;
  if (l->blocks.n) hipLaunchKernelGGL(kernel, dim3((l->blocks.n + rows - 1) / rows, rows), dim3(64), lds, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(k_list_applied, dim3(1), dim3(1), 0, (hipStream_t)stream, l->st);
  PT_LAUNCH_CHECK(nullptr, "k_list_adamw");
  l->open = false;
  return PT_OK;
}

extern "C" int pt_tensors_report_read(pt_tensors* l, pt_step_report* out, void* stream) {
  if (!l || !out) return pt_fail(nullptr, PT_ERR_INVALID_ARG, "pt_tensors_report_read: NULL argument");
  ListState h;
  PT_HIP(nullptr, hipMemcpyAsync(&h, l->st, sizeof h, hipMemcpyDeviceToHost, (hipStream_t)stream));
  PT_HIP(nullptr, hipStreamSynchronize((hipStream_t)stream));
  out->sqnorm = h.s.sqnorm; out->norm = h.s.norm; out->clip_coef = h.s.clip_coef;
  out->loss_scale = h.s.loss_scale; out->grad_mult = h.s.c[8]; out->found_inf = h.s.found_inf;
  out->step = h.s.step; out->good_steps = h.s.good_steps;
  // The next norm ends the step on the device; until then these are what the update leaves behind.
  if (h.applied) {
    const bool inf = h.s.found_inf != 0, grown = !inf && h.s.good_steps + 1 >= h.s.growth_interval;
    out->step += inf ? 0 : 1;
    if (h.s.scaler_enabled) {
      out->good_steps = inf || grown ? 0 : h.s.good_steps + 1;
      if (inf) out->loss_scale = std::max(h.s.loss_scale * h.s.backoff, 1.0);
      if (grown) out->loss_scale = h.s.loss_scale * h.s.growth;
    }
  }
  return PT_OK;
}
