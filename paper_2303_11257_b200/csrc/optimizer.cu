// us_adamw: one AdamW step over many tensors in one launch, with states in 32 or 8 bits and the matmul operands of the next step;
// us_grad_norm: the 2-norm of all gradients and the factor that clips them.
//
// Both are bound by the bytes of their tensors.  These are cut into blocks of 256 consecutive elements, of which a warp steps one at a time: a lane has two groups of
// four, so that its accesses are 16 bytes wide and the warp's are whole lines.  The descriptions of the tensors travel as a kernel parameter: no table in device
// memory has to be kept or written, and a captured launch holds its own.  The next grid is not released early (several CTAs an SM): captured norm and step of a small block 8.8 -> 7.5 us in 32 bits, 10.7 ->
// 10.0 in 8; norms of 201 million elements 126 -> 118.
//
// Measured on 201 million parameters (a copy moves 6.46 TB/s on the same card): states in 32 bits, FP8 operands written, 29 bytes an element, 841 us = 6.9 TB/s; states
// in 8 bits, BF16 gradients and operands, 16 bytes, 489 us = 6.6 TB/s, 526 under a load that holds the clock down: this one is bound by its instructions as
// well, 57 a lane and element.  What made the difference, in us (32 bits, 8 bits): the type of gradients and copies chosen once a block instead of for every
// element (984 -> 974, 823 -> 599); a warp number that the compiler knows to be uniform, so that fields and addresses are worked out once a warp (974 -> 943);
// chunks taken in order (943 -> 845; 599 -> 566); 8-bit blocks fetched ahead through shared memory, no register spilled (566 -> 501), in pairs and in pieces of 16
// bytes (501 -> 495, under load 578 -> 519).  Gradient norms: 118 us for 806 MB, 62 in BF16.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "host.h"
#include "sm100.cuh"

namespace us {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
__host__ __device__ constexpr int adam_ctas(bool eight) { return eight ? 4 : 3; }             // CTAs per SM
constexpr int kUnit = 256;                   // elements that a warp steps at a time, and of a block of states in 8 bits
__host__ __device__ constexpr int blocks_of_unit(bool eight) { return eight ? 2 : 1; }
constexpr int kFew = 30, kMany = 240;        // tensors that a launch describes: in 4 KB of parameters, or in 32 KB
constexpr float kTiny = 0x1p-100f;           // blocks whose largest magnitude is not above this are stored as zeros
constexpr float kMostE4 = 448.0f;

struct AdamTensor {
  float* p;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;                  // 8-bit states, else nullptr
  void* copy;
  int64_t n, p_ld, g_ld, copy_ld;
  uint32_t unit_end;                         // units up to and including this tensor
  int32_t cols;
  FastDiv by_cols;
  float copy_scale, lr_factor, decay;
  uint8_t g_dt, copy_dt;
  uint8_t wide, dense;                       // dense: p and g have no padded rows; wide: and the pieces in which all are fetched are aligned
  uint8_t copy_wide, copy_dense;
};
template <int MOST>
struct AdamArgs {
  float lr, beta1, beta2, root_beta2, rest1, root_rest2, eps;   // rest1 = 1 - beta1, root_rest2 = sqrt(1 - beta2); each rounded once
  float ln_beta1, ln_beta2;
  const float *lr_factor, *grad_factor;
  int64_t* step;
  int count, last;                           // last: the launch that counts the step
  uint32_t units;
  AdamTensor t[MOST];
};

// (A v below 2^-126 has a root too, of as many digits as it holds: gradients of 10^-19 and less are stepped by lr as others are.)
__device__ __forceinline__ float sqrt_approx(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Four elements of a gradient.
template <int DT>
__device__ __forceinline__ void load4(const void* base, int64_t i, float* v) {
  if (DT == US_F32) {
    const float4 t = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + i);
    v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
  } else {
    const uint2 t = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + i);
    const float2 a = DT == US_BF16 ? unpack_bf16x2(t.x) : unpack_f16x2(t.x), b = DT == US_BF16 ? unpack_bf16x2(t.y) : unpack_f16x2(t.y);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
  }
}
template <int DT>
__device__ __forceinline__ void store4(void* base, int64_t i, const float* v) {
  if (DT == US_F32) *reinterpret_cast<float4*>(static_cast<float*>(base) + i) = make_float4(v[0], v[1], v[2], v[3]);
  else if (DT == US_BF16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + i) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else if (DT == US_F16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + i) = make_uint2(pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]));
  else *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(base) + i) = cvt_fp8x4<DT == US_E5M2>(v[0], v[1], v[2], v[3]);
}
// Four elements as they were fetched.
__device__ __forceinline__ void four(const float4& t, int, float* v) { v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w; }
__device__ __forceinline__ void four(const uint2& t, int dt, float* v) {
  const float2 a = dt == US_BF16 ? unpack_bf16x2(t.x) : unpack_f16x2(t.x), b = dt == US_BF16 ? unpack_bf16x2(t.y) : unpack_f16x2(t.y);
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
__device__ __forceinline__ void four(uint32_t w, int, float* v) {
  const float2 a = unpack_fp8x2((uint16_t)w, false), b = unpack_fp8x2((uint16_t)(w >> 16), false);
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
// f(std::integral_constant<int, dtype>()): the choice of a type is taken once, not for every element.
template <class F>
__device__ __forceinline__ void with_grad_type(int dt, F f) {
  if (dt == US_F32) f(std::integral_constant<int, US_F32>());
  else if (dt == US_BF16) f(std::integral_constant<int, US_BF16>());
  else f(std::integral_constant<int, US_F16>());
}
template <class F>
__device__ __forceinline__ void with_type(int dt, F f) {
  if (dt == US_E4M3) f(std::integral_constant<int, US_E4M3>());
  else if (dt == US_E5M2) f(std::integral_constant<int, US_E5M2>());
  else with_grad_type(dt, f);
}

// Largest magnitude of the warp's values; a NaN is none.
__device__ __forceinline__ float warp_most(const float (&x)[8]) {
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
  return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
}

// Random bits for the rounding of states in 8 bits, from the number of the step and the element's place alone: a step that is made again rounds alike, on whatever path an element is
// stepped and whatever else the call has.  mix() spreads every bit of its argument over all (shifts and products with odd numbers, each of which can be undone); a block's seed is mixed twice,
// and what its elements make of it is one to one in the seed, so that each element's numbers are spread evenly whatever its neighbours' are.
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0xbb67ae85u;
  x ^= x >> 15;
  x *= 0x9e3779b1u;
  return x ^ x >> 16;
}
__device__ __forceinline__ uint32_t step_seed(uint64_t step) { return mix((uint32_t)step + mix((uint32_t)(step >> 32))); }
__device__ __forceinline__ uint32_t block_seed(uint32_t seed, uint32_t block) { return mix(seed + block * 0x9e3779b9u); }
__device__ __forceinline__ uint32_t element_bits(uint32_t block_seed, uint32_t element) {
  uint32_t x = block_seed + element * 0x9e3779b9u;
  x ^= x >> 15;
  x *= 0xbb67ae85u;
  return x ^ x >> 16;
}
// x rounded to one of the two E4M3 values around it, up where the part of the way that lies behind it and r 2^-20 (r: 20 bits) are 1 or more together.  A float32 has 20 bits more than a normal
// code: r is added to them, and they are dropped.  2^-6 is put under smaller magnitudes, whose codes are as far apart as those from 2^-6 on.  NaN stays; what is added to 448 is
// dropped too, or taken back by the conversion.
__device__ __forceinline__ float round_randomly(float x, uint32_t r) {
  const float under = fabsf(x) < 0x1p-6f ? copysignf(0x1p-6f, x) : 0.f;
  const float y = __uint_as_float((__float_as_uint(x + under) + r) & 0xfff00000u) - under;
  return fabsf(x) <= 512.f ? y : x;
}

// Four codes of roots above or at zero; one that is above zero has at least the smallest code.
__device__ __forceinline__ uint32_t root_codes4(const float* x) {
  uint32_t w = cvt_fp8x4<false>(x[0], x[1], x[2], x[3]);
  if ((w - 0x01010101u) & ~w & 0x80808080u) {                // a byte of zeros
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (x[i] > 0.f && !(w >> 8 * i & 0xffu)) w |= 1u << 8 * i;
  }
  return w;
}

// Where element `off` behind (row0, col0) of a matrix with padded rows is.
struct Place {
  int64_t row0;
  int col0;
};
__device__ __forceinline__ Place place_of(const AdamTensor& t, int64_t e) {
  const int64_t row = t.n < (1ll << 31) ? (int64_t)t.by_cols.div((int)e) : e / t.cols;
  return {row, (int)(e - row * t.cols)};
}
__device__ __forceinline__ int64_t at(const AdamTensor& t, const Place& w, int off, int64_t ld) {
  const int rows = t.cols >= kUnit ? (int)(w.col0 + off >= t.cols) : t.by_cols.div(w.col0 + off);   // that lie between
  return w.row0 * ld + w.col0 + off + rows * (ld - t.cols);
}

// What all units of a launch share.
//   m = beta1 m + gm g,   v = beta2 v + (gv g)^2,   p = p - lr wd p - rate m / (sqrt(v) + eps)
// with gm = (1 - beta1) grad_factor, gv = sqrt(1 - beta2) grad_factor, and sqrt(1 - beta2^t) taken out of the denominator into rate and eps.
struct AdamStep {
  float beta1, beta2, root_beta2, gm, gv, eps, lr, rate;
  float grad_factor, rest1;
  uint32_t seed;                                              // of this step's roundings
};

// The step of a lane's eight elements; sm, sv: the scales of states in 8 bits, whose codes m and v are (v's root).  Afterwards m is what is stored, and v, or where EIGHT root,
// codes before their rounding (RANDOM: after it); the block's scales are written.  element(i): the place in its block of the lane's element i.
template <bool EIGHT, bool RANDOM, class F>
__device__ __forceinline__ void step8(const AdamStep& a, const AdamTensor& t, uint32_t block, int lane, float sm, float sv, float (&p)[8], const float (&g)[8], float (&m)[8],
                                      float (&v)[8], float (&root)[8], F element) {
  const f32x2 rate = splat2(-(a.rate * t.lr_factor)), decay = splat2(-(a.lr * t.lr_factor * t.decay));
  const f32x2 keep_v = splat2(EIGHT ? a.root_beta2 * sv : a.beta2), gm = splat2(a.gm), gv = splat2(a.gv), eps = splat2(a.eps);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const f32x2 gg = pack2(g[i], g[i + 1]), x = mul2(gv, gg), x2 = mul2(x, x);
    // In 8 bits the operations of m are rounded one by one, as the formula has them: a code that falls the other way, because a fused form is off by 2^-24, is a block's largest
    // value in a later step every now and then, and moves all of its codes.  (The root, of which a step moves a thousandth, is not as sensitive.)  Scalar: the compiler makes
    // packed products and sums one operation again.
    f32x2 mm = mul2(EIGHT ? splat2(a.grad_factor) : gm, gg);
    if (EIGHT) {
      float m0, m1, g0, g1;
      unpack2(mul2(splat2(sm), pack2(m[i], m[i + 1])), m0, m1);
      unpack2(mul2(splat2(a.rest1), mm), g0, g1);
      mm = pack2(__fadd_rn(__fmul_rn(a.beta1, m0), g0), __fadd_rn(__fmul_rn(a.beta1, m1), g1));
    } else {
      mm = fma2(splat2(a.beta1), pack2(m[i], m[i + 1]), mm);
    }
    f32x2 vv = pack2(v[i], v[i + 1]);
    if (EIGHT) {
      vv = mul2(keep_v, vv);
      vv = fma2(vv, vv, x2);
    } else {
      vv = fma2(keep_v, vv, x2);
    }
    unpack2(mm, m[i], m[i + 1]);
    unpack2(vv, v[i], v[i + 1]);
    root[i] = sqrt_approx(v[i]);
    root[i + 1] = sqrt_approx(v[i + 1]);
    float d0, d1;
    unpack2(add2(pack2(root[i], root[i + 1]), eps), d0, d1);
    const f32x2 pp = pack2(p[i], p[i + 1]);                  // (rounded once: what comes off it is formed first)
    unpack2(add2(pp, fma2(decay, pp, mul2(rate, mul2(mm, pack2(rcp_approx(d0), rcp_approx(d1)))))), p[i], p[i + 1]);
  }
  if (EIGHT) {
    const float most_m = warp_most(m), most_v = warp_most(root);
    const f32x2 inv_m = splat2(most_m > kTiny ? __frcp_rn(most_m) * kMostE4 : 0.f), inv_v = splat2(most_v > kTiny ? __fdividef(kMostE4, most_v) : 0.f);
    if (lane == 0) { t.m_scale[block] = most_m * (1.0f / kMostE4); t.v_scale[block] = most_v * (1.0f / kMostE4); }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      unpack2(mul2(pack2(m[i], m[i + 1]), inv_m), m[i], m[i + 1]);
      unpack2(mul2(pack2(root[i], root[i + 1]), inv_v), root[i], root[i + 1]);
    }
    if (RANDOM) {
      const uint32_t seed = block_seed(a.seed, block);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t r = element_bits(seed, (uint32_t)element(i));
        m[i] = round_randomly(m[i], (r << 8 & 0xfff00u) | 0x80u);     // (12 bits are enough for what a step changes of m)
        root[i] = root[i] > 0.f ? round_randomly(fmaxf(root[i], 0x1p-9f), r >> 12) : root[i];
      }
    }
  }
}

// A unit's copies whose rows cut groups of four: one element a lane, 32 neighbours at a time.
__device__ __noinline__ void store_row(const AdamTensor& t, int64_t base, int lane, const float* row) {
  __syncwarp();
  const Place w = place_of(t, base);
  char* first = static_cast<char*>(t.copy) + (w.row0 * t.copy_ld + w.col0) * dtype_size(t.copy_dt);
  const int left = t.cols - w.col0;
  const int64_t between = t.copy_ld - t.cols;                  // columns of the first row, and what lies between two rows
  with_type(t.copy_dt, [&](auto dt) {
    if (t.cols >= kUnit) {                                     // two rows at most
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int off = 32 * i + lane;
        store_one(first, decltype(dt)::value, off + (off >= left ? between : 0), row[off]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int off = 32 * i + lane;
        store_one(first, decltype(dt)::value, off + t.by_cols.div(w.col0 + off) * between, row[off]);
      }
    }
  });
  __syncwarp();
}

// With states in 8 bits a block is more work for fewer bytes: a unit of two comes through shared memory while the warp works on the unit before, in pieces of 16 bytes
// a lane.  A warp's slot: param, grad, the codes of m and of v, and the four scales.
constexpr int kPair = 2 * kUnit, kGradAt = 4 * kPair, kMAt = 8 * kPair, kVAt = 9 * kPair, kScaleAt = 10 * kPair, kSlotBytes = 10 * kPair + 16;
__host__ __device__ constexpr int warp_bytes(bool eight) { return kUnit * 4 + (eight ? kSlotBytes : 0); }   // of shared memory: a block's copies, and the slot
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copy4(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ void fetch_unit(const AdamTensor& t, uint32_t unit, int lane, uint32_t slot) {
  const int64_t base = (int64_t)unit * kPair;
  const uint32_t at = slot + 16 * lane;
  const float* p = t.p + base + 4 * lane;
#pragma unroll
  for (int k = 0; k < 4; ++k) copy16(at + 512 * k, p + 128 * k);
  if (t.g_dt == US_F32) {
    const float* g = static_cast<const float*>(t.g) + base + 4 * lane;
#pragma unroll
    for (int k = 0; k < 4; ++k) copy16(at + kGradAt + 512 * k, g + 128 * k);
  } else {
    const uint16_t* g = static_cast<const uint16_t*>(t.g) + base + 8 * lane;
#pragma unroll
    for (int k = 0; k < 2; ++k) copy16(at + kGradAt + 512 * k, g + 256 * k);
  }
  copy16(at + kMAt, static_cast<const uint8_t*>(t.m) + base + 16 * lane);
  copy16(at + kVAt, static_cast<const uint8_t*>(t.v) + base + 16 * lane);
  if (lane < 4) copy4(slot + kScaleAt + 4 * lane, (lane < 2 ? t.m_scale : t.v_scale) + (int64_t)unit * 2 + (lane & 1));
}

// What a block's step leaves, to its tensor.
template <bool EIGHT, bool RANDOM>
__device__ __forceinline__ void store_block(const AdamTensor& t, int64_t base, int lane, float* row, const float (&p)[8], const float (&m)[8], const float (&v)[8],
                                            const float (&root)[8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int off = 128 * k + 4 * lane;
    store4<US_F32>(t.p, base + off, &p[4 * k]);
    store4<EIGHT ? US_E4M3 : US_F32>(t.m, base + off, &m[4 * k]);
    if (RANDOM) store4<US_E4M3>(t.v, base + off, &root[4 * k]);
    else if (EIGHT) *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + base + off) = root_codes4(&root[4 * k]);
    else store4<US_F32>(t.v, base + off, &v[4 * k]);
  }
  if (!t.copy) return;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = t.copy_scale * p[i];
  if (t.copy_wide) {
    const Place w = t.copy_dense ? Place{0, 0} : place_of(t, base);
    with_type(t.copy_dt, [&](auto dt) {
      constexpr int DT = decltype(dt)::value;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int off = 128 * k + 4 * lane;
        store4<DT>(t.copy, t.copy_dense ? base + off : at(t, w, off, t.copy_ld), &y[4 * k]);
      }
    });
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) *reinterpret_cast<float4*>(row + 128 * k + 4 * lane) = make_float4(y[4 * k], y[4 * k + 1], y[4 * k + 2], y[4 * k + 3]);
    store_row(t, base, lane, row);
  }
}

// A whole unit of a tensor whose pieces are aligned, from its tensor or (EIGHT) from the slot; `refill` starts the copies that take the slot next, once the warp
// has read what is there.
template <bool EIGHT, bool RANDOM, int GRAD, class F>
__device__ __forceinline__ void unit_step(const AdamStep& a, const AdamTensor& t, uint32_t unit, int lane, const char* slot, float* row, F refill) {
  using Grads = std::conditional_t<GRAD == US_F32, float4, uint2>;
  const auto element = [&](int i) { return 4 * lane + (i < 4 ? i : 124 + i); };
  if constexpr (EIGHT) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float p[8], g[8], m[8], v[8], root[8];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = 64 * j + 32 * k + lane;
        four(reinterpret_cast<const float4*>(slot)[i], US_F32, &p[4 * k]);
        four(reinterpret_cast<const Grads*>(slot + kGradAt)[i], GRAD, &g[4 * k]);
        four(reinterpret_cast<const uint32_t*>(slot + kMAt)[i], US_E4M3, &m[4 * k]);
        four(reinterpret_cast<const uint32_t*>(slot + kVAt)[i], US_E4M3, &v[4 * k]);
      }
      const float sm = reinterpret_cast<const float*>(slot + kScaleAt)[j], sv = reinterpret_cast<const float*>(slot + kScaleAt)[2 + j];
      if (j == 1) {
        __syncwarp();
        refill();
      }
      step8<true, RANDOM>(a, t, 2 * unit + j, lane, sm, sv, p, g, m, v, root, element);
      store_block<true, RANDOM>(t, (int64_t)unit * kPair + kUnit * j, lane, row, p, m, v, root);
    }
  } else {
    const int64_t base = (int64_t)unit * kUnit;
    float4 p4[2], m4[2], v4[2];
    Grads g4[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int off = 128 * k + 4 * lane;
      p4[k] = *reinterpret_cast<const float4*>(t.p + base + off);
      g4[k] = *reinterpret_cast<const Grads*>(static_cast<const char*>(t.g) + (base + off) * (GRAD == US_F32 ? 4 : 2));
      m4[k] = *reinterpret_cast<const float4*>(static_cast<const float*>(t.m) + base + off);
      v4[k] = *reinterpret_cast<const float4*>(static_cast<const float*>(t.v) + base + off);
    }
    float p[8], g[8], m[8], v[8], root[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      four(p4[k], US_F32, &p[4 * k]);
      four(g4[k], GRAD, &g[4 * k]);
      four(m4[k], US_F32, &m[4 * k]);
      four(v4[k], US_F32, &v[4 * k]);
    }
    step8<false, false>(a, t, unit, lane, 0.f, 0.f, p, g, m, v, root, element);
    store_block<false, false>(t, base, lane, row, p, m, v, root);
  }
}

// One element as it was fetched.
template <int DT>
__device__ __forceinline__ float one(float x) { return x; }
template <int DT>
__device__ __forceinline__ float one(uint16_t x) { return DT == US_BF16 ? __uint_as_float((uint32_t)x << 16) : __half2float(__ushort_as_half(x)); }
template <int DT>
__device__ __forceinline__ float one(uint8_t x) { return unpack_fp8x2(x, false).x; }

// Any block: a lane has every 32nd element.  All are fetched before the first is converted, since a tensor's last block is often the last to end (one by one: three vectors of
// 1000 and one of 77 took 8.3 us, now 4.6; with states in 8 bits 14.6 and 9.0).
template <bool EIGHT, bool RANDOM, int GRAD>
__device__ __forceinline__ void block_step_any(const AdamStep& a, const AdamTensor& t, uint32_t block, int lane) {
  const int64_t base = (int64_t)block * kUnit;
  const int here = (int)min((int64_t)kUnit, t.n - base);     // elements of this block
  const Place w = !t.dense || (t.copy && !t.copy_dense) ? place_of(t, base) : Place{0, 0};
  using Grad = std::conditional_t<GRAD == US_F32, float, uint16_t>;
  using State = std::conditional_t<EIGHT, uint8_t, float>;
  float p[8], g[8], m[8], v[8];
  Grad g1[8];
  State m1[8], v1[8];
  const float sm = EIGHT ? t.m_scale[block] : 0.f, sv = EIGHT ? t.v_scale[block] : 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int off = min(32 * i + lane, here - 1);
    p[i] = t.p[t.dense ? base + off : at(t, w, off, t.p_ld)];
    g1[i] = static_cast<const Grad*>(t.g)[t.dense ? base + off : at(t, w, off, t.g_ld)];
    m1[i] = static_cast<const State*>(t.m)[base + off];
    v1[i] = static_cast<const State*>(t.v)[base + off];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const bool is = 32 * i + lane < here;
    p[i] = is ? p[i] : 0.f;
    g[i] = is ? one<GRAD>(g1[i]) : 0.f;
    m[i] = is ? one<US_E4M3>(m1[i]) : 0.f;
    v[i] = is ? one<US_E4M3>(v1[i]) : 0.f;
  }
  float root[8];
  step8<EIGHT, RANDOM>(a, t, block, lane, sm, sv, p, g, m, v, root, [&](int i) { return 32 * i + lane; });
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int off = 32 * i + lane;
    if (off < here) {
      t.p[t.dense ? base + off : at(t, w, off, t.p_ld)] = p[i];
      store_one(t.m, EIGHT ? US_E4M3 : US_F32, base + off, m[i]);
      store_one(t.v, EIGHT ? US_E4M3 : US_F32, base + off, EIGHT && root[i] > 0.f ? fmaxf(root[i], 0x1p-9f) : EIGHT ? root[i] : v[i]);
      if (t.copy) store_one(t.copy, t.copy_dt, t.copy_dense ? base + off : at(t, w, off, t.copy_ld), t.copy_scale * p[i]);
    }
  }
}

// Out of line, so that the kernel's own registers stay in place: with states in 8 bits one call, which has the choice of the type in it (a call for each type: 528 us in the
// place of 524 for 201 million parameters), with states in 32 bits one for each type (4.9 us in the place of 5.3 for half a million).
template <bool EIGHT, bool RANDOM, int GRAD>
__device__ __noinline__ void unit_step_any(AdamStep a, const AdamTensor& t, uint32_t unit, int lane) {
  if constexpr (EIGHT) {
    with_grad_type(t.g_dt, [&](auto dt) {
      for (uint32_t block = 2 * unit; block < 2 * unit + 2 && (int64_t)block * kUnit < t.n; ++block) block_step_any<true, RANDOM, decltype(dt)::value>(a, t, block, lane);
    });
  } else {
    block_step_any<false, false, GRAD>(a, t, unit, lane);
  }
}

// EIGHT: tensors with states in 8 bits (RANDOM: rounded randomly, else to the nearest code), else those in 32.  (The random bits and the rounding: 201 million parameters 655 us in the
// place of 499, bound by instructions; with three CTAs an SM and fewer spilled registers 680.)
template <bool EIGHT, bool RANDOM, int MOST>
__global__ void __launch_bounds__(kThreads, adam_ctas(EIGHT)) adamw_kernel(const __grid_constant__ AdamArgs<MOST> a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ int64_t made;
  __shared__ uint32_t taken[2];
  (void)ptx::grid_wait_previous();
  if (threadIdx.x == 0) made = *a.step;
  const float grad_factor = a.grad_factor ? *a.grad_factor : 1.0f, lr_factor = a.lr_factor ? *a.lr_factor : 1.0f;
  __syncthreads();
  if (!(fabsf(grad_factor) < INFINITY)) return;              // the gradients were not finite: no step
  const int64_t step = made + 1;
  // 1 - beta^t without cancellation at small t
  const float fix1 = -expm1f((float)step * a.ln_beta1), root_fix2 = sqrtf(-expm1f((float)step * a.ln_beta2));
  AdamStep s;
  s.beta1 = a.beta1; s.beta2 = a.beta2; s.root_beta2 = a.root_beta2;
  s.gm = a.rest1 * grad_factor; s.gv = a.root_rest2 * grad_factor;
  s.grad_factor = grad_factor; s.rest1 = a.rest1;
  s.seed = RANDOM ? step_seed((uint64_t)step) : 0u;
  s.eps = fmaxf(a.eps * root_fix2, 0x1p-126f);               // (0 x 1 / 0 where an element has had no gradient)
  s.lr = a.lr * lr_factor;
  s.rate = s.lr * root_fix2 / fix1;
  // (handed round from one lane, the warp's number is known to be the same in all of them: what depends on it alone -- which tensor, where its
  // fields and addresses are -- is worked out once for the warp, by the uniform datapath)
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0);
  float* row = reinterpret_cast<float*>(smem + warp * warp_bytes(EIGHT));
  char* slot = smem + warp * warp_bytes(EIGHT) + kUnit * 4;
  unsigned int* count = reinterpret_cast<unsigned int*>(a.step + 1);
  const uint32_t chunks = (a.units + kWarps - 1) / kWarps;
  int cur = 0, ahead = 0;                                    // tensors of the unit at hand, and of the one fetched
  {                                                          // the first tensor whose units end behind this CTA's first
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (blockIdx.x * kWarps < a.t[mid].unit_end) hi = mid; else lo = mid + 1;
    }
    cur = ahead = lo;
  }
  constexpr int kBlocks = blocks_of_unit(EIGHT);
  auto in_tensor = [&](uint32_t unit, int k) { return unit - (k ? a.t[k - 1].unit_end : 0u); };
  auto whole = [&](const AdamTensor& t, uint32_t unit) { return t.wide && (int64_t)(unit + 1) * (kBlocks * kUnit) <= t.n; };
  auto fetch = [&](uint32_t unit) {
    if (EIGHT && unit < a.units) {
      while (unit >= a.t[ahead].unit_end) ++ahead;
      const uint32_t i = in_tensor(unit, ahead);
      if (whole(a.t[ahead], i)) fetch_unit(a.t[ahead], i, lane, ptx::smem_addr(slot));
    }
  };
  // A CTA's first chunks (one unit a warp) are set, the others are taken as it comes to them, so that chunks are worked on in their order and what all SMs read
  // and write at a time stays close together (us, 201 million parameters, states in 32 bits: 943 where every CTA walks with a fixed stride and SMs drift apart,
  // 845 so; two chunks at a time 857, four 862).  What is fetched ahead has to be taken one chunk sooner.
  constexpr uint32_t kSet = EIGHT ? 2 : 1;
  uint32_t chunk = blockIdx.x, after = gridDim.x + blockIdx.x;
  fetch(chunk * kWarps + warp);
  for (int turn = 0; chunk < chunks; turn ^= 1) {
    uint32_t next = 0;
    if (threadIdx.x == 0) next = atomicAdd(count, 1u);       // (needed only once the chunk is done)
    const uint32_t unit = chunk * kWarps + warp;
    if (EIGHT) {
      copies_wait();
      __syncwarp();
    }
    auto refill = [&] { fetch(after * kWarps + warp); };
    if (unit < a.units) {
      while (unit >= a.t[cur].unit_end) ++cur;
      const AdamTensor& t = a.t[cur];
      const uint32_t i = in_tensor(unit, cur);
      if (whole(t, i)) {
        with_grad_type(t.g_dt, [&](auto dt) { unit_step<EIGHT, RANDOM, decltype(dt)::value>(s, t, i, lane, slot, row, refill); });
      } else {
        refill();
        if constexpr (EIGHT) unit_step_any<true, RANDOM, 0>(s, t, i, lane);
        else with_grad_type(t.g_dt, [&](auto dt) { unit_step_any<false, false, decltype(dt)::value>(s, t, i, lane); });
      }
    }
    if (threadIdx.x == 0) {
      taken[turn] = kSet * gridDim.x + next;
      // As many have counted as there are chunks: none will, and all CTAs have read the count of steps.
      if (next == chunks - 1) {
        if (a.last) *a.step = step;
        *count = 0;
      }
    }
    __syncthreads();
    chunk = EIGHT ? after : taken[turn];
    after = taken[turn];
  }
}

// The step of a call whose tensors have no elements.
__global__ void count_step_kernel(int64_t* step, const float* grad_factor) {
  (void)ptx::grid_wait_previous();
  if (threadIdx.x == 0 && (!grad_factor || fabsf(*grad_factor) < INFINITY)) *step += 1;
}

// ---------------------------------------------------------------- norm
constexpr int kNormUnit = 1024;              // elements of a warp's unit
constexpr int kNormMany = 640, kNormFew = 80;
constexpr int kMostCtas = 2048;
struct NormTensor {
  const void* g;
  int64_t n, ld;
  uint32_t unit_end;
  int32_t cols;
  FastDiv by_cols;
  uint8_t dt, wide, dense;
};
template <int MOST>
struct NormArgs {
  double* partial;                           // one per CTA
  unsigned int* ended;
  float* out;
  float most;
  int count, first, last;                    // the first launch writes the partial sums, later ones add to them; the last one joins them
  uint32_t units;
  NormTensor t[MOST];
};

template <int MOST>
__global__ void __launch_bounds__(kThreads) norm_kernel(const __grid_constant__ NormArgs<MOST> a) {
  __shared__ double sums[kWarps];
  __shared__ bool join;
  (void)ptx::grid_wait_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t stride = gridDim.x * kWarps;
  uint32_t unit = blockIdx.x * kWarps + warp;
  int cur = 0;
  if (unit < a.units) {
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (unit < a.t[mid].unit_end) hi = mid; else lo = mid + 1;
    }
    cur = lo;
  }
  double sum = 0;
  for (; unit < a.units; unit += stride) {
    while (unit >= a.t[cur].unit_end) ++cur;
    const NormTensor& t = a.t[cur];
    const int64_t base = (int64_t)(unit - (cur ? a.t[cur - 1].unit_end : 0u)) * kNormUnit;
    const int here = (int)min((int64_t)kNormUnit, t.n - base);
    // sums of 8 squares in float32, then in float64
    if (t.wide && here == kNormUnit) {
      with_grad_type(t.dt, [&](auto dt) {
        float x[32];
#pragma unroll
        for (int k = 0; k < 8; ++k) load4<decltype(dt)::value>(t.g, base + 128 * k + 4 * lane, &x[4 * k]);
        float s[4] = {};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
          for (int i = 0; i < 8; ++i) s[k] = fmaf(x[8 * k + i], x[8 * k + i], s[k]);
        }
        const float all = (s[0] + s[1]) + (s[2] + s[3]);
        if (decltype(dt)::value == US_F16 || (all >= 0x1p-80f && all < INFINITY)) {
#pragma unroll
          for (int k = 0; k < 4; ++k) sum += (double)s[k];
        } else {                                               // squares beyond float32's range, or below it with no larger one beside them
#pragma unroll
          for (int i = 0; i < 32; ++i) sum += (double)x[i] * (double)x[i];
        }
      });
    } else {
      const int64_t row0 = t.dense ? 0 : base / t.cols;
      const int col0 = t.dense ? 0 : (int)(base - row0 * t.cols);
      with_grad_type(t.dt, [&](auto dt) {
        for (int first = lane; first < here; first += 256) {    // eight at a time (one at a time: the same vectors 10.1 us, now 4.9)
          float x[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int off = min(first + 32 * k, here - 1);
            int64_t i = base + off;
            if (!t.dense) {
              const int q = t.by_cols.div(col0 + off);
              i = (row0 + q) * t.ld + (col0 + off - q * t.cols);
            }
            x[k] = load_one(t.g, decltype(dt)::value, i);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) sum += first + 32 * k < here ? (double)x[k] * (double)x[k] : 0.0;
        }
      });
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) sums[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = 0;
    for (int w = 0; w < kWarps; ++w) s += sums[w];
    a.partial[blockIdx.x] = a.first ? s : a.partial[blockIdx.x] + s;
    join = false;
    if (a.last) {
      __threadfence();
      join = atomicAdd(a.ended, 1u) == gridDim.x - 1;
    }
  }
  __syncthreads();
  if (!join) return;
  // the CTA that ends last adds the partial sums, in a fixed order
  __threadfence();
  double s = 0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) s += __ldcg(a.partial + i);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  if (lane == 0) sums[warp] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double all = 0;
    for (int w = 0; w < kWarps; ++w) all += sums[w];
    const float norm = (float)sqrt(all);
    a.out[0] = norm;
    a.out[1] = norm < INFINITY ? (norm > a.most ? (float)((double)a.most / sqrt(all)) : 1.0f) : NAN;
    *a.ended = 0;
  }
}

// ---------------------------------------------------------------- host side
us_status check_mat(const us_mat& m) {
  if (m.dtype < US_F32 || m.dtype > US_E5M2 || m.rows < 0 || m.cols < 0 || m.rows >= (1ll << 31) || m.cols >= (1ll << 31) - 2 * kNormUnit) return US_ERR_INVALID_ARG;
  if (m.rows == 0 || m.cols == 0) return US_OK;
  if (!m.ptr || m.ld < m.cols) return US_ERR_INVALID_ARG;
  return US_OK;
}
bool natural(const us_mat& m) { return reinterpret_cast<uintptr_t>(m.ptr) % dtype_size(m.dtype) == 0; }
bool dense(const us_mat& m) { return m.rows <= 1 || m.ld == m.cols; }
bool is_grad(int dt) { return dt == US_F32 || dt == US_BF16 || dt == US_F16; }
int64_t elements(const us_mat& m) { return m.rows * m.cols; }
// Groups of four consecutive elements are aligned, and, with padded rows, lie in one row.
bool fours(const us_mat& m) {
  const int bytes = 4 * dtype_size(m.dtype);
  return reinterpret_cast<uintptr_t>(m.ptr) % bytes == 0 && (dense(m) || (m.cols % 4 == 0 && m.ld % 4 == 0));
}
constexpr int64_t kMostElements = 1ll << 36;

us_status check_tensor(const us_adamw_tensor& t) {
  const us_mat* all[] = {&t.param, &t.grad, &t.m, &t.v};
  for (const us_mat* m : all) {
    const us_status s = check_mat(*m);
    if (s != US_OK) return s;
  }
  const int64_t n = elements(t.param);
  if (t.grad.rows != t.param.rows || t.grad.cols != t.param.cols || elements(t.m) != n || elements(t.v) != n) return US_ERR_INVALID_ARG;
  if (!isfinite(t.copy_scale) || !isfinite(t.lr_factor) || !isfinite(t.weight_decay)) return US_ERR_INVALID_ARG;
  const bool small = t.m.dtype == US_E4M3;
  if (t.param.dtype != US_F32 || !is_grad(t.grad.dtype) || t.m.dtype != t.v.dtype || (!small && t.m.dtype != US_F32)) return US_ERR_UNSUPPORTED;
  if (t.rounding != US_ROUND_NEAREST && t.rounding != US_ROUND_RANDOM) return US_ERR_INVALID_ARG;
  if (n > kMostElements || !dense(t.m) || !dense(t.v) || (!small && t.rounding == US_ROUND_RANDOM)) return US_ERR_UNSUPPORTED;
  if (small) {
    for (const us_mat* m : {&t.m_scale, &t.v_scale}) {
      const us_status s = check_mat(*m);
      if (s != US_OK) return s;
      if (elements(*m) != (n + kUnit - 1) / kUnit) return US_ERR_INVALID_ARG;
      if (m->dtype != US_F32 || !dense(*m)) return US_ERR_UNSUPPORTED;
      if (n && !natural(*m)) return US_ERR_ALIGNMENT;
    }
  }
  if (t.copy.ptr) {
    const us_status s = check_mat(t.copy);
    if (s != US_OK) return s;
    if (t.copy.rows != t.param.rows || t.copy.cols != t.param.cols) return US_ERR_INVALID_ARG;
    if (n && !natural(t.copy)) return US_ERR_ALIGNMENT;
  }
  if (n)
    for (const us_mat* m : all)
      if (!natural(*m)) return US_ERR_ALIGNMENT;
  return US_OK;
}

AdamTensor describe(const us_adamw_tensor& t) {
  AdamTensor d{};
  const bool small = t.m.dtype == US_E4M3;
  d.p = static_cast<float*>(t.param.ptr); d.g = t.grad.ptr; d.m = t.m.ptr; d.v = t.v.ptr;
  d.m_scale = small ? static_cast<float*>(t.m_scale.ptr) : nullptr;
  d.v_scale = small ? static_cast<float*>(t.v_scale.ptr) : nullptr;
  d.copy = t.copy.ptr;
  d.n = elements(t.param);
  d.p_ld = t.param.ld; d.g_ld = t.grad.ld; d.copy_ld = t.copy.ld;
  d.cols = (int32_t)t.param.cols;
  d.by_cols = make_fast_div(d.cols);
  d.copy_scale = t.copy_scale; d.lr_factor = t.lr_factor; d.decay = t.weight_decay;
  d.g_dt = (uint8_t)t.grad.dtype; d.copy_dt = (uint8_t)t.copy.dtype;
  d.dense = dense(t.param) && dense(t.grad);
  const auto aligned16 = [](const us_mat& m) { return reinterpret_cast<uintptr_t>(m.ptr) % 16 == 0; };
  d.wide = d.dense && (small ? aligned16(t.param) && aligned16(t.grad) && aligned16(t.m) && aligned16(t.v) : fours(t.param) && fours(t.grad) && fours(t.m) && fours(t.v));
  d.copy_dense = t.copy.ptr && dense(t.copy);
  d.copy_wide = t.copy.ptr && fours(t.copy);
  return d;
}

template <bool EIGHT, bool RANDOM, int MOST>
us_status launch_adamw(AdamArgs<MOST>& a, const us_adamw_tensor* const* ts, int count, cudaStream_t stream) {
  const int sms = host::sm_count();
  if (sms <= 0) return US_ERR_CUDA;
  uint64_t units = 0;
  for (int i = 0; i < count; ++i) {
    a.t[i] = describe(*ts[i]);
    constexpr int kElements = kUnit * blocks_of_unit(EIGHT);
    units += (uint64_t)((a.t[i].n + kElements - 1) / kElements);
    if (units >= (1ull << 31)) return US_ERR_UNSUPPORTED;
    a.t[i].unit_end = (uint32_t)units;
  }
  a.count = count;
  a.units = (uint32_t)units;
  const int grid = (int)std::min<uint64_t>((units + kWarps - 1) / kWarps, (uint64_t)(sms * adam_ctas(EIGHT)));
  static std::atomic<uint64_t> smem_set{0};
  return host::launch(adamw_kernel<EIGHT, RANDOM, MOST>, &smem_set, grid, kThreads, kWarps * warp_bytes(EIGHT), 1, stream, a);
}

template <class A>
void set_options(A& a, double lr, double beta1, double beta2, double eps, const float* lr_factor, const float* grad_factor, int64_t* step) {
  a.lr = (float)lr; a.beta1 = (float)beta1; a.beta2 = (float)beta2; a.eps = (float)eps;
  a.rest1 = (float)(1.0 - beta1); a.root_rest2 = (float)sqrt(1.0 - beta2); a.root_beta2 = (float)sqrt(beta2);
  a.ln_beta1 = (float)log(beta1); a.ln_beta2 = (float)log(beta2);
  a.lr_factor = lr_factor; a.grad_factor = grad_factor; a.step = step;
}

template <int MOST>
us_status launch_norm(NormArgs<MOST>& a, const us_mat* const* ms, int count, cudaStream_t stream) {
  const int sms = host::sm_count();
  if (sms <= 0) return US_ERR_CUDA;
  uint64_t units = 0;
  for (int i = 0; i < count; ++i) {
    const us_mat& m = *ms[i];
    NormTensor& t = a.t[i];
    t.g = m.ptr; t.n = elements(m); t.ld = m.ld; t.cols = (int32_t)m.cols; t.by_cols = make_fast_div(t.cols);
    t.dt = (uint8_t)m.dtype; t.dense = dense(m); t.wide = t.dense && fours(m);
    units += (uint64_t)((t.n + kNormUnit - 1) / kNormUnit);
    if (units >= (1ull << 31)) return US_ERR_UNSUPPORTED;
    t.unit_end = (uint32_t)units;
  }
  a.count = count;
  a.units = (uint32_t)units;
  // where there are several launches, all have one grid: a CTA's sum is carried on by the CTA of that number
  const uint64_t want = a.first && a.last ? std::max<uint64_t>(1, (units + kWarps - 1) / kWarps) : kMostCtas;
  const int grid = (int)std::min<uint64_t>({want, (uint64_t)sms * 4, (uint64_t)kMostCtas});
  return host::launch(norm_kernel<MOST>, nullptr, grid, kThreads, 0, 1, stream, a);
}

}  // namespace
}  // namespace us

using namespace us;

extern "C" us_status us_adamw(int count, const us_adamw_tensor* tensors, double lr, double beta1, double beta2, double eps, const float* lr_factor,
                              const float* grad_factor, int64_t* step, void* stream) {
  if (count < 1 || !tensors || !step) return US_ERR_INVALID_ARG;
  if (!(lr >= 0.0) || !isfinite((float)lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !((float)eps > 0.f) || !isfinite((float)eps)) return US_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(step) % 8 || reinterpret_cast<uintptr_t>(lr_factor) % 4 || reinterpret_cast<uintptr_t>(grad_factor) % 4) return US_ERR_ALIGNMENT;
  for (int i = 0; i < count; ++i) {
    const us_status s = check_tensor(tensors[i]);
    if (s != US_OK) return s;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // Launches: the tensors with states in 32 bits, then those in 8, rounded to the nearest code, then randomly; as many to one as its table holds.  The last launch counts the step.
  auto go = [&](auto& a, auto kind, const us_adamw_tensor* const* ts, int n, bool last) {
    set_options(a, lr, beta1, beta2, eps, lr_factor, grad_factor, step);
    a.last = last;
    return launch_adamw<(decltype(kind)::value > 0), (decltype(kind)::value > 1)>(a, ts, n, st);
  };
  auto table = [&](auto kind, const us_adamw_tensor* const* ts, int n, bool last) {
    if (n <= kFew) {
      AdamArgs<kFew> a;
      return go(a, kind, ts, n, last);
    }
    AdamArgs<kMany> a;
    return go(a, kind, ts, n, last);
  };
  auto kind_of = [](const us_adamw_tensor& t) { return t.m.dtype != US_E4M3 ? 0 : t.rounding == US_ROUND_RANDOM ? 2 : 1; };
  int64_t left[3] = {0, 0, 0};                               // tensors with elements, not launched yet
  for (int i = 0; i < count; ++i)
    if (elements(tensors[i].param) > 0) ++left[kind_of(tensors[i])];
  if (left[0] + left[1] + left[2] == 0) return us::host::launch(count_step_kernel, nullptr, 1, 32, 0, 1, st, step, grad_factor);
  const us_adamw_tensor* ts[kMany];
  for (int kind = 0; kind < 3; ++kind) {
    for (int i = 0, n = 0; left[kind] > 0; ++i) {
      if (elements(tensors[i].param) == 0 || kind_of(tensors[i]) != kind) continue;
      ts[n++] = &tensors[i];
      if (n < kMany && n < left[kind]) continue;
      left[kind] -= n;
      const bool last = left[0] + left[1] + left[2] == 0;
      const us_status s = kind == 0   ? table(std::integral_constant<int, 0>(), ts, n, last)
                          : kind == 1 ? table(std::integral_constant<int, 1>(), ts, n, last)
                                      : table(std::integral_constant<int, 2>(), ts, n, last);
      if (s != US_OK) return s;
      n = 0;
    }
  }
  return US_OK;
}

extern "C" size_t us_grad_norm_workspace_bytes(void) { return 64 + kMostCtas * sizeof(double); }

extern "C" us_status us_grad_norm(int count, const us_mat* grads, float max_norm, float* out, void* ws, size_t ws_bytes, void* stream) {
  if (count < 1 || !grads || !out || !(max_norm > 0.f)) return US_ERR_INVALID_ARG;
  for (int i = 0; i < count; ++i) {
    const us_status s = check_mat(grads[i]);
    if (s != US_OK) return s;
    if (!is_grad(grads[i].dtype) || elements(grads[i]) > kMostElements) return US_ERR_UNSUPPORTED;
    if (elements(grads[i]) > 0 && !natural(grads[i])) return US_ERR_ALIGNMENT;
  }
  if (reinterpret_cast<uintptr_t>(out) % 4) return US_ERR_ALIGNMENT;
  if (!ws || ws_bytes < us_grad_norm_workspace_bytes()) return US_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) % 16) return US_ERR_ALIGNMENT;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const us_mat* ms[kNormMany];
  bool first = true;
  auto go = [&](auto& a, int n, bool last) {
    a.ended = static_cast<unsigned int*>(ws);
    a.partial = reinterpret_cast<double*>(static_cast<char*>(ws) + 64);
    a.out = out; a.most = max_norm; a.first = first; a.last = last;
    first = false;
    return launch_norm(a, ms, n, st);
  };
  int n = 0;
  for (int i = 0; i < count; ++i) {
    if (elements(grads[i]) > 0) {
      if (n == kNormMany) {
        NormArgs<kNormMany> a;
        const us_status s = go(a, n, false);
        if (s != US_OK) return s;
        n = 0;
      }
      ms[n++] = &grads[i];
    }
  }
  if (n <= kNormFew) {
    NormArgs<kNormFew> a;
    return go(a, n, true);
  }
  NormArgs<kNormMany> a;
  return go(a, n, true);
}
