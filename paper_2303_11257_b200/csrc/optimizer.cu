// us_adamw: one AdamW step over many tensors in one launch, with states in 32 or 8 bits and the matmul operands of the next step;
// us_grad_norm: the 2-norm of all gradients and the factor that clips them.
//
// Both are bound by the bytes of their tensors.  The tensors are cut into units of 256 consecutive elements, which are dealt to the warps
// of a grid that is resident at once; a lane has two groups of four elements, so that every access is 16 bytes wide and a warp's accesses
// are whole lines.  The descriptions of the tensors travel as a kernel parameter: no table in device memory has to be kept or written,
// and a captured launch holds its own.
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "host.h"
#include "sm100.cuh"

namespace us {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnit = 256;                   // elements of a unit, and of a block of states in 8 bits
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
  uint8_t wide, dense;                       // groups of four are 16-byte accesses; p and g have no padded rows
  uint8_t copy_wide, copy_dense;
};
template <int MOST>
struct AdamArgs {
  float lr, beta1, beta2, rest1, rest2, eps;  // rest = 1 - beta, rounded once
  float ln_beta1, ln_beta2;
  const float *lr_factor, *grad_factor;
  int64_t* step;
  int count, last;                           // last: the launch that counts the step
  uint32_t units;
  AdamTensor t[MOST];
};

__device__ __forceinline__ float sqrt_approx(float x) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ void load4(const void* base, int dt, int64_t i, float* v) {
  if (dt == US_F32) {
    const float4 t = *reinterpret_cast<const float4*>(static_cast<const float*>(base) + i);
    v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
  } else {
    const uint2 t = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + i);
    const float2 a = dt == US_BF16 ? unpack_bf16x2(t.x) : unpack_f16x2(t.x), b = dt == US_BF16 ? unpack_bf16x2(t.y) : unpack_f16x2(t.y);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
  }
}
__device__ __forceinline__ void store4(void* base, int dt, int64_t i, const float* v) {
  if (dt == US_F32) *reinterpret_cast<float4*>(static_cast<float*>(base) + i) = make_float4(v[0], v[1], v[2], v[3]);
  else if (dt == US_BF16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + i) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else if (dt == US_F16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + i) = make_uint2(pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]));
  else *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(base) + i) = dt == US_E5M2 ? cvt_fp8x4<true>(v[0], v[1], v[2], v[3]) : cvt_fp8x4<false>(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void load_codes4(const void* base, int64_t i, float scale, float* v) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(base) + i);
  const float2 a = unpack_fp8x2((uint16_t)w, false), b = unpack_fp8x2((uint16_t)(w >> 16), false);
  v[0] = scale * a.x; v[1] = scale * a.y; v[2] = scale * b.x; v[3] = scale * b.y;
}

// Largest magnitude of the warp's values; a NaN is the largest.
__device__ __forceinline__ float warp_most(const float (&x)[8]) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
  return __uint_as_float(__reduce_max_sync(0xffffffffu, most));
}

// Where an element of a matrix with padded rows is: element `off` counted from (row0, col0).
struct Place {
  int64_t row0;
  int col0;
};
__device__ __forceinline__ Place place_of(const AdamTensor& t, int64_t e) {
  const int64_t row = t.n < (1ll << 31) ? (int64_t)t.by_cols.div((int)e) : e / t.cols;
  return {row, (int)(e - row * t.cols)};
}
__device__ __forceinline__ int64_t at(const AdamTensor& t, const Place& w, int off, int64_t ld) {
  const int q = t.by_cols.div(w.col0 + off);
  return (w.row0 + q) * ld + (w.col0 + off - q * t.cols);
}

template <int MOST>
__global__ void __launch_bounds__(kThreads, 4) adamw_kernel(const __grid_constant__ AdamArgs<MOST> a) {
  ptx::grid_sync_previous();
  const float gf = a.grad_factor ? *a.grad_factor : 1.0f;
  if (!(fabsf(gf) < INFINITY)) return;                       // the gradients were not finite: no step
  const int64_t step = *a.step + 1;
  // 1 - beta^t without cancellation at small t
  const float fix1 = -expm1f((float)step * a.ln_beta1), fix2 = -expm1f((float)step * a.ln_beta2);
  const float root_factor = 1.0f / sqrtf(fix2), lr = a.lr * (a.lr_factor ? *a.lr_factor : 1.0f), rate = lr / fix1;
  const int lane = threadIdx.x & 31;
  const uint32_t stride = gridDim.x * kWarps;
  uint32_t unit = blockIdx.x * kWarps + (threadIdx.x >> 5);
  int cur = 0;
  if (unit < a.units) {                                      // the first tensor whose units end behind this one
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (unit < a.t[mid].unit_end) hi = mid; else lo = mid + 1;
    }
    cur = lo;
  }
  for (; unit < a.units; unit += stride) {
    while (unit >= a.t[cur].unit_end) ++cur;
    const AdamTensor& t = a.t[cur];
    const uint32_t block = unit - (cur ? a.t[cur - 1].unit_end : 0u);
    const int64_t base = (int64_t)block * kUnit;
    const int here = (int)min((int64_t)kUnit, t.n - base);   // elements of this unit
    const bool small = t.m_scale != nullptr, wide = t.wide && here == kUnit;
    const bool padded = !t.dense || (t.copy && !t.copy_dense);
    const Place w = padded ? place_of(t, base) : Place{0, 0};
    float p[8], g[8], m[8], v[8];                            // v: the root of v where states are in 8 bits
    const float sm = small ? t.m_scale[block] : 0.f, sv = small ? t.v_scale[block] : 0.f;
    // element i of a lane: groups of four, or one of every 32
    auto offset = [&](int i) { return wide ? 128 * (i >> 2) + 4 * lane + (i & 3) : 32 * i + lane; };
    if (wide) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int off = 128 * k + 4 * lane;
        load4(t.p, US_F32, t.dense ? base + off : at(t, w, off, t.p_ld), &p[4 * k]);
        load4(t.g, t.g_dt, t.dense ? base + off : at(t, w, off, t.g_ld), &g[4 * k]);
        if (small) {
          load_codes4(t.m, base + off, sm, &m[4 * k]);
          load_codes4(t.v, base + off, sv, &v[4 * k]);
        } else {
          load4(t.m, US_F32, base + off, &m[4 * k]);
          load4(t.v, US_F32, base + off, &v[4 * k]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int off = 32 * i + lane;
        p[i] = g[i] = m[i] = v[i] = 0.f;
        if (off < here) {
          p[i] = t.p[t.dense ? base + off : at(t, w, off, t.p_ld)];
          g[i] = load_one(t.g, t.g_dt, t.dense ? base + off : at(t, w, off, t.g_ld));
          m[i] = small ? sm * load_one(t.m, US_E4M3, base + off) : static_cast<const float*>(t.m)[base + off];
          v[i] = small ? sv * load_one(t.v, US_E4M3, base + off) : static_cast<const float*>(t.v)[base + off];
        }
      }
    }
    const float my_rate = rate * t.lr_factor, decay = lr * t.lr_factor * t.decay;
    float root[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = gf * g[i];
      if (small) v[i] *= v[i];
      m[i] = fmaf(a.beta1, m[i], a.rest1 * x);
      v[i] = fmaf(a.beta2, v[i], a.rest2 * x * x);
      root[i] = sqrt_approx(v[i]);
      // p - (lr wd p + rate m / (root / sqrt(1 - beta2^t) + eps)): p is rounded once
      p[i] -= fmaf(decay, p[i], my_rate * __fdividef(m[i], fmaf(root[i], root_factor, a.eps)));
    }
    float inv_m = 0.f, inv_v = 0.f;
    if (small) {
      const float most_m = warp_most(m), most_v = warp_most(root);
      inv_m = most_m > kTiny ? kMostE4 / most_m : 0.f;
      inv_v = most_v > kTiny ? kMostE4 / most_v : 0.f;
      if (lane == 0) { t.m_scale[block] = most_m / kMostE4; t.v_scale[block] = most_v / kMostE4; }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m[i] *= inv_m;
        v[i] = root[i] * inv_v;
        v[i] = v[i] > 0.f ? fmaxf(v[i], 0x1p-9f) : v[i];     // the smallest code: no denominator is lost
      }
    }
    const int state_dt = small ? US_E4M3 : US_F32;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = t.copy_scale * p[i];
    if (wide) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int off = 128 * k + 4 * lane;
        store4(t.p, US_F32, t.dense ? base + off : at(t, w, off, t.p_ld), &p[4 * k]);
        store4(t.m, state_dt, base + off, &m[4 * k]);
        store4(t.v, state_dt, base + off, &v[4 * k]);
        if (t.copy && t.copy_wide) store4(t.copy, t.copy_dt, t.copy_dense ? base + off : at(t, w, off, t.copy_ld), &y[4 * k]);
      }
      if (t.copy && !t.copy_wide) {
#pragma unroll
        for (int i = 0; i < 8; ++i) store_one(t.copy, t.copy_dt, t.copy_dense ? base + offset(i) : at(t, w, offset(i), t.copy_ld), y[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int off = 32 * i + lane;
        if (off < here) {
          t.p[t.dense ? base + off : at(t, w, off, t.p_ld)] = p[i];
          store_one(t.m, state_dt, base + off, m[i]);
          store_one(t.v, state_dt, base + off, v[i]);
          if (t.copy) store_one(t.copy, t.copy_dt, t.copy_dense ? base + off : at(t, w, off, t.copy_ld), y[i]);
        }
      }
    }
  }
  // Every CTA has read the count of steps; the last one to end raises it.
  if (a.last) {
    __syncthreads();
    if (threadIdx.x == 0) {
      unsigned int* ended = reinterpret_cast<unsigned int*>(a.step + 1);
      if (atomicAdd(ended, 1u) == gridDim.x - 1) { *a.step = step; *ended = 0; }
    }
  }
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
  ptx::grid_sync_previous();
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
      float x[32];
#pragma unroll
      for (int k = 0; k < 8; ++k) load4(t.g, t.dt, base + 128 * k + 4 * lane, &x[4 * k]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x[8 * k + i], x[8 * k + i], s);
        sum += (double)s;
      }
    } else {
      const int64_t row0 = t.dense ? 0 : base / t.cols;
      const int col0 = t.dense ? 0 : (int)(base - row0 * t.cols);
      for (int off = lane; off < here; off += 32) {
        int64_t i = base + off;
        if (!t.dense) {
          const int q = t.by_cols.div(col0 + off);
          i = (row0 + q) * t.ld + (col0 + off - q * t.cols);
        }
        const float x = load_one(t.g, t.dt, i);
        sum += (double)(x * x);
      }
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
  if (n > kMostElements || !dense(t.m) || !dense(t.v)) return US_ERR_UNSUPPORTED;
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
  // (a matrix without padded rows beside one with them is walked as those are)
  const bool rows_of_four = d.dense || t.param.cols % 4 == 0;
  d.wide = fours(t.param) && fours(t.grad) && fours(t.m) && fours(t.v) && rows_of_four;
  d.copy_dense = t.copy.ptr && dense(t.copy);
  d.copy_wide = t.copy.ptr && fours(t.copy);
  return d;
}

template <int MOST>
us_status launch_adamw(AdamArgs<MOST>& a, const us_adamw_tensor* const* ts, int count, cudaStream_t stream) {
  const int sms = host::sm_count();
  if (sms <= 0) return US_ERR_CUDA;
  uint64_t units = 0;
  for (int i = 0; i < count; ++i) {
    a.t[i] = describe(*ts[i]);
    units += (uint64_t)((a.t[i].n + kUnit - 1) / kUnit);
    if (units >= (1ull << 31)) return US_ERR_UNSUPPORTED;
    a.t[i].unit_end = (uint32_t)units;
  }
  a.count = count;
  a.units = (uint32_t)units;
  const int grid = (int)std::max<uint64_t>(1, std::min<uint64_t>((units + kWarps - 1) / kWarps, (uint64_t)sms * 4));
  return host::launch(adamw_kernel<MOST>, nullptr, grid, kThreads, 0, 1, stream, a);
}

template <class A>
void set_options(A& a, double lr, double beta1, double beta2, double eps, const float* lr_factor, const float* grad_factor, int64_t* step) {
  a.lr = (float)lr; a.beta1 = (float)beta1; a.beta2 = (float)beta2; a.eps = (float)eps;
  a.rest1 = (float)(1.0 - beta1); a.rest2 = (float)(1.0 - beta2);
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
  // the same grid for every launch of a call: a CTA's sum is carried on by the CTA of that number
  const int grid = std::min(sms * 4, kMostCtas);
  return host::launch(norm_kernel<MOST>, nullptr, grid, kThreads, 0, 1, stream, a);
}

}  // namespace
}  // namespace us

using namespace us;

extern "C" us_status us_adamw(int count, const us_adamw_tensor* tensors, double lr, double beta1, double beta2, double eps, const float* lr_factor,
                              const float* grad_factor, int64_t* step, void* stream) {
  if (count < 1 || !tensors || !step) return US_ERR_INVALID_ARG;
  if (!(lr >= 0.0) || !isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !((float)eps > 0.f) || !isfinite((float)eps)) return US_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(step) % 8 || reinterpret_cast<uintptr_t>(lr_factor) % 4 || reinterpret_cast<uintptr_t>(grad_factor) % 4) return US_ERR_ALIGNMENT;
  for (int i = 0; i < count; ++i) {
    const us_status s = check_tensor(tensors[i]);
    if (s != US_OK) return s;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const us_adamw_tensor* ts[kMany];
  auto go = [&](auto& a, int n, bool last) {
    set_options(a, lr, beta1, beta2, eps, lr_factor, grad_factor, step);
    a.last = last;
    return launch_adamw(a, ts, n, st);
  };
  int n = 0;
  for (int i = 0; i < count; ++i) {
    if (elements(tensors[i].param) > 0) {
      if (n == kMany) {                                      // the table is full, and there is more
        AdamArgs<kMany> a;
        const us_status s = go(a, n, false);
        if (s != US_OK) return s;
        n = 0;
      }
      ts[n++] = &tensors[i];
    }
  }
  if (n <= kFew) {
    AdamArgs<kFew> a;
    return go(a, n, true);
  }
  AdamArgs<kMany> a;
  return go(a, n, true);
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
