// us_qk_norm_fwd / us_qk_norm_bwd: root-mean-square norms of queries and keys, head by head, with the rotation of their positions in the
// same pass, forward and backward; us_rotary_table: the angles' cosines and sines.
//
//   forward    r = 1 / sqrt(mean x^2 + eps),  n = w x r,  y = R n          R: each pair (a, b) of the rotated features -> (a c - b s, b c + a s)
//   backward   n' = R^T g,  u = w n',  dx = beta_x r (u - x r mean(u x r)),  dw = beta_w sum n' x r
//
// Bound by HBM: every element is read once and written once.  A head is held by a group of G lanes (a power of two), each with two chunks of
// eight features that hold whole pairs -- features i .. i + 7 and their partners half a rotation further, or sixteen neighbours -- so that the
// rotation needs no exchange and one group sum (forward) or two (backward) are all that lanes tell one another.  A warp takes 32 / G heads at
// once and kIter such steps of one token, whose cosines and sines it holds in registers over all of them; the norm's weight it holds for the
// whole launch, since a CTA works for one part (queries or keys) only.  Weight gradients are summed in the registers of the lane that has
// the feature, then over groups, warps and, in a second launch, CTAs, in a fixed order without atomics.
// Rows that are not on 16-byte boundaries, and widths that are no multiple of eight, take the general kernels: a warp a head, through shared memory.
#include <cuda.h>

#include <algorithm>

#include "common.cuh"
#include "host.h"
#include "rowwise.cuh"
#include "sm100.cuh"

namespace us {
namespace {

constexpr int kMostParts = 4, kMostWidth = 1024, kMostVecWidth = 512;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBwdCtasPerSm = 2, kFwdCtasPerSm = 4;

struct QkPart {
  const void *x, *g, *w;
  void* y;                     // forward: output; backward: dX
  void* dw;
  int64_t x_ld, g_ld, y_ld;
  int x_dt, g_dt, w_dt, y_dt, dw_dt;
  int heads, blocks;           // heads, and warp units per row
  FastDiv d_blocks;            // by blocks
  int first_cta, ctas;         // CTAs that work for this part
  float beta_w;
};
struct QkArgs {
  QkPart part[kMostParts];
  int count, width;            // features of a head
  int64_t rows;
  const float* table; int64_t table_ld; int64_t table_rows;    // (cos, sin) pairs; nullptr: no rotation
  const int32_t* positions; int64_t start; uint32_t period;   // period 0: positions count on over all rows
  int rotated;                 // features of a head that are rotated
  float eps, inv_width, beta_x;
  float* partial;              // weight gradients of each CTA, [CTAs x width]
  int lanes, group;            // vector kernels: lanes of a group that hold features, and the group's size
};

// The table row of a matrix row, nullptr where its position is not in the table.
__device__ __forceinline__ const float* angles_of(const QkArgs& p, int64_t row) {
  const int64_t at = p.positions ? (int64_t)__ldg(p.positions + row) : p.start + (p.period ? (int64_t)((uint32_t)row % p.period) : row);
  return at >= 0 && at < p.table_rows ? p.table + at * p.table_ld : nullptr;
}

__device__ __forceinline__ int64_t row_of(const QkPart& q, int64_t unit) {
  return q.blocks == 1 ? unit : unit < (1ll << 31) ? (int64_t)q.d_blocks.div((int)unit) : unit / q.blocks;
}

__device__ __forceinline__ float group_sum(float v, int group) {
  for (int o = group >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Eight features: as they are stored (one register for two 16-bit ones), and as float32.
template <int DT> struct Chunk { uint4 r; };
template <> struct Chunk<US_F32> { float4 a, b; };
template <int DT>
__device__ __forceinline__ void fetch(Chunk<DT>& c, const void* base, int64_t at) {
  if constexpr (DT == US_F32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
    c.a = __ldg(q); c.b = __ldg(q + 1);
  } else {
    c.r = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at));
  }
}
template <int DT>
__device__ __forceinline__ void clear(Chunk<DT>& c) {
  if constexpr (DT == US_F32) c.a = c.b = make_float4(0.f, 0.f, 0.f, 0.f); else c.r = make_uint4(0u, 0u, 0u, 0u);
}
template <int DT>
__device__ __forceinline__ void widen(const Chunk<DT>& c, float (&v)[8]) {
  if constexpr (DT == US_F32) {
    v[0] = c.a.x; v[1] = c.a.y; v[2] = c.a.z; v[3] = c.a.w; v[4] = c.b.x; v[5] = c.b.y; v[6] = c.b.z; v[7] = c.b.w;
  } else {
    unpack16x8(c.r, DT, v);
  }
}

// Which features a lane has, and which of them are rotated.
struct Lane {
  int a, b;                    // first feature of each chunk
  bool has_a, has_b, rot_a, rot_b;
};
template <bool NEIGHBOURS>
__device__ __forceinline__ Lane lane_of(const QkArgs& p, int j) {
  Lane l;
  if (NEIGHBOURS) {
    l.a = 16 * j; l.b = 16 * j + 8;
    l.rot_a = l.a < p.rotated; l.rot_b = l.b < p.rotated;
  } else {
    const int turning = p.rotated / 16;
    l.rot_a = l.rot_b = j < turning;
    l.a = l.rot_a ? 8 * j : p.rotated + 16 * (j - turning);
    l.b = l.rot_a ? l.a + p.rotated / 2 : l.a + 8;
  }
  l.has_a = j < p.lanes && l.a < p.width;
  l.has_b = j < p.lanes && l.b < p.width;
  l.rot_a = l.rot_a && l.has_a; l.rot_b = l.rot_b && l.has_b;
  return l;
}
// Cosines and sines of a lane's pairs: eight pairs from pair 8 j on.
__device__ __forceinline__ void fetch_angles(const QkArgs& p, int64_t row, int j, const Lane& l, float (&cs)[16]) {
  if (!(l.rot_a || l.rot_b)) return;
  const float* t = angles_of(p, row);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool there = i < 2 ? l.rot_a : l.rot_b;
    const float4 v = there && t ? __ldg(reinterpret_cast<const float4*>(t + 16 * j) + i)
                                : make_float4(__int_as_float(0x7fffffff), __int_as_float(0x7fffffff), __int_as_float(0x7fffffff), __int_as_float(0x7fffffff));
    cs[4 * i] = v.x; cs[4 * i + 1] = v.y; cs[4 * i + 2] = v.z; cs[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float t = a * c - b * s;
  b = b * c + a * s;
  a = t;
}
template <bool NEIGHBOURS, bool BACK>
__device__ __forceinline__ void rotate(float (&a)[8], float (&b)[8], const float (&cs)[16], const Lane& l) {
  if (NEIGHBOURS) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (l.rot_a) turn(a[2 * i], a[2 * i + 1], cs[2 * i], BACK ? -cs[2 * i + 1] : cs[2 * i + 1]);
      if (l.rot_b) turn(b[2 * i], b[2 * i + 1], cs[8 + 2 * i], BACK ? -cs[8 + 2 * i + 1] : cs[8 + 2 * i + 1]);
    }
  } else if (l.rot_a) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(a[i], b[i], cs[2 * i], BACK ? -cs[2 * i + 1] : cs[2 * i + 1]);
  }
}

__device__ __forceinline__ int part_of(const QkArgs& p, int cta) {
  int k = 0;
  while (k + 1 < p.count && cta >= p.part[k + 1].first_cta) ++k;
  return k;
}
__device__ __forceinline__ void load_weight(const QkPart& q, const Lane& l, float (&wa)[8], float (&wb)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    wa[i] = l.has_a ? (q.w ? load_one(q.w, q.w_dt, l.a + i) : 1.f) : 0.f;
    wb[i] = l.has_b ? (q.w ? load_one(q.w, q.w_dt, l.b + i) : 1.f) : 0.f;
  }
}

// DT: type of the inputs.  ITER: steps of 32 / G heads whose loads are in flight together.
template <int DT, int ITER, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads) qk_fwd_kernel(const __grid_constant__ QkArgs p) {
  const int zero = ptx::grid_wait_previous();
  const QkPart& q = p.part[part_of(p, blockIdx.x)];
  const int lane = threadIdx.x & 31, j = lane & (p.group - 1), per = 32 / p.group;
  const Lane l = lane_of<NEIGHBOURS>(p, j);
  float wa[8], wb[8];
  load_weight(q, l, wa, wb);
  const int64_t units = p.rows * q.blocks, step = (int64_t)q.ctas * kWarps;
  for (int64_t u = (int64_t)(blockIdx.x - q.first_cta) * kWarps + (threadIdx.x >> 5) + zero; u < units; u += step) {
    const int64_t row = row_of(q, u);
    const int head0 = (int)(u - row * q.blocks) * (per * ITER) + lane / p.group;
    Chunk<DT> ca[ITER], cb[ITER];
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
      const int head = head0 + k * per;
      const int64_t at = row * q.x_ld + (int64_t)head * p.width;
      if (head < q.heads && l.has_a) fetch(ca[k], q.x, at + l.a); else clear(ca[k]);
      if (head < q.heads && l.has_b) fetch(cb[k], q.x, at + l.b); else clear(cb[k]);
    }
    float cs[16];
    if (p.table) fetch_angles(p, row, j, l, cs);
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
      const int head = head0 + k * per;
      float a[8], b[8], ss = 0.f;
      widen(ca[k], a); widen(cb[k], b);
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
      const float r = rsqrtf(fmaf(group_sum(ss, p.group), p.inv_width, p.eps));
#pragma unroll
      for (int i = 0; i < 8; ++i) { a[i] *= r * wa[i]; b[i] *= r * wb[i]; }
      if (p.table) rotate<NEIGHBOURS, false>(a, b, cs, l);
      const int64_t at = row * q.y_ld + (int64_t)head * p.width;
      if (head < q.heads && l.has_a) store8(q.y, q.y_dt, at, l.a, p.width, true, a);
      if (head < q.heads && l.has_b) store8(q.y, q.y_dt, at, l.b, p.width, true, b);
    }
  }
}

template <int DT, int ITER, bool NEIGHBOURS>
__global__ void __launch_bounds__(kThreads, 2) qk_bwd_kernel(const __grid_constant__ QkArgs p) {
  __shared__ float sums[kWarps][kMostVecWidth];
  const int zero = ptx::grid_wait_previous();
  const QkPart& q = p.part[part_of(p, blockIdx.x)];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & (p.group - 1), per = 32 / p.group;
  const Lane l = lane_of<NEIGHBOURS>(p, j);
  float wa[8], wb[8], da[8], db[8];
  load_weight(q, l, wa, wb);
#pragma unroll
  for (int i = 0; i < 8; ++i) da[i] = db[i] = 0.f;
  const int64_t units = p.rows * q.blocks, step = (int64_t)q.ctas * kWarps;
  for (int64_t u = (int64_t)(blockIdx.x - q.first_cta) * kWarps + warp + zero; u < units; u += step) {
    const int64_t row = row_of(q, u);
    const int head0 = (int)(u - row * q.blocks) * (per * ITER) + lane / p.group;
    Chunk<DT> ca[ITER], cb[ITER], ga[ITER], gb[ITER];
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
      const int head = head0 + k * per;
      const int64_t at = row * q.x_ld + (int64_t)head * p.width, ag = row * q.g_ld + (int64_t)head * p.width;
      if (head < q.heads && l.has_a) { fetch(ca[k], q.x, at + l.a); fetch(ga[k], q.g, ag + l.a); } else { clear(ca[k]); clear(ga[k]); }
      if (head < q.heads && l.has_b) { fetch(cb[k], q.x, at + l.b); fetch(gb[k], q.g, ag + l.b); } else { clear(cb[k]); clear(gb[k]); }
    }
    float cs[16];
    if (p.table) fetch_angles(p, row, j, l, cs);
#pragma unroll
    for (int k = 0; k < ITER; ++k) {
      const int head = head0 + k * per;
      float a[8], b[8], na[8], nb[8], ss = 0.f, dot = 0.f;
      widen(ca[k], a); widen(cb[k], b);
      widen(ga[k], na); widen(gb[k], nb);
      if (p.table) rotate<NEIGHBOURS, true>(na, nb, cs, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
        dot = fmaf(na[i] * wa[i], a[i], fmaf(nb[i] * wb[i], b[i], dot));
      }
      for (int o = p.group >> 1; o > 0; o >>= 1) {
        ss += __shfl_xor_sync(0xffffffffu, ss, o);
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
      }
      if (head >= q.heads) continue;                      // (its chunks are zero, but 1 / sigma of nothing may not be finite)
      const float r = rsqrtf(fmaf(ss, p.inv_width, p.eps));
      const float m = dot * r * r * p.inv_width, br = p.beta_x * r;       // mean(u xhat) = r dot / width, times xhat = x r
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        da[i] = fmaf(na[i], a[i] * r, da[i]);
        db[i] = fmaf(nb[i], b[i] * r, db[i]);
        a[i] = br * fmaf(-a[i], m, na[i] * wa[i]);
        b[i] = br * fmaf(-b[i], m, nb[i] * wb[i]);
      }
      const int64_t at = row * q.y_ld + (int64_t)head * p.width;
      if (l.has_a) store8(q.y, q.y_dt, at, l.a, p.width, true, a);
      if (l.has_b) store8(q.y, q.y_dt, at, l.b, p.width, true, b);
    }
  }
  if (!q.dw) return;
  for (int o = p.group; o < 32; o <<= 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      da[i] += __shfl_xor_sync(0xffffffffu, da[i], o);
      db[i] += __shfl_xor_sync(0xffffffffu, db[i], o);
    }
  }
  if (lane < p.group) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (l.has_a) sums[warp][l.a + i] = da[i];
      if (l.has_b) sums[warp][l.b + i] = db[i];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < p.width; c += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) v += sums[k][c];
    p.partial[(int64_t)blockIdx.x * p.width + c] = v;
  }
}

// The partner of feature e of a head, and its pair; pair -1: not rotated.
__device__ __forceinline__ int pair_of(const QkArgs& p, bool neighbours, int e, int& partner, bool& first) {
  if (!p.table || e >= p.rotated) return -1;
  if (neighbours) { first = !(e & 1); partner = e ^ 1; return e >> 1; }
  const int half = p.rotated / 2;
  first = e < half;
  partner = first ? e + half : e - half;
  return first ? e : e - half;
}

// Any width up to kMostWidth, any alignment: a warp a head.
template <bool BWD>
__global__ void __launch_bounds__(kThreads) qk_general_kernel(const __grid_constant__ QkArgs p, int neighbours) {
  extern __shared__ float smem[];
  const int zero = ptx::grid_wait_previous();
  const QkPart& q = p.part[part_of(p, blockIdx.x)];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* xs = smem + (int64_t)warp * p.width * (BWD ? 3 : 1);
  float *gs = xs + p.width, *acc = xs + 2 * p.width;
  if (BWD)
    for (int e = lane; e < p.width; e += 32) acc[e] = 0.f;
  const int64_t units = p.rows * q.heads, step = (int64_t)q.ctas * kWarps;
  for (int64_t u = (int64_t)(blockIdx.x - q.first_cta) * kWarps + warp + zero; u < units; u += step) {
    const int64_t row = u / q.heads, head = u - row * q.heads;
    const int64_t at = row * q.x_ld + head * p.width, ag = row * q.g_ld + head * p.width, ay = row * q.y_ld + head * p.width;
    float ss = 0.f;
    for (int e = lane; e < p.width; e += 32) {
      const float v = load_one(q.x, q.x_dt, at + e);
      xs[e] = v;
      if (BWD) gs[e] = load_one(q.g, q.g_dt, ag + e);
      ss = fmaf(v, v, ss);
    }
    __syncwarp();
    const float r = rsqrtf(fmaf(warp_sum(ss), p.inv_width, p.eps));
    const float* t = p.table ? angles_of(p, row) : nullptr;
    auto weight = [&](int e) { return q.w ? load_one(q.w, q.w_dt, e) : 1.f; };
    // feature e of v turned (BACK: back)
    auto turned = [&](const float* v, int e, bool weighted) {
      int partner = e;
      bool first = true;
      const int pair = pair_of(p, neighbours != 0, e, partner, first);
      const float own = weighted ? v[e] * r * weight(e) : v[e];
      if (pair < 0) return own;
      const float other = weighted ? v[partner] * r * weight(partner) : v[partner];
      const float c = t ? t[2 * pair] : __int_as_float(0x7fffffff), s = t ? t[2 * pair + 1] : __int_as_float(0x7fffffff);
      return fmaf(own, c, (first != BWD ? -s : s) * other);
    };
    if (!BWD) {
      for (int e = lane; e < p.width; e += 32) store_one(q.y, q.y_dt, ay + e, turned(xs, e, true));
    } else {
      float dot = 0.f;
      for (int e = lane; e < p.width; e += 32) dot = fmaf(turned(gs, e, false) * weight(e), xs[e], dot);
      const float m = warp_sum(dot) * r * r * p.inv_width;
      for (int e = lane; e < p.width; e += 32) {
        const float n = turned(gs, e, false);
        acc[e] = fmaf(n, xs[e] * r, acc[e]);
        store_one(q.y, q.y_dt, ay + e, p.beta_x * r * fmaf(-xs[e], m, n * weight(e)));
      }
    }
    __syncwarp();
  }
  if (!BWD || !q.dw) return;
  __syncthreads();
  for (int c = threadIdx.x; c < p.width; c += kThreads) {
    float v = 0.f;
    for (int k = 0; k < kWarps; ++k) v += smem[(int64_t)(3 * k + 2) * p.width + c];
    p.partial[(int64_t)blockIdx.x * p.width + c] = v;
  }
}

// The CTAs' sums of weight gradients: 32 columns of a part a CTA, added by 32 warps in a fixed order.
__global__ void __launch_bounds__(1024) qk_weight_kernel(const __grid_constant__ QkArgs p) {
  __shared__ float s[32][33];
  const int zero = ptx::grid_wait_previous();
  const QkPart& q = p.part[blockIdx.y];
  if (!q.dw) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (c < p.width)
    for (int k = warp + zero; k < q.ctas; k += 32) v += __ldcg(p.partial + (int64_t)(q.first_cta + k) * p.width + c);
  s[warp][lane] = v;
  __syncthreads();
  const float t = warp_sum(s[lane][warp]);
  const int col = blockIdx.x * 32 + warp;
  if (lane == 0 && col < p.width) store_one(q.dw, q.dw_dt, col, q.beta_w * t);
}

__global__ void __launch_bounds__(kThreads) rotary_table_kernel(float* table, int64_t ld, int64_t rows, int pairs, double base, double scale, double first) {
  ptx::grid_wait_previous();
  const int64_t total = rows * pairs;
  for (int64_t k = blockIdx.x * (int64_t)kThreads + threadIdx.x; k < total; k += (int64_t)gridDim.x * kThreads) {
    const int64_t row = k / pairs, i = k - row * pairs;
    double s, c;
    sincos((first + (double)row) * scale * pow(base, -(double)i / (double)pairs), &s, &c);
    table[row * ld + 2 * i] = (float)c;
    table[row * ld + 2 * i + 1] = (float)s;
  }
}

// ---------------------------------------------------------------- host
bool is_input(int dt) { return dt == US_F32 || dt == US_BF16 || dt == US_F16; }

us_status check_mat(const us_mat& m, int64_t rows, int64_t cols, bool input) {
  if (m.rows != rows || m.cols != cols || m.ld < m.cols) return US_ERR_INVALID_ARG;
  if (m.dtype < US_F32 || m.dtype > US_E5M2) return US_ERR_INVALID_ARG;
  if (rows * cols > 0 && !m.ptr) return US_ERR_INVALID_ARG;
  if (input && !is_input(m.dtype)) return US_ERR_UNSUPPORTED;
  if (reinterpret_cast<uintptr_t>(m.ptr) % dtype_size(m.dtype)) return US_ERR_ALIGNMENT;
  return US_OK;
}
bool aligned(const us_mat& m, int bytes) {
  const int es = dtype_size(m.dtype);
  return reinterpret_cast<uintptr_t>(m.ptr) % bytes == 0 && m.ld * es % bytes == 0;
}

struct Call {
  QkArgs a{};
  bool vec = true, empty = false;
  int dt = -1;
};

us_status prepare(Call& c, int count, const us_mat* X, const us_mat* w, const us_mat* G, const us_mat* Y, const us_mat* dw, const float* beta_w,
                  int64_t width, float eps, const us_mat* table, const int32_t* positions, int64_t start, int64_t period, int neighbours) {
  if (count < 1 || count > kMostParts || !X || !Y || width < 1 || width > (1 << 20) || !(eps >= 0.f) || start < 0 || period < 0) return US_ERR_INVALID_ARG;
  if (neighbours != 0 && neighbours != 1) return US_ERR_INVALID_ARG;
  QkArgs& a = c.a;
  a.count = count; a.width = (int)width; a.rows = X[0].rows; a.eps = eps; a.inv_width = 1.0f / (float)width;
  if (a.rows < 0 || a.rows >= (1ll << 31)) return US_ERR_INVALID_ARG;
  const bool turns = table && table->ptr && table->cols > 0;
  if (turns) {
    const us_status s = check_mat(*table, table->rows, table->cols, true);
    if (s != US_OK) return s;
    if (table->dtype != US_F32) return US_ERR_UNSUPPORTED;
    if (table->rows < 1 || table->cols % 2 || table->cols > width) return US_ERR_INVALID_ARG;
    // positions on the host's side of the call are known to be in the table; those on the device are checked there
    if (!positions && a.rows > 0 && start + (period ? std::min(period, a.rows) : a.rows) > table->rows) return US_ERR_INVALID_ARG;
    if (positions && reinterpret_cast<uintptr_t>(positions) % 4) return US_ERR_ALIGNMENT;
    a.table = static_cast<const float*>(table->ptr); a.table_ld = table->ld; a.table_rows = table->rows;
    a.positions = positions; a.start = start; a.period = period < a.rows ? (uint32_t)period : 0; a.rotated = (int)table->cols;
    c.vec = c.vec && aligned(*table, 16) && a.rotated % (neighbours ? 8 : 16) == 0;
  }
  c.vec = c.vec && width % 8 == 0 && width <= kMostVecWidth;
  bool any = false;
  for (int k = 0; k < count; ++k) {
    QkPart& q = a.part[k];
    if (X[k].cols < 0 || X[k].cols % width || X[k].cols >= (1ll << 31)) return US_ERR_INVALID_ARG;
    us_status s = check_mat(X[k], a.rows, X[k].cols, true);
    if (s == US_OK) s = check_mat(Y[k], a.rows, X[k].cols, false);
    if (s == US_OK && G) s = check_mat(G[k], a.rows, X[k].cols, true);
    if (s != US_OK) return s;
    if (w && w[k].ptr) {
      s = check_mat(w[k], 1, width, true);
      if (s != US_OK) return s;
      q.w = w[k].ptr; q.w_dt = w[k].dtype;
    }
    if (dw && dw[k].ptr) {
      s = check_mat(dw[k], 1, width, true);
      if (s != US_OK) return s;
      q.dw = dw[k].ptr; q.dw_dt = dw[k].dtype; q.beta_w = beta_w ? beta_w[k] : 1.f;
      if (!q.w) return US_ERR_INVALID_ARG;
    }
    q.x = X[k].ptr; q.x_dt = X[k].dtype; q.x_ld = X[k].ld;
    q.y = Y[k].ptr; q.y_dt = Y[k].dtype; q.y_ld = Y[k].ld;
    if (G) { q.g = G[k].ptr; q.g_dt = G[k].dtype; q.g_ld = G[k].ld; }
    q.heads = (int)(X[k].cols / width);
    any = any || q.heads > 0 || q.dw;
    // the vector kernels take parts of one input type (its gradients too)
    if (c.dt < 0) c.dt = q.x_dt;
    c.vec = c.vec && q.x_dt == c.dt && aligned(X[k], 16) && aligned(Y[k], dtype_size(Y[k].dtype) == 1 ? 8 : 16) &&
            (!G || (q.g_dt == c.dt && aligned(G[k], 16)));
  }
  c.empty = !any || (a.rows == 0 && !dw);
  return US_OK;
}

// Deals the CTAs to the parts by their heads; returns the grid.
int deal(QkArgs& a, int per_block, int most) {
  int64_t all = 0;
  for (int k = 0; k < a.count; ++k) {
    QkPart& q = a.part[k];
    q.blocks = (q.heads + per_block - 1) / per_block;
    q.d_blocks = make_fast_div(std::max(1, q.blocks));
    all += a.rows * q.heads;
  }
  int grid = 0;
  for (int k = 0; k < a.count; ++k) {
    QkPart& q = a.part[k];
    const int64_t units = a.rows * q.blocks, want = (units + kWarps - 1) / kWarps;
    const int64_t share = all > 0 ? ((int64_t)most * a.rows * q.heads + all / 2) / all : 0;
    q.first_cta = grid;
    q.ctas = (int)std::max<int64_t>(1, std::min(want, share));
    grid += q.ctas;
  }
  return grid;
}

template <bool BWD, int DT, int ITER>
us_status launch_vec(const Call& c, int neighbours, int grid, cudaStream_t st) {
  if constexpr (BWD)
    return neighbours ? host::launch(qk_bwd_kernel<DT, ITER, true>, nullptr, grid, kThreads, 0, 1, st, c.a)
                      : host::launch(qk_bwd_kernel<DT, ITER, false>, nullptr, grid, kThreads, 0, 1, st, c.a);
  else
    return neighbours ? host::launch(qk_fwd_kernel<DT, ITER, true>, nullptr, grid, kThreads, 0, 1, st, c.a)
                      : host::launch(qk_fwd_kernel<DT, ITER, false>, nullptr, grid, kThreads, 0, 1, st, c.a);
}
template <bool BWD, int DT>
us_status pick_iter(const Call& c, int iter, int neighbours, int grid, cudaStream_t st) {
  if constexpr (!BWD) {
    if (iter >= 4) return launch_vec<BWD, DT, 4>(c, neighbours, grid, st);
  }
  if constexpr (!BWD || DT != US_F32) {
    if (iter >= 2) return launch_vec<BWD, DT, 2>(c, neighbours, grid, st);
  }
  return launch_vec<BWD, DT, 1>(c, neighbours, grid, st);
}

template <bool BWD>
us_status issue(Call& c, int neighbours, cudaStream_t st) {
  const int sms = host::sm_count();
  if (sms <= 0) return US_ERR_CUDA;
  QkArgs& a = c.a;
  if (!c.vec) {
    if (a.width > kMostWidth) return US_ERR_UNSUPPORTED;
    const int grid = deal(a, 1, sms * (BWD ? kBwdCtasPerSm : kFwdCtasPerSm));
    const size_t smem = (size_t)kWarps * a.width * sizeof(float) * (BWD ? 3 : 1);
    static std::atomic<uint64_t> smem_set{0};
    constexpr size_t most = (size_t)kWarps * kMostWidth * sizeof(float) * (BWD ? 3 : 1);
    return host::launch_plain(qk_general_kernel<BWD>, &smem_set, grid, kThreads, (int)most, smem, st, a, neighbours);
  }
  const int chunks = a.width / 8;
  a.lanes = neighbours ? (chunks + 1) / 2 : a.rotated / 16 + (chunks - a.rotated / 8 + 1) / 2;
  for (a.group = 1; a.group < a.lanes; a.group *= 2) {}
  const int per = 32 / a.group;
  int heads = 1;
  for (int k = 0; k < a.count; ++k) heads = std::max(heads, a.part[k].heads);
  const int steps = (heads + per - 1) / per, most_iter = !BWD ? 4 : c.dt == US_F32 ? 1 : 2;       // (what the registers hold)
  int iter = steps >= most_iter ? most_iter : steps >= 2 ? 2 : 1;
  // few tokens: a step to a warp, so that all of them are under way at once
  while (iter > 1 && a.rows * ((steps + iter - 1) / iter) < (int64_t)sms * kWarps) iter /= 2;
  const int grid = deal(a, per * iter, sms * (BWD ? kBwdCtasPerSm : kFwdCtasPerSm));
  if (c.dt == US_F32) return pick_iter<BWD, US_F32>(c, iter, neighbours, grid, st);
  return c.dt == US_BF16 ? pick_iter<BWD, US_BF16>(c, iter, neighbours, grid, st) : pick_iter<BWD, US_F16>(c, iter, neighbours, grid, st);
}

}  // namespace
}  // namespace us

using namespace us;

extern "C" us_status us_qk_norm_fwd(int count, const us_mat* X, const us_mat* w, const us_mat* Y, int64_t head_width, float eps, const us_mat* table,
                                    const int32_t* positions, int64_t start, int64_t period, int neighbours, void* stream) {
  Call c;
  const us_status s = prepare(c, count, X, w, nullptr, Y, nullptr, nullptr, head_width, eps, table, positions, start, period, neighbours);
  if (s != US_OK) return s;
  if (head_width > kMostWidth) return US_ERR_UNSUPPORTED;
  if (c.empty) return US_OK;
  return issue<false>(c, neighbours, static_cast<cudaStream_t>(stream));
}

extern "C" size_t us_qk_norm_bwd_workspace_bytes(int64_t head_width) {
  if (head_width < 1 || head_width > kMostWidth) return 0;
  const int sms = host::sm_count();
  return (size_t)((sms > 0 ? sms : 1) * kBwdCtasPerSm + 2 * kMostParts) * (size_t)head_width * sizeof(float);
}

extern "C" us_status us_qk_norm_bwd(int count, const us_mat* X, const us_mat* w, const us_mat* G, const us_mat* dX, const us_mat* dw, const float* beta_w,
                                    int64_t head_width, float eps, float beta_x, const us_mat* table, const int32_t* positions, int64_t start,
                                    int64_t period, int neighbours, void* ws, size_t ws_bytes, void* stream) {
  if (!G) return US_ERR_INVALID_ARG;
  Call c;
  us_status s = prepare(c, count, X, w, G, dX, dw, beta_w, head_width, eps, table, positions, start, period, neighbours);
  if (s != US_OK) return s;
  if (head_width > kMostWidth) return US_ERR_UNSUPPORTED;
  bool sums = false;
  for (int k = 0; k < count; ++k) sums = sums || c.a.part[k].dw;
  if (sums) {
    if (!ws || ws_bytes < us_qk_norm_bwd_workspace_bytes(head_width)) return US_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(ws) % 16) return US_ERR_ALIGNMENT;
  }
  if (c.empty) return US_OK;
  c.a.beta_x = beta_x;
  c.a.partial = static_cast<float*>(ws);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  s = issue<true>(c, neighbours, st);
  if (s != US_OK || !sums) return s;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((head_width + 31) / 32), (unsigned)count);
  cfg.blockDim = dim3(1024);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 1;
  void* params[] = {&c.a};
  return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(qk_weight_kernel), params) == cudaSuccess ? US_OK : host::failed();
}

extern "C" us_status us_rotary_table(const us_mat* table, double base, double scale, int64_t first, void* stream) {
  if (!table || first < 0 || !(base > 0.0) || !(scale > 0.0)) return US_ERR_INVALID_ARG;
  if (table->rows < 0 || table->cols < 0 || table->cols % 2) return US_ERR_INVALID_ARG;
  const us_status s = check_mat(*table, table->rows, table->cols, true);
  if (s != US_OK) return s;
  if (table->dtype != US_F32) return US_ERR_UNSUPPORTED;
  const int64_t total = table->rows * (table->cols / 2);
  if (total == 0) return US_OK;
  const int sms = host::sm_count();
  if (sms <= 0) return US_ERR_CUDA;
  const int grid = (int)std::min<int64_t>((total + kThreads - 1) / kThreads, (int64_t)sms * 8);
  return host::launch(rotary_table_kernel, nullptr, grid, kThreads, 0, 1, static_cast<cudaStream_t>(stream), static_cast<float*>(table->ptr), table->ld,
                      table->rows, (int)(table->cols / 2), base, scale, (double)first);
}
