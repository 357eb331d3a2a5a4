// us_bias_grad: gradients of biases, the column sums of the gradients of linear layers' outputs, for several matrices in one launch.
//
// Bound by the bytes of G, which the matmuls around it have just written or read.  A cluster of CTAs shares a strip of columns 128 bytes
// wide: each CTA sums its part of the rows (a thread 16 bytes of every 32nd row), the CTAs' sums meet in shared memory, and
// every CTA finishes some of the strip's columns.  One launch, no workspace and no atomics.  The next grid is not released early (several CTAs an SM): captured steps of an FFN block with biases, us,
// 256 x 128 x 512 13.6 -> 11.9, though 1000 x 528 x 2096 26.5 -> 27.4; in a row, 8192 x 4096 E5M2 7.3 -> 6.0, BF16 9.3 -> 7.4.
#include <algorithm>

#include "common.cuh"
#include "host.h"
#include "sm100.cuh"

namespace us {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMostParts = 8, kStripBytes = 128;
constexpr int kStep = kThreads / 8;          // rows that a CTA has side by side
constexpr int kAhead = 16;                   // rows that a thread has in flight,
constexpr int kRest = 8;                     // and where fewer are left

struct BiasPart {
  const void* g;
  void* out;
  int64_t rows, ld;
  int cols, strip_end;                       // strips up to and including this matrix
  int g_dt, out_dt, wide;                    // wide: rows start on 16-byte boundaries
  float beta;
};
struct BiasArgs {
  BiasPart part[kMostParts];
  int count;
};

// acc += each of two 16-bit numbers, widened by the addition itself.
template <bool BF16>
__device__ __forceinline__ void add_halves(uint32_t w, float& a, float& b) {
  if (BF16) asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.bf16 %0, l, %0;\n\tadd.rn.f32.bf16 %1, h, %1;\n\t}" : "+f"(a), "+f"(b) : "r"(w));
  else asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.f16 %0, l, %0;\n\tadd.rn.f32.f16 %1, h, %1;\n\t}" : "+f"(a), "+f"(b) : "r"(w));
}
// Two FP8 codes as F16 numbers; a code of E5M2 is the upper half of one.  (The additions that widen, and E5M2 codes put in their places instead of converted, took an
// 8192 x (4096 + 1024) E5M2 block from 12.2 to 11.4 us: beside the bytes it costs one addition and half a permutation per element.)
template <int DT, int HIGH>
__device__ __forceinline__ uint32_t fp8_halves(uint32_t w) {
  if (DT == US_E5M2) return __byte_perm(w, 0u, HIGH ? 0x3424 : 0x1404);
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(HIGH ? w >> 16 : w)));
  return h;
}

template <int DT>
__device__ __forceinline__ void add16(const uint4& t, float* acc) {
  const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (DT == US_F32) {
      acc[j] += __uint_as_float(w[j]);
    } else if (DT == US_BF16 || DT == US_F16) {
      add_halves<DT == US_BF16>(w[j], acc[2 * j], acc[2 * j + 1]);
    } else {
      add_halves<false>(fp8_halves<DT, 0>(w[j]), acc[4 * j], acc[4 * j + 1]);
      add_halves<false>(fp8_halves<DT, 1>(w[j]), acc[4 * j + 2], acc[4 * j + 3]);
    }
  }
}

// 16 bytes, or zeros; a predicated load (of a conditional one the compiler makes a branch, which keeps the next load waiting).
__device__ __forceinline__ uint4 load16_if(bool there, const void* at) {
  uint4 t;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
               "@p ld.global.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}" : "=&r"(t.x), "=&r"(t.y), "=&r"(t.z), "=&r"(t.w) : "l"(at), "r"((int)there));
  return t;
}

// Sums of a strip's columns over rows first .. end - 1, one line of `sums` (kStripBytes / element size columns) per warp.
template <int DT>
__device__ __forceinline__ void strip_sums(const BiasPart& p, int strip, int64_t first, int64_t end, float (*sums)[kStripBytes]) {
  constexpr int kEs = DT == US_F32 ? 4 : DT == US_BF16 || DT == US_F16 ? 2 : 1, kCols = kStripBytes / kEs, kChunk = 16 / kEs;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (p.wide) {
    const int chunk = lane & 7, col = strip * kCols + chunk * kChunk, cols = p.cols - col;
    float acc[kChunk] = {};
    if (cols > 0) {
      // The last piece of a row may be cut by the matrix's last column.  It is read whole where a row follows.
      const bool cut = cols < kChunk;
      const int64_t whole = cut ? min(end, p.rows - 1) : end;
      const char* g = static_cast<const char*>(p.g) + (int64_t)col * kEs;
      const int64_t pitch = p.ld * kEs;
      int64_t r = first + warp * 4 + (lane >> 3);
      for (; r + kStep * (kAhead - 1) < whole; r += kStep * kAhead) {
        uint4 t[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) t[k] = *reinterpret_cast<const uint4*>(g + (r + kStep * k) * pitch);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) add16<DT>(t[k], acc);
      }
      for (; r < whole; r += kStep * kRest) {                  // (of rows that are not there, zeros)
        uint4 t[kRest];
#pragma unroll
        for (int k = 0; k < kRest; ++k) t[k] = load16_if(r + kStep * k < whole, g + (r + kStep * k) * pitch);
#pragma unroll
        for (int k = 0; k < kRest; ++k) add16<DT>(t[k], acc);
      }
      if (cut && end == p.rows && (p.rows - 1 - first) % kStep == warp * 4 + (lane >> 3)) {    // the matrix's last row
#pragma unroll
        for (int i = 0; i < kChunk; ++i)
          if (i < cols) acc[i] += load_one(p.g, DT, (p.rows - 1) * p.ld + col + i);
      }
    }
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
      acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 8);
      acc[i] += __shfl_xor_sync(0xffffffffu, acc[i], 16);
    }
    if (lane < 8) {
#pragma unroll
      for (int i = 0; i < kChunk; ++i) sums[warp][chunk * kChunk + i] = acc[i];
    }
  } else {
    // A lane has every 32nd column of every 8th row, kRows of them at a time (behind the last row, that one and not added); lanes behind the last column have that
    // one's too.
    constexpr int kRows = kEs == 1 ? 8 : 16;
    float acc[kCols / 32] = {};
    int col[kCols / 32];
#pragma unroll
    for (int j = 0; j < kCols / 32; ++j) col[j] = min(strip * kCols + 32 * j + lane, p.cols - 1);
    const char* g = static_cast<const char*>(p.g);
    const int64_t pitch = p.ld * kEs;
    for (int64_t r = first + warp; r < end; r += kWarps * kRows) {
      const int left = (int)min((end - 1 - r) / kWarps, (int64_t)kRows - 1);
      float x[kRows][kCols / 32];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const char* row = g + (r + kWarps * min(k, left)) * pitch;
#pragma unroll
        for (int j = 0; j < kCols / 32; ++j) x[k][j] = load_one(row, DT, col[j]);
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
#pragma unroll
        for (int j = 0; j < kCols / 32; ++j) acc[j] += k <= left ? x[k][j] : 0.f;
      }
    }
#pragma unroll
    for (int j = 0; j < kCols / 32; ++j) sums[warp][32 * j + lane] = acc[j];
  }
}

// (Registers for three CTAs an SM: with four the loads in flight do not fit, 8192 x (4096 + 1024) E5M2 9.7 us in the place of 8.0; with two 10.9.)
__global__ void __launch_bounds__(kThreads, 3) bias_grad_kernel(const __grid_constant__ BiasArgs a) {
  __shared__ float sums[kWarps][kStripBytes];
  __shared__ float mine[kStripBytes];
  (void)ptx::grid_wait_previous();
  const int parts = (int)ptx::cluster_nctarank(), rank = (int)ptx::cluster_ctarank();
  int strip = blockIdx.x / parts, k = 0;
  while (strip >= a.part[k].strip_end) ++k;
  const BiasPart& p = a.part[k];
  if (k > 0) strip -= a.part[k - 1].strip_end;
  const int64_t first = p.rows * rank / parts, end = p.rows * (rank + 1) / parts;
  switch (p.g_dt) {
    case US_F32: strip_sums<US_F32>(p, strip, first, end, sums); break;
    case US_BF16: strip_sums<US_BF16>(p, strip, first, end, sums); break;
    case US_F16: strip_sums<US_F16>(p, strip, first, end, sums); break;
    case US_E4M3: strip_sums<US_E4M3>(p, strip, first, end, sums); break;
    default: strip_sums<US_E5M2>(p, strip, first, end, sums); break;
  }
  __syncthreads();
  const int cols = kStripBytes / dtype_size(p.g_dt), i = threadIdx.x, col = strip * cols + i;
  float s = 0.f;
  if (i < cols) {
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += sums[w][i];
    mine[i] = s;
  }
  if (parts > 1) {
    ptx::cluster_sync();
    const int share = (cols + parts - 1) / parts;                            // columns that a CTA finishes
    if (i < cols && i / share == rank) {
      s = 0.f;
      for (int r = 0; r < parts; ++r) s += ptx::ld_cluster(ptx::in_cta(ptx::smem_addr(&mine[i]), (uint32_t)r));
    }
    if (i < cols && i / share == rank && col < p.cols) store_one(p.out, p.out_dt, col, p.beta * s);
    ptx::cluster_meet();                                       // nobody leaves while its sums are being read
  } else if (i < cols && col < p.cols) {
    store_one(p.out, p.out_dt, col, p.beta * s);
  }
}

us_status check(const us_mat& G, const us_mat& db) {
  for (const us_mat* m : {&G, &db})
    if (m->dtype < US_F32 || m->dtype > US_E5M2 || m->rows < 0 || m->cols < 0 || m->rows >= (1ll << 31) || m->cols >= (1ll << 31) - kStripBytes) return US_ERR_INVALID_ARG;
  if (db.rows != 1 || db.cols != G.cols) return US_ERR_INVALID_ARG;
  if (db.dtype == US_E4M3 || db.dtype == US_E5M2) return US_ERR_UNSUPPORTED;
  if (G.cols == 0) return US_OK;
  if (!db.ptr || (G.rows > 0 && (!G.ptr || G.ld < G.cols))) return US_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(db.ptr) % dtype_size(db.dtype) || (G.rows > 0 && reinterpret_cast<uintptr_t>(G.ptr) % dtype_size(G.dtype))) return US_ERR_ALIGNMENT;
  return US_OK;
}

}  // namespace
}  // namespace us

using namespace us;

extern "C" us_status us_bias_grad(int count, const us_mat* G, const float* beta, const us_mat* db, void* stream) {
  if (count < 1 || count > kMostParts || !G || !db) return US_ERR_INVALID_ARG;
  BiasArgs a{};
  int64_t strips = 0, rows = 0;
  bool wide = true;
  for (int k = 0; k < count; ++k) {
    const us_status s = check(G[k], db[k]);
    if (s != US_OK) return s;
    BiasPart& p = a.part[k];
    const int es = dtype_size(G[k].dtype);
    p.g = G[k].ptr; p.out = db[k].ptr; p.rows = G[k].rows; p.ld = G[k].ld; p.cols = (int)G[k].cols;
    p.g_dt = G[k].dtype; p.out_dt = db[k].dtype; p.beta = beta ? beta[k] : 1.f;
    p.wide = reinterpret_cast<uintptr_t>(p.g) % 16 == 0 && (p.rows <= 1 || p.ld * es % 16 == 0);
    strips += (G[k].cols * es + kStripBytes - 1) / kStripBytes;
    if (strips * 8 >= (1ll << 31)) return US_ERR_UNSUPPORTED;
    p.strip_end = (int)strips;
    rows = std::max(rows, G[k].rows);
    wide = wide && p.wide;
  }
  if (strips == 0) return US_OK;
  a.count = count;
  // At most the three CTAs an SM that run at once, of at least 128 rows each, and no cluster for up to 1024 rows: more of them, or the cluster's launch and barriers, cost more
  // than they share (us, E5M2: 1024 x (4096 + 1024) 3.6 alone, 4.1 shared by two; 1500 x (512 + 128) 4.3 alone, 3.5 by eight).  Powers of two: 8192 x (4096 + 1024) BF16 takes
  // 15.7 with clusters of four and 18.5 with five.  Rows that are not aligned, which take longer, are shared from 129 on, 64 at least for each (up to four CTAs
  // an SM, of which three run at once: 8192 x 4097 BF16 23.8 in the place of 19.7, 600 x 8191 9.2 of 5.8, nowhere less).
  const int sms = host::sm_count();
  if (sms <= 0) return US_ERR_CUDA;
  int parts = 1;
  while (parts < 8 && rows > (wide ? 1024 : 128) && strips * parts * 2 <= 3 * sms && rows >= (wide ? 256 : 128) * parts) parts *= 2;
  return host::launch(bias_grad_kernel, nullptr, (int)strips * parts, kThreads, 0, parts, static_cast<cudaStream_t>(stream), a);
}
