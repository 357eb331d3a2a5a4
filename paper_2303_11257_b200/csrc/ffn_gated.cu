// us_ffn_gated_fwd / us_ffn_gated_bwd: the hidden layer of a gated FFN block, one launch each way.
//
//   forward    h = alpha X Wg,  u = alpha X Wu,  A = round(act_out * f(act_in * h) * u),  H, U = round(h), round(u)     (optional)
//   backward   dA = beta_x G W2^T,  dU = round(beta_u * f(act_in * H) * dA),  dH = round(beta_h * act_in * f'(act_in * H) * U * dA)
//
// One warp-specialised persistent tcgen05 kernel for both: warp 0 fetches operand stages by TMA, one thread of warp 1 issues the MMAs,
// the other warps turn finished accumulators into results, while the MMAs of the next tile run.  Forward, a tile is HC hidden columns of
// both projections side by side in one accumulator: B is HC columns of Wg followed by HC columns of Wu, one MMA multiplies both by the same
// A tile, and a lane finds h and u of the same element HC columns apart.  (Of a CTA pair the even CTA fetches Wg's half of B, the odd one
// Wu's.)  Neither projection is written unless the caller wants the copies the backward pass reads; those are 16-bit or, at unit scale, E4M3
// without a factor.  Backward, a tile is HC columns of dA, from which the epilogue makes both gradients with the copies it has fetched.
//
// Bound, us from one GPU to another, launches over seconds (power cap) / in a burst: forward the tensor pipe and power: 8192 x 1024 x 4096 BF16 with copies 120 to 133 / 98 to 110
// (F16 140 / 115), FP8 with copies in BF16 79 / 65, 16384 x 2048 x 8192 FP8 with copies in E4M3 429 to 478 / 407 (2.3 to 2.7 PFLOP/s).  Backward, BF16 85 to 90 / 75 (268 MB of copies and gradients beside
// 69 GFLOP: the SM's memory path), FP8 from E4M3 copies 53 to 56 / 46, from BF16 copies 63 / 54: the epilogue, by the latency of its chain (no unit above 55 %; a warp waits for fixed latencies, the
// accumulator's loads and other warps in turn).  One token of 1024 x 4096 in BF16 5.3, FP8 4.1 in a graph; 64 tokens the same.
//
// Every wait is bounded as in the other GEMM kernels.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "gemm_kernel.cuh"
#include "host.h"

namespace us {
namespace {

// Epilogue warps.  Of a CTA pair's tiles sixteen a CTA, whose arithmetic is the longest part of an FP8 tile; backward with 16-bit operands, where the MMAs
// take twice as long, eight.  (8192 x 1024 x 4096 backward, us, sixteen / eight: FP8 54.0 / 57.5, BF16 90.9 / 88.3.)
// (With sixteen the forward kernel whose results leave by the lanes spills 28 bytes at the 96 registers that a thread has; with 60 bytes it took the same time.)
__host__ __device__ constexpr bool gated_few(bool bwd, int es, int cg) { return cg == 1 || (bwd && es == 2); }
__host__ __device__ constexpr int gated_ew(bool bwd, int es, int cg) { return gated_few(bwd, es, cg) ? 8 : 16; }
constexpr int kRoom = 229376;                 // shared memory for stages and the epilogue's boxes
constexpr int kMostStages = 16;
// Backward, an epilogue warp has slots for the copies of h and u that arrive and the dH and dU that leave, in boxes of 32 rows x 32 columns.  Where copies and gradients have one
// width a gradient leaves from the box of its copy, and there are three slots: a store has a unit's time to read one before it is filled again (8192 x 1024 x 4096, two / three / four slots, the last in a stage's room:
// BF16 92.7 / 84.7 / 91.8 us, FP8 56.8 / 53.3 / 54.8).  Elsewhere a slot has
// boxes for both (6144 bytes), in as many slots as fit: two of eight warps, one of sixteen (FP8 from 16-bit copies, 63 us at that size, where the bytes take 33: the copies of
// a unit are asked for when the one before has been stored).
constexpr int kMostSlots = 3;
__host__ __device__ constexpr int epi_room(int ew) { return ew == 16 ? 6144 : 12288; }      // bytes of a warp

struct GatedParams {
  int M, N, K;                                // results are [M x N]; length of the contraction
  int tiles_m, tiles_n;
  int band_m, full_bands;                     // tile rows of a band of the tile order, and the bands that have as many
  FastDiv d_band, d_rows, d_rows_last;        // by band_m * tiles_n, band_m, tiles_m % band_m
  uint32_t idesc;
  float scale;                                // alpha / beta_x
  float act_in, c0, c1;                       // c0: act_out / beta_u; c1: - / beta_h * act_in
  int fn;
  int kept_dt, out_dt;                        // types of the copies of h and u, and of the results
  uint8_t *h, *u, *o0; long long h_ld, u_ld, o0_ld; int kept_sectors, out_sectors;     // forward: the copies (nullptr: not wanted) and A
  int slots;                                  // backward: slots of an epilogue warp
  unsigned int* status;
  uint32_t wait_limit;
  uint32_t a_bytes; int stages;               // bytes of A in a stage (single CTAs: the rows that exist), and the stages that fit
  int starved, served;                        // test hook (starved_cta)
};

template <bool BWD, int ES, int HC, int CG, bool BOXED = false>
struct GatedShape {
  static constexpr int kN = BWD ? HC : 2 * HC;             // columns of an accumulator
  static constexpr int kEW = gated_ew(BWD, ES, CG);         // epilogue warps
  static constexpr int kRowsB = kN / CG;                   // rows of B a CTA fetches
  static constexpr int kBBytes = kRowsB * kStageKBytes;
  static constexpr int kStageBytes = kBM * kStageKBytes + kBBytes;
  static constexpr int kEpiBytes = BWD ? kEW * epi_room(kEW) : BOXED ? kEW * 3 * 2048 : 0;
  static constexpr int kStages = (kRoom - kEpiBytes) / kStageBytes;
  static constexpr int kBarrierBytes = 1024;
  static constexpr int kTotal = kRoom + kBarrierBytes + 1024;
  // Forward: B is N-major, in chunks of rows of K: 128 bytes wide, or the columns of one projection where they are fewer
  static constexpr int kChunkRow = CG == 2 || HC * ES >= 128 ? 128 : HC * ES;
  static constexpr int kChunkBytes = (kStageKBytes / ES) * kChunkRow;
  static constexpr int kWarpCols = HC / (kEW / 4);    // hidden columns of an epilogue warp
};

// ---------------------------------------------------------------- the gate
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two values at a time (packed float32 arithmetic): x holds pre-activations, in2 = splat(act_in), nl2 = splat(-act_in log2 e).
// sigmoid(act_in x) = 1 / (1 + e^-z): relative error of a few 2^-22 and |z| 2^-23, far inside a step of the 16 and 8 bits that results are rounded to.
__device__ __forceinline__ f32x2 sigmoid2(f32x2 x, f32x2 nl2) {
  float p0, p1;
  unpack2(mul2(x, nl2), p0, p1);
  unpack2(add2(pack2(ex2_approx(p0), ex2_approx(p1)), splat2(1.0f)), p0, p1);
  return pack2(rcp_approx(p0), rcp_approx(p1));
}
// min(x, m), or x where that is NaN.
__device__ __forceinline__ float min_nan(float x, float m) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(m));
  return r;
}
// s = sigmoid(z) and c = 1 - s = e^-z s, z = act_in x.  (1 - s itself cancels where s is close to 1: the slope s c would be 1 % off at z = 12, and nothing from 17 on.)
// e^-z is kept finite, so that c stays a number where s is nothing.
__device__ __forceinline__ void sigmoid_both2(f32x2 x, f32x2 nl2, f32x2& s, f32x2& c) {
  float p0, p1;
  unpack2(mul2(x, nl2), p0, p1);
  const f32x2 e = pack2(ex2_approx(min_nan(p0, 127.f)), ex2_approx(min_nan(p1, 127.f)));
  unpack2(add2(e, splat2(1.0f)), p0, p1);
  s = pack2(rcp_approx(p0), rcp_approx(p1));
  c = mul2(e, s);
}
// tanh(z) = 2 s - 1 with s = sigmoid(2 z), which cancels near zero: there z - z^3 / 3 + 2 z^5 / 15, whose next term is 2^-22 of it at 1/8.
__device__ __forceinline__ f32x2 tanh2(f32x2 z, f32x2 s) {
  float z0, z1, f0, f1, n0, n1;
  const f32x2 zz = mul2(z, z);
  unpack2(mul2(z, fma2(zz, fma2(zz, splat2(2.0f / 15.0f), splat2(-1.0f / 3.0f)), splat2(1.0f))), n0, n1);
  unpack2(fma2(s, splat2(2.0f), splat2(-1.0f)), f0, f1);
  unpack2(z, z0, z1);
  return pack2(fabsf(z0) < 0.125f ? n0 : f0, fabsf(z1) < 0.125f ? n1 : f1);
}
__device__ __forceinline__ f32x2 normal_cdf2(f32x2 z) {
  float z0, z1, q0, q1;
  unpack2(z, z0, z1);
  normal_tail2(sat_mul_abs(z0, 1.0f / kTailRange), sat_mul_abs(z1, 1.0f / kTailRange), q0, q1);
  return pack2(z0 >= 0.f ? 1.0f - q0 : q0, z1 >= 0.f ? 1.0f - q1 : q1);
}
// f(act_in x)
template <int FN>
__device__ __forceinline__ f32x2 gate_value2(f32x2 x, f32x2 in2, f32x2 nl2) {
  if (FN == US_FN_SILU) return mul2(mul2(x, in2), sigmoid2(x, nl2));
  if (FN == US_FN_SIGMOID) return sigmoid2(x, nl2);
  if (FN == US_FN_TANH) return tanh2(mul2(x, in2), sigmoid2(x, add2(nl2, nl2)));
  const f32x2 z = mul2(x, in2);
  if (FN == US_FN_GELU) return mul2(z, normal_cdf2(z));
  float z0, z1;
  unpack2(z, z0, z1);
  return pack2(act_value(US_FN_RELU, z0), act_value(US_FN_RELU, z1));
}
// Both gradients of a product: yh = c1 f'(act_in x) u d, yu = c0 f(act_in x) d; c0, c1 splat.
template <int FN>
__device__ __forceinline__ void gate_grads2(f32x2 x, f32x2 u, f32x2 d, float act_in, f32x2 nl2, f32x2 c0, f32x2 c1, f32x2& yh, f32x2& yu) {
  const f32x2 one = splat2(1.0f), in2 = splat2(act_in);
  f32x2 f, df;
  if (FN == US_FN_SILU) {                                 // f' = s (1 + z (1 - s)), f = z s; c0 holds act_in, too
    const f32x2 s = sigmoid2(x, nl2), g = mul2(s, d);
    yu = mul2(mul2(g, x), c0);
    yh = mul2(mul2(mul2(g, fma2(x, fma2(s, splat2(-act_in), in2), one)), u), c1);
    return;
  }
  if (FN == US_FN_SIGMOID) {
    f32x2 c;
    sigmoid_both2(x, nl2, f, c);
    df = mul2(f, c);
  } else if (FN == US_FN_TANH) {
    f32x2 s, c;
    sigmoid_both2(x, add2(nl2, nl2), s, c);
    f = tanh2(mul2(x, in2), s);
    df = mul2(mul2(s, splat2(4.0f)), c);
  } else {
    const f32x2 z = mul2(x, in2);
    float z0, z1;
    if (FN == US_FN_GELU) {
      const f32x2 Phi = normal_cdf2(z);
      unpack2(mul2(mul2(splat2(-0.72134752044448170f), z), z), z0, z1);
      f = mul2(z, Phi);
      df = fma2(mul2(z, splat2(0.39894228040143268f)), pack2(ex2_approx(z0), ex2_approx(z1)), Phi);
    } else {
      unpack2(z, z0, z1);
      f = pack2(act_value(US_FN_RELU, z0), act_value(US_FN_RELU, z1));
      df = pack2(z0 > 0.f ? 1.0f : z0 <= 0.f ? 0.f : z0, z1 > 0.f ? 1.0f : z1 <= 0.f ? 0.f : z1);          // NaN of NaN
    }
  }
  yh = mul2(mul2(mul2(c1, df), u), d);
  yu = mul2(mul2(c0, f), d);
}

// What is computed from v is computed behind this, and behind the stores before it: of the halves of a unit one after the other, because both at once do not
// fit the registers.
template <int N>
__device__ __forceinline__ void from_here(uint32_t (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(v[i]));
}
template <int N, class G>
__device__ __forceinline__ void unrolled(G g) {              // g(0) .. g(N - 1), the argument as a constant
  if constexpr (N > 0) {
    unrolled<N - 1>(g);
    g(std::integral_constant<int, N - 1>());
  }
}
// Calls g with the launch's activation as a constant.
template <class G>
__device__ __forceinline__ void with_gate(int fn, G g) {
  if (fn == US_FN_SILU) g(std::integral_constant<int, US_FN_SILU>());
  else if (fn == US_FN_SIGMOID) g(std::integral_constant<int, US_FN_SIGMOID>());
  else if (fn == US_FN_TANH) g(std::integral_constant<int, US_FN_TANH>());
  else if (fn == US_FN_GELU) g(std::integral_constant<int, US_FN_GELU>());
  else g(std::integral_constant<int, US_FN_RELU>());
}
// ---------------------------------------------------------------- a lane's S columns of a row (16 or 32)
// S results rounded to dt, packed.
template <int S>
__device__ __forceinline__ void pack_row(int dt, const float (&y)[S], uint32_t (&w)[S / 2]) {
  if (dt == US_BF16) {
#pragma unroll
    for (int i = 0; i < S / 2; ++i) w[i] = pack_bf16x2(y[2 * i], y[2 * i + 1]);
  } else if (dt == US_F16) {
#pragma unroll
    for (int i = 0; i < S / 2; ++i) w[i] = pack_f16x2(y[2 * i], y[2 * i + 1]);
  } else if (dt == US_E4M3) {
#pragma unroll
    for (int i = 0; i < S / 4; ++i) w[i] = cvt_fp8x4<false>(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < S / 4; ++i) w[i] = cvt_fp8x4<true>(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
  }
}
// Those to memory; cols of them exist.  sectors: rows start on 32-byte boundaries (otherwise on 16-byte ones).
template <int S>
__device__ __forceinline__ void put_row(uint8_t* dst, int es, const uint32_t (&w)[S / 2], int cols, bool sectors) {
  if (cols >= S) {
    if (es == 2) {
#pragma unroll
      for (int i = 0; i < S / 16; ++i) {
        if (sectors) {
          ptx::stg256(dst + 32 * i, &w[8 * i]);
        } else {
          reinterpret_cast<uint4*>(dst)[2 * i] = make_uint4(w[8 * i], w[8 * i + 1], w[8 * i + 2], w[8 * i + 3]);
          reinterpret_cast<uint4*>(dst)[2 * i + 1] = make_uint4(w[8 * i + 4], w[8 * i + 5], w[8 * i + 6], w[8 * i + 7]);
        }
      }
    } else if (S == 32 && sectors) {
      ptx::stg256(dst, w);
    } else {
#pragma unroll
      for (int i = 0; i < S / 16; ++i) reinterpret_cast<uint4*>(dst)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (i < cols) {
        if (es == 2) reinterpret_cast<uint16_t*>(dst)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        else dst[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
      }
  }
}
// Columns 2 i and 2 i + 1 of a row of stored words of type KEPT.
template <int KEPT, int N>
__device__ __forceinline__ f32x2 widen2(const uint32_t (&w)[N], int i) {
  const float2 v = KEPT == US_E4M3 ? unpack_fp8x2((uint16_t)(w[i >> 1] >> (16 * (i & 1))), false) : KEPT == US_BF16 ? unpack_bf16x2(w[i]) : unpack_f16x2(w[i]);
  return pack2(v.x, v.y);
}
// Sixteen results rounded to type DT, packed: four words of 8-bit ones, eight of 16-bit ones.
template <int DT>
__device__ __forceinline__ void pack16(const f32x2 (&y)[8], uint32_t (&w)[8]) {
  float v[16];
#pragma unroll
  for (int i = 0; i < 8; ++i) unpack2(y[i], v[2 * i], v[2 * i + 1]);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (DT == US_BF16) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    else if (DT == US_F16) w[i] = pack_f16x2(v[2 * i], v[2 * i + 1]);
    else if (i < 4) w[i] = cvt_fp8x4<DT == US_E5M2>(v[(4 * i) & 15], v[(4 * i + 1) & 15], v[(4 * i + 2) & 15], v[(4 * i + 3) & 15]);
  }
}
__device__ __forceinline__ void pack16(int dt, const f32x2 (&y)[8], uint32_t (&w)[8]) {
  if (dt == US_BF16) pack16<US_BF16>(y, w);
  else if (dt == US_F16) pack16<US_F16>(y, w);
  else if (dt == US_E4M3) pack16<US_E4M3>(y, w);
  else pack16<US_E5M2>(y, w);
}
// Calls g with the types of the copies and of the results (of operands of ES bytes) as constants.
template <int ES, class G>
__device__ __forceinline__ void with_formats(int kept, int out, G g) {
  auto with_out = [&](auto k) {
    constexpr int kOne = ES == 1 ? US_E5M2 : US_BF16, kOther = ES == 1 ? US_E4M3 : US_F16;
    if (out == kOne) g(k, std::integral_constant<int, kOne>()); else g(k, std::integral_constant<int, kOther>());
  };
  if (kept == US_E4M3) with_out(std::integral_constant<int, US_E4M3>());
  else if (kept == US_BF16) with_out(std::integral_constant<int, US_BF16>());
  else with_out(std::integral_constant<int, US_F16>());
}

__device__ __forceinline__ uint64_t chunk_desc(uint32_t addr, int row_bytes, uint32_t lbo) {      // N-major B, swizzled by its row width
  const uint64_t d = ptx::smem_desc_sw128(addr, lbo, 8u * row_bytes) & ~((uint64_t)7 << 61);
  return d | ((uint64_t)(row_bytes == 128 ? 2 : row_bytes == 64 ? 4 : 6) << 61);
}

// ES: operand bytes per element (1 = FP8, 2 = BF16 / F16).  HC: hidden columns of a tile.  CG = 2: tiles of 256 rows by a CTA pair, 1: of 128 by a CTA.  BOXED (forward):
// results leave by TMA, not by the lanes; the boxes take a stage or two.  That pays where the stores are not hidden behind the MMAs of a unit's next tile (boxed_pairs; single
// CTAs of 64 hidden columns, always).  (us, lanes / boxes.  One tile a unit: 1000 x 528 x 2096 F16 13.3 / 9.4; 700 x 2048 x 1500 FP8 20.4 / 9.5, BF16 26 / 13;
// 1000 x 1024 x 1024 FP8 5.8 / 6.2.)
template <bool BWD, int ES, int HC, int CG, bool BOXED>
__global__ void __launch_bounds__(gemm_threads(gated_ew(BWD, ES, CG)), 1)
gated_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b0, const __grid_constant__ CUtensorMap tm_b1,
             const __grid_constant__ CUtensorMap tm_h, const __grid_constant__ CUtensorMap tm_u, const __grid_constant__ CUtensorMap tm_dh,
             const __grid_constant__ CUtensorMap tm_du, const GatedParams p) {
  using S = GatedShape<BWD, ES, HC, CG, BOXED>;
  constexpr int kEW = S::kEW, kBK = kStageKBytes / ES, kTileM = kBM * CG, kN = S::kN;
  constexpr uint32_t kTmemCols = 2 * kN;
  const uint32_t a_bytes = CG == 2 ? (uint32_t)(kBM * kStageKBytes) : p.a_bytes, stage_bytes = a_bytes + S::kBBytes;
  const int stages = CG == 2 ? S::kStages : p.stages;

  ptx::grid_release_next();
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (ptx::smem_addr(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - ptx::smem_addr(smem_raw));
  const uint32_t bars = smem_base + kRoom;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kMostStages + s); };
  auto acc_full_bar = [&](int a) { return bars + 8u * (2 * kMostStages + a); };
  auto acc_empty_bar = [&](int a) { return bars + 8u * (2 * kMostStages + 2 + a); };
  const uint32_t drained_bar = bars + 8u * (2 * kMostStages + 4);
  auto in_bar = [&](int w, int s) { return bars + 8u * (2 * kMostStages + 5 + kMostSlots * w + s); };
  constexpr int kBars = 2 * kMostStages + 5 + kMostSlots * kEW;
  static_assert(8 * kBars + 8 <= S::kBarrierBytes, "barrier area too small");
  uint8_t* tail = smem_gen + kRoom + 8 * kBars;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail + 4);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CG == 2 ? (int)ptx::cluster_ctarank() : 0;
  const int unit = blockIdx.x / CG, num_units = gridDim.x / CG;
  const int num_tiles = p.tiles_m * p.tiles_n, num_kb = (p.K + kBK - 1) / kBK;
  // in bands of band_m tile rows, down a band first and then across: what runs together covers whole rows of the results
  auto tile_mn2 = [&](int tile, int& tm, int& tn) {
    const int band = p.d_band.div(tile), first = band * p.band_m, r = tile - first * p.tiles_n;
    const bool last = band >= p.full_bands;
    tn = last ? p.d_rows_last.div(r) : p.d_rows.div(r);
    tm = first + r - tn * (last ? p.tiles_m - first : p.band_m);
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) { ptx::mbar_init(full_bar(s), 1); ptx::mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { ptx::mbar_init(acc_full_bar(a), 1); ptx::mbar_init(acc_empty_bar(a), CG * kEW); }
    ptx::mbar_init(drained_bar, 1);
    if (BWD) for (int w = 0; w < kMostSlots * kEW; ++w) ptx::mbar_init(in_bar(0, w), 1);
    *abort_flag = 0;
    ptx::mbar_init_fence();
    ptx::prefetch_tensormap(&tm_a);
    ptx::prefetch_tensormap(&tm_b0);
    ptx::prefetch_tensormap(&tm_b1);
  }
  if (warp == 1) {
    if (CG == 2) { ptx::tmem_alloc_pair(ptx::smem_addr(const_cast<uint32_t*>(tmem_slot)), kTmemCols); ptx::tmem_relinquish_pair(); }
    else { ptx::tmem_alloc(ptx::smem_addr(const_cast<uint32_t*>(tmem_slot)), kTmemCols); ptx::tmem_relinquish(); }
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (CG == 2) ptx::cluster_meet();
  ptx::tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer (every CTA)
    if (ptx::elect_one()) {
      uint32_t issued = 0;
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      const int end = starved_cta(p.starved, rank) ? min(num_tiles, unit + p.served * num_units) : num_tiles;
      for (int tile = unit; ok && tile < end; tile += num_units) {
        int tm, tn;
        tile_mn2(tile, tm, tn);
        const int m0 = tm * kTileM + rank * kBM, n0 = tn * HC;
        for (int kb = 0; kb < num_kb; ++kb) {
          ok = wait_bounded(empty_bar(stage), phase ^ 1u, abort_flag, p.status, p.wait_limit);
          if (!ok) break;
          const uint32_t a_dst = smem_base + stage * stage_bytes, b_dst = a_dst + a_bytes;
          const int k0 = kb * kBK;
          if (issued == 0) ptx::grid_wait_previous();       // coordinates and barriers are ready: only the loads wait
          const uint32_t fb = CG == 2 ? ptx::in_even_cta(full_bar(stage)) : full_bar(stage);
          if (rank == 0) ptx::mbar_expect_tx(full_bar(stage), CG * stage_bytes);
          auto load = [&](uint32_t dst, const void* tmap, int x, int y) {
            if (CG == 2) ptx::tma_load_2d_pair(dst, tmap, fb, x, y); else ptx::tma_load_2d(dst, tmap, fb, x, y);
          };
          load(a_dst, &tm_a, k0, m0);                                            // X / G [M x K], K-major
          if (BWD) {
            load(b_dst, &tm_b0, k0, n0 + rank * S::kRowsB);                      // W2 [N x K], K-major
          } else if (CG == 2) {                                                  // Wg / Wu [K x N], N-major, 128 / ES columns per box
#pragma unroll
            for (int c = 0; c < ES; ++c) load(b_dst + c * S::kChunkBytes, rank == 0 ? &tm_b0 : &tm_b1, n0 + c * kBK, k0);
          } else {
            load(b_dst, &tm_b0, n0, k0);
            load(b_dst + S::kChunkBytes, &tm_b1, n0, k0);
          }
          ++issued;
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
      }
      if (*abort_flag && rank == 0) {
        // Let copies that are still in flight land before the CTA gives up its shared memory.
        const uint32_t n = issued < (uint32_t)stages ? issued : (uint32_t)stages;
        for (uint32_t i = 0; i < n; ++i) {
          if (stage == 0) { stage = stages; phase ^= 1u; }
          --stage;
          for (uint32_t it = 0; it < p.wait_limit && !ptx::mbar_try_wait(full_bar(stage), phase); ++it) {}
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (even CTA of a pair only)
    if (ptx::elect_one() && rank == 0) {
      ptx::grid_wait_previous();                       // no operand comes earlier: the bounded waits begin when the loads do
      int stage = 0; uint32_t phase = 0, local = 0;
      bool ok = true;
      const uint32_t stage_step = stage_bytes >> 4;
      const uint64_t a_desc = ptx::smem_desc_sw128(smem_base, 16, 1024);
      const uint64_t b_desc = BWD ? ptx::smem_desc_sw128(smem_base + a_bytes, 16, 1024) : chunk_desc(smem_base + a_bytes, S::kChunkRow, S::kChunkBytes);
      const uint32_t a_hi = (uint32_t)(a_desc >> 32), a_lo0 = (uint32_t)a_desc, b_hi = (uint32_t)(b_desc >> 32), b_lo0 = (uint32_t)b_desc;
      constexpr uint32_t b_step = (BWD ? 32u : (uint32_t)S::kChunkBytes / kKSteps) >> 4;
      for (int tile = unit; ok && tile < num_tiles; tile += num_units, ++local) {
        const uint32_t acc = local & 1u, acc_phase = (local >> 1) & 1u;
        ok = wait_bounded(acc_empty_bar(acc), acc_phase ^ 1u, abort_flag, p.status, p.wait_limit);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const uint32_t d_tmem = tmem_base + acc * kN;
        uint32_t accumulate = 0;
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!ptx::mbar_try_wait(full_bar(stage), phase)) {
            ok = wait_bounded(full_bar(stage), phase, abort_flag, p.status, p.wait_limit);
            if (!ok) break;
          }
          ptx::tc_fence_after_sync();
          const uint32_t a_lo = a_lo0 + stage * stage_step, b_lo = b_lo0 + stage * stage_step;
#pragma unroll
          for (int k = 0; k < kKSteps; ++k) {
            const uint64_t adesc = ((uint64_t)a_hi << 32) | (a_lo + k * 2u);
            const uint64_t bdesc = ((uint64_t)b_hi << 32) | (b_lo + k * b_step);
            if (CG == 2) ptx::mma_ss_pair<ES == 1>(d_tmem, adesc, bdesc, p.idesc, accumulate);
            else ptx::mma_ss<ES == 1>(d_tmem, adesc, bdesc, p.idesc, accumulate);
            accumulate = 1;
          }
          if (CG == 2) ptx::mma_commit_pair(empty_bar(stage), 3); else ptx::mma_commit(empty_bar(stage));
          if (++stage == stages) { stage = 0; phase ^= 1u; }
        }
        if (ok) { if (CG == 2) ptx::mma_commit_pair(acc_full_bar(acc), 3); else ptx::mma_commit(acc_full_bar(acc)); }
      }
      if (*abort_flag) {
        if (CG == 2) ptx::mma_commit_pair(drained_bar, 1); else ptx::mma_commit(drained_bar);
        for (uint32_t it = 0; it < p.wait_limit && !ptx::mbar_try_wait(drained_bar, 0); ++it) {}
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue warps
    ptx::grid_wait_previous();
    // Warp (lane quarter q, part) owns 32 rows x kWarpCols hidden columns of the tile; a lane holds one row of them.
    const int q = warp & 3, part = (warp - 2) >> 2;
    const int out_es = dtype_size(p.out_dt), kept_es = dtype_size(p.kept_dt);
    const f32x2 scale2 = splat2(p.scale), in2 = splat2(p.act_in), nl2 = splat2(-1.4426950408889634f * p.act_in), c0 = splat2(!BWD ? p.c0 : p.fn == US_FN_SILU ? p.c0 * p.scale * p.act_in : p.c0 * p.scale), c1 = splat2(p.c1 * p.scale);
    auto release_acc = [&](uint32_t a, int tile) {              // (where no later tile takes it nobody waits)
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0 && tile + 2 * num_units < num_tiles) {
        if (CG == 2) ptx::mbar_arrive_cluster(ptx::in_even_cta(acc_empty_bar(a)));
        else ptx::mbar_arrive(acc_empty_bar(a));
      }
    };
    auto place = [&](int tile, int& row, int& col) {            // of this lane's first element
      int tm, tn;
      tile_mn2(tile, tm, tn);
      row = tm * kTileM + rank * kBM + q * 32 + lane;
      col = tn * HC + part * S::kWarpCols;
    };
    uint32_t local = 0;
    bool ok = true;
    if constexpr (BOXED) {
      // A warp has 32 hidden columns of a tile; A and the copies leave through a box each.
      static_assert(S::kWarpCols == 32, "a box holds 32 columns");
      const uint32_t box_a = smem_base + (uint32_t)(kRoom - S::kEpiBytes + (warp - 2) * S::kEpiBytes / kEW), box_h = box_a + 1024u * out_es, box_u = box_h + 1024u * kept_es;
      const uint32_t out_sw = out_es == 2 ? (uint32_t)((lane >> 1) & 3) : 0u, kept_sw = kept_es == 2 ? (uint32_t)((lane >> 1) & 3) : 0u;
      for (int tile = unit; ok && tile < num_tiles; tile += num_units, ++local) {
        int row, col;
        place(tile, row, col);
        const uint32_t acc = local & 1u, acc_phase = (local >> 1) & 1u;
        ok = wait_bounded(acc_full_bar(acc), acc_phase, abort_flag, p.status, p.wait_limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        if (col >= p.N) {                                        // (the same for all lanes)
          release_acc(acc, tile);
          continue;
        }
        const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * kN + part * S::kWarpCols;
        if (ptx::elect_one()) ptx::bulk_wait_group_read<0>();    // the last tile's stores have read the boxes
        __syncwarp();
        unrolled<2>([&](auto half) {                             // sixteen columns
          constexpr int k = decltype(half)::value;
          uint32_t r0[16], r1[16], w[8];
          ptx::tmem_ld_32x32_issue(t_row + 16 * k, r0);
          ptx::tmem_ld_32x32_issue(t_row + HC + 16 * k, r1);
          ptx::tmem_ld_fence(r0);
          ptx::tmem_ld_fence(r1);
          if (k == 1) release_acc(acc, tile);                    // the values are in registers
          f32x2 h[8], u[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            h[i] = mul2(scale2, pack2(__uint_as_float(r0[2 * i]), __uint_as_float(r0[2 * i + 1])));
            u[i] = mul2(scale2, pack2(__uint_as_float(r1[2 * i]), __uint_as_float(r1[2 * i + 1])));
          }
          auto stage = [&](uint32_t box, int es, uint32_t sw) {  // a 16-byte chunk of 8-bit values, two of 16-bit ones
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              if (c == 1 && es == 1) break;
              ptx::sts128(box + (uint32_t)(lane * 32 * es) + (((uint32_t)(k * es + c) ^ sw) << 4), make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]));
            }
          };
          if (p.h) {
            pack16(p.kept_dt, h, w);
            stage(box_h, kept_es, kept_sw);
            pack16(p.kept_dt, u, w);
            stage(box_u, kept_es, kept_sw);
          }
          with_gate(p.fn, [&](auto fn) {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = mul2(mul2(gate_value2<decltype(fn)::value>(h[i], in2, nl2), c0), u[i]);
          });
          pack16(p.out_dt, h, w);
          stage(box_a, out_es, out_sw);
        });
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (ptx::elect_one()) {
          ptx::tma_store_2d(&tm_dh, box_a, col, row - lane);
          if (p.h) {
            ptx::tma_store_2d(&tm_h, box_h, col, row - lane);
            ptx::tma_store_2d(&tm_u, box_u, col, row - lane);
          }
          ptx::bulk_commit_group();
        }
      }
      if (ptx::elect_one()) ptx::bulk_wait_group_read<0>();
      __syncwarp();
    } else if constexpr (!BWD) {
      constexpr int kCols = S::kWarpCols;                        // of a warp: all at once in its registers
      static_assert(kCols <= 32, "a lane's columns of both projections would not fit its registers");
      for (int tile = unit; ok && tile < num_tiles; tile += num_units, ++local) {
        int row, col;
        place(tile, row, col);
        const uint32_t acc = local & 1u, acc_phase = (local >> 1) & 1u;
        ok = wait_bounded(acc_full_bar(acc), acc_phase, abort_flag, p.status, p.wait_limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * kN + part * S::kWarpCols;
        const int cols = row < p.M ? p.N - col : 0;
        uint32_t r0[kCols], r1[kCols];
        ptx::tmem_ld_32x32_issue(t_row, r0);
        ptx::tmem_ld_32x32_issue(t_row + HC, r1);
        ptx::tmem_ld_fence(r0);
        ptx::tmem_ld_fence(r1);
        release_acc(acc, tile);                                  // the values are in registers
        float a[kCols], b[kCols];
        uint32_t w[kCols / 2];
#pragma unroll
        for (int i = 0; i < kCols; i += 2) {
          unpack2(mul2(scale2, pack2(__uint_as_float(r0[i]), __uint_as_float(r0[i + 1]))), a[i], a[i + 1]);
          unpack2(mul2(scale2, pack2(__uint_as_float(r1[i]), __uint_as_float(r1[i + 1]))), b[i], b[i + 1]);
        }
        if (p.h) {
          pack_row<kCols>(p.kept_dt, a, w);
          put_row<kCols>(p.h + (row * p.h_ld + col) * kept_es, kept_es, w, cols, p.kept_sectors);
          pack_row<kCols>(p.kept_dt, b, w);
          put_row<kCols>(p.u + (row * p.u_ld + col) * kept_es, kept_es, w, cols, p.kept_sectors);
        }
        float y[kCols];
        with_gate(p.fn, [&](auto fn) {
#pragma unroll
          for (int i = 0; i < kCols; i += 2)
            unpack2(mul2(mul2(gate_value2<decltype(fn)::value>(pack2(a[i], a[i + 1]), in2, nl2), c0), pack2(b[i], b[i + 1])), y[i], y[i + 1]);
        });
        pack_row<kCols>(p.out_dt, y, w);
        put_row<kCols>(p.o0 + (row * p.o0_ld + col) * out_es, out_es, w, cols, p.out_sectors);
      }
    } else {
      // Units of 32 columns, whose copies arrive in a slot's boxes ahead of the accumulator.  A lane's row of a box is read and written by that lane, 16-byte chunk c at c ^ the
      // pattern of its row (64-byte rows swizzled, 32-byte ones not).
      const int ew = warp - 2;
      const bool in_place = kept_es == out_es;
      const uint32_t boxes = smem_base + (uint32_t)(kRoom - S::kEpiBytes + ew * epi_room(kEW)), in_row = 32u * kept_es, out_row = 32u * out_es;
      const uint32_t in_box = 32u * in_row, out_box = 32u * out_row, box_out = in_place ? 0u : 2u * in_box, slot_bytes = box_out + 2u * out_box;
      const uint32_t in_sw = in_row == 64 ? (uint32_t)((lane >> 1) & 3) : 0u, out_sw = out_row == 64 ? (uint32_t)((lane >> 1) & 3) : 0u;
      int pending = 0, fetch_slot = 0, slot = 0;                 // units whose copies have been asked for, the slot of the next one, and that of the unit that is worked on next
      uint32_t slot_phase = 0;
      int next_tile = unit, next_col = 0;                        // the unit whose copies are fetched next: columns from the warp's first on
      // In place: called once a unit has been stored, it fills the slot of the unit before, whose store is the last but one.
      auto fetch = [&]() {
        int row = 0, col = 0;
        for (; next_tile < num_tiles; next_tile += num_units, next_col = 0) {
          place(next_tile, row, col);
          if (next_col < S::kWarpCols && col + next_col < p.N) break;
        }
        if (next_tile >= num_tiles) return;
        if (ptx::elect_one()) {
          if (in_place) ptx::bulk_wait_group_read<1>();
          const uint32_t bar = in_bar(ew, fetch_slot), to = boxes + fetch_slot * slot_bytes;
          ptx::mbar_expect_tx(bar, 2 * in_box);
          ptx::tma_load_2d(to, &tm_h, bar, col + next_col, row - lane);
          ptx::tma_load_2d(to + in_box, &tm_u, bar, col + next_col, row - lane);
        }
        if (++fetch_slot == p.slots) fetch_slot = 0;
        ++pending;
        next_col += 32;
      };
      auto next_slot = [&]() {
        if (++slot == p.slots) { slot = 0; slot_phase ^= 1u; }
        --pending;
      };
      for (int k = in_place ? 1 : 0; k < p.slots; ++k) fetch();
      for (int tile = unit; ok && tile < num_tiles; tile += num_units, ++local) {
        int row, col0;
        place(tile, row, col0);
        const uint32_t acc = local & 1u, acc_phase = (local >> 1) & 1u;
        ok = wait_bounded(acc_full_bar(acc), acc_phase, abort_flag, p.status, p.wait_limit);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const uint32_t t_row = tmem_base + ((uint32_t)(q * 32) << 16) + acc * kN + part * S::kWarpCols;
        const int end = min(S::kWarpCols, p.N - col0);           // columns of this warp that exist
        if (end <= 0) release_acc(acc, tile);
#pragma unroll 1
        for (int at = 0; at < end; at += 32) {
          ok = wait_bounded(in_bar(ew, slot), slot_phase, abort_flag, p.status, p.wait_limit);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (!in_place) {                                       // the boxes that gradients leave from have been read by the stores before
            if (ptx::elect_one()) ptx::bulk_wait_group_read<0>();
            __syncwarp();
          }
          const uint32_t box = boxes + slot * slot_bytes, src = box + lane * in_row, dst = box + box_out + lane * out_row;
          with_formats<ES>(p.kept_dt, p.out_dt, [&](auto kept, auto out) {
            with_gate(p.fn, [&](auto fn) {
              constexpr int kWords = decltype(kept)::value == US_E4M3 ? 4 : 8;         // of sixteen kept values
              unrolled<2>([&](auto half) {                       // sixteen columns
                uint32_t r0[16], rh[kWords], ru[kWords], wh[8], wu[8];
                ptx::tmem_ld_32x32_issue(t_row + at + 16 * decltype(half)::value, r0);
#pragma unroll
                for (int k = 0; k < kWords / 4; ++k) {
                  const uint32_t chunk = ((decltype(half)::value * (kWords / 4) + k) ^ in_sw) << 4;
                  const uint4 vh = ptx::lds128(src + chunk), vu = ptx::lds128(src + in_box + chunk);
                  rh[4 * k] = vh.x; rh[4 * k + 1] = vh.y; rh[4 * k + 2] = vh.z; rh[4 * k + 3] = vh.w;
                  ru[4 * k] = vu.x; ru[4 * k + 1] = vu.y; ru[4 * k + 2] = vu.z; ru[4 * k + 3] = vu.w;
                }
                ptx::tmem_ld_fence(r0);
                if (decltype(half)::value == 1 && at + 32 >= end) release_acc(acc, tile);            // the values are in registers
                f32x2 yh[8], yu[8];
                from_here(r0);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  gate_grads2<decltype(fn)::value>(widen2<decltype(kept)::value>(rh, i), widen2<decltype(kept)::value>(ru, i),
                                                   pack2(__uint_as_float(r0[2 * i]), __uint_as_float(r0[2 * i + 1])), p.act_in, nl2, c0, c1, yh[i], yu[i]);
                pack16<decltype(out)::value>(yh, wh);
                pack16<decltype(out)::value>(yu, wu);
#pragma unroll
                for (int k = 0; k < ES; ++k) {          // one chunk of 8-bit results, two of 16-bit ones
                  const uint32_t chunk = ((decltype(half)::value * ES + k) ^ out_sw) << 4;
                  ptx::sts128(dst + chunk, make_uint4(wh[4 * k], wh[4 * k + 1], wh[4 * k + 2], wh[4 * k + 3]));
                  ptx::sts128(dst + out_box + chunk, make_uint4(wu[4 * k], wu[4 * k + 1], wu[4 * k + 2], wu[4 * k + 3]));
                }
              });
            });
          });
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (ptx::elect_one()) {
            ptx::tma_store_2d(&tm_dh, box + box_out, col0 + at, row - lane);
            ptx::tma_store_2d(&tm_du, box + box_out + out_box, col0 + at, row - lane);
            ptx::bulk_commit_group();
          }
          next_slot();
          fetch();
        }
      }
      // Copies that are still in flight after a wait that ran out land, and stores have read their boxes, before the CTA gives up its shared memory.
      for (; pending > 0; next_slot())
        for (uint32_t it = 0; it < p.wait_limit && !ptx::mbar_try_wait(in_bar(ew, slot), slot_phase); ++it) {}
      if (ptx::elect_one()) ptx::bulk_wait_group_read<0>();
      __syncwarp();
    }
    // Leaving (early too, when a wait ran out somewhere in the CTA): tensor-memory loads have landed.
    ptx::tmem_ld_wait_all();
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  if (CG == 2) ptx::cluster_part(*abort_flag != 0);
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    if (CG == 2) ptx::tmem_dealloc_pair(tmem_base, kTmemCols); else ptx::tmem_dealloc(tmem_base, kTmemCols);
  }
}

// ---------------------------------------------------------------- host
bool valid_mat(const us_mat* m) {
  return m && m->ptr && m->rows >= 1 && m->cols >= 1 && m->ld >= m->cols && m->rows < (1ll << 31) && m->cols < (1ll << 31) && m->dtype >= US_F32 && m->dtype <= US_E5M2;
}
bool given(const us_mat* m) { return m && m->ptr; }
bool aligned(const us_mat* m, int bytes) { return reinterpret_cast<uintptr_t>(m->ptr) % bytes == 0 && (m->ld * dtype_size(m->dtype)) % bytes == 0; }
bool is_fp8(int dt) { return dt == US_E4M3 || dt == US_E5M2; }

// host::make_tmap for boxes of 32 bytes a row that are multiplied as they are: swizzled with that width's pattern.
bool make_chunk_tmap(CUtensorMap* tm, const us_mat* m, int es, int box_rows, int box_bytes) {
  if (box_bytes != 32) return host::make_tmap(tm, m, es, box_rows, box_bytes);
  host::EncodeTiledFn fn = host::encode_tiled_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)m->cols, (cuuint64_t)m->rows}, strides[1] = {(cuuint64_t)m->ld * es};
  cuuint32_t box[2] = {(cuuint32_t)(box_bytes / es), (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return fn(tm, es == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, m->ptr, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct GatedMats { const us_mat *a, *b0, *b1, *h, *u, *dh, *du; };       // forward: dh is A, du not used

template <bool BWD, int ES, int HC, int CG, bool BOXED = false>
us_status launch_gated(const GatedMats& m, GatedParams& p, int sms, cudaStream_t st) {
  const us_mat *A = m.a, *B0 = m.b0, *B1 = m.b1;
  using S = GatedShape<BWD, ES, HC, CG, BOXED>;
  if (CG == 2 && p.starved == 2) return US_ERR_INVALID_ARG;        // test hook: of a pair only the odd CTA may starve alone (nobody would wait for its copies)
  p.tiles_m = (p.M + kBM * CG - 1) / (kBM * CG);
  p.tiles_n = (p.N + HC - 1) / HC;
  if ((int64_t)p.tiles_m * p.tiles_n >= (1ll << 30)) return US_ERR_UNSUPPORTED;
  // Whole rows of the results one after another while the weights stay in L2, else bands of 1024 tokens or so, which read them once each (us, bands of 1 / 4 / 8
  // tile rows / all: forward FP8 16384 x 2048 x 8192 443 / 449 / 463 / 471, BF16 8192 x 1024 x 4096 126 / 127 / 128 / 130, its backward pass 90 / 91 / 92 / 96).
  const bool resident = (int64_t)p.K * p.N * ES * (BWD ? 1 : 2) <= (64ll << 20);
  p.band_m = std::min(p.tiles_m, resident ? 1 : 8 / CG);
  p.full_bands = p.tiles_m / p.band_m;
  p.d_band = make_fast_div(p.band_m * p.tiles_n);
  p.d_rows = make_fast_div(p.band_m);
  p.d_rows_last = make_fast_div(p.tiles_m % p.band_m ? p.tiles_m % p.band_m : 1);
  const int one = ES == 1 ? US_E5M2 : US_BF16;
  p.idesc = make_idesc(A->dtype == one, B0->dtype == one, false, !BWD, kBM * CG, S::kN);
  // a short A: its rows in groups of eight.  The MMA still reads 128; what lies behind them ends up in rows that do not exist.
  const int a_rows = CG == 1 && p.M < kBM ? (p.M + 7) / 8 * 8 : kBM;
  p.a_bytes = (uint32_t)a_rows * kStageKBytes;
  p.stages = std::min(kMostStages, (kRoom - std::max((int)S::kEpiBytes, kBM * kStageKBytes)) / ((int)p.a_bytes + S::kBBytes));
  CUtensorMap t[7];
  constexpr int kBK = kStageKBytes / ES;
  if (!host::make_tmap(&t[0], A, ES, a_rows, kStageKBytes)) return US_ERR_CUDA;
  if (!(BWD ? host::make_tmap(&t[1], B0, ES, S::kRowsB, kStageKBytes) : make_chunk_tmap(&t[1], B0, ES, kBK, S::kChunkRow))) return US_ERR_CUDA;
  if (BWD) t[2] = t[1];
  else if (!make_chunk_tmap(&t[2], B1, ES, kBK, S::kChunkRow)) return US_ERR_CUDA;
  if (BWD) {
    const int kept_es = dtype_size(m.h->dtype), out_es = dtype_size(m.dh->dtype);
    p.slots = kept_es == out_es ? kMostSlots : epi_room(S::kEW) / (2048 * (kept_es + out_es));
    if (!host::make_tmap(&t[3], m.h, kept_es, 32, 32 * kept_es) || !host::make_tmap(&t[4], m.u, kept_es, 32, 32 * kept_es) ||
        !host::make_tmap(&t[5], m.dh, out_es, 32, 32 * out_es) || !host::make_tmap(&t[6], m.du, out_es, 32, 32 * out_es))
      return US_ERR_CUDA;
  } else {
    t[3] = t[4] = t[5] = t[6] = t[0];
    const int kept_es = dtype_size(p.kept_dt), out_es = dtype_size(p.out_dt);
    if (BOXED && (!host::make_tmap(&t[5], m.dh, out_es, 32, 32 * out_es) || (p.h && (!host::make_tmap(&t[3], m.h, kept_es, 32, 32 * kept_es) ||
                                                                                      !host::make_tmap(&t[4], m.u, kept_es, 32, 32 * kept_es)))))
      return US_ERR_CUDA;
  }
  const int tiles = p.tiles_m * p.tiles_n, most = sms / CG;
  static std::atomic<uint64_t> smem_set{0};
  return host::launch(gated_kernel<BWD, ES, HC, CG, BOXED>, &smem_set, CG * (tiles < most ? tiles : most), gemm_threads(S::kEW), S::kTotal, CG, st, t[0], t[1], t[2], t[3],
                      t[4], t[5], t[6], static_cast<const GatedParams&>(p));
}

// Boxes for CTA pairs: no unit has a second tile, or the contraction is too short (nine stages) to hide the stores.  (us, lanes / boxes, copies of h and u in BF16:
// 2048 x 528 x 2096 BF16 17.5 / 12.7, FP8 16.4 / 11.1; 8192 x 1024 x 4096 FP8 82 / 72, BF16 121 / 126; 4096 x K x 4096 BF16, K = 576: 55 / 48, 640: 47.6 / 46.7,
// 768: 51.8 / 53.5; FP8, K = 1152: 50 / 45, 1536: 49.8 / 52.5; 16384 x 2048 x 8192 FP8 with copies in E4M3 443 / 474.)
inline bool boxed_pairs(int64_t tiles, int64_t k_bytes, int sms) { return 2 * tiles <= sms || k_bytes <= 9 * kStageKBytes; }

// Tiles of CTA pairs unless they would leave more than half of the pairs idle, else the widest of single CTAs, else, where the machine has
// an SM for each of them, the narrow ones.
template <bool BWD, int ES>
us_status pick_gated(const GatedMats& m, GatedParams& p, cudaStream_t st) {
  const int sms = host::sm_count();
  if (sms <= 0) return US_ERR_CUDA;
  constexpr int kWide = BWD ? 256 : 128;
  const int64_t M = p.M, N = p.N;
  if (4 * ((M + 255) / 256) * ((N + kWide - 1) / kWide) >= sms && M > kBM) {
    if constexpr (!BWD) {
      if (boxed_pairs(((M + 255) / 256) * ((N + kWide - 1) / kWide), (int64_t)p.K * ES, sms)) return launch_gated<BWD, ES, kWide, 2, true>(m, p, sms, st);
    }
    return launch_gated<BWD, ES, kWide, 2>(m, p, sms, st);
  }
  const int64_t narrow = ((M + kBM - 1) / kBM) * ((N + kWide / 4 - 1) / (kWide / 4));
  if (narrow <= sms) return launch_gated<BWD, ES, kWide / 4, 1>(m, p, sms, st);
  return launch_gated<BWD, ES, kWide / 2, 1, !BWD>(m, p, sms, st);
}

// The checks that both directions share: operands of one width (f8: 8-bit), workspace.
constexpr int64_t kMostSize = 0x7fffff00;        // rows, columns and contraction: the coordinates of a tile that ends behind them are 32-bit numbers
us_status check_common(const us_mat* const* in, int n, const us_mat* const* out, int outs, const us_mat* H, const us_mat* U, const void* ws, size_t ws_bytes, bool& f8) {
  if (!ws || ws_bytes < us_workspace_bytes()) return US_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) % 16) return US_ERR_ALIGNMENT;
  for (int i = 0; i < n; ++i) if (!aligned(in[i], 16)) return US_ERR_ALIGNMENT;
  for (int i = 0; i < outs; ++i) if (!aligned(out[i], 16)) return US_ERR_ALIGNMENT;
  if (given(H) && (!aligned(H, 16) || !aligned(U, 16))) return US_ERR_ALIGNMENT;
  for (int i = 0; i < n; ++i) if (in[i]->rows > kMostSize || in[i]->cols > kMostSize) return US_ERR_UNSUPPORTED;
  f8 = is_fp8(in[0]->dtype);
  const bool h16 = in[0]->dtype == US_BF16 || in[0]->dtype == US_F16;
  if (!f8 && !h16) return US_ERR_UNSUPPORTED;
  for (int i = 1; i < n; ++i) if (f8 ? !is_fp8(in[i]->dtype) : in[i]->dtype != in[0]->dtype) return US_ERR_UNSUPPORTED;
  for (int i = 0; i < outs; ++i) if (f8 ? !is_fp8(out[i]->dtype) : out[i]->dtype != in[0]->dtype) return US_ERR_UNSUPPORTED;
  if (given(H) && H->dtype != US_BF16 && H->dtype != US_F16 && H->dtype != US_E4M3) return US_ERR_UNSUPPORTED;
  return US_OK;
}

us_status gated_fwd(int fn, const us_mat* X, const us_mat* Wg, const us_mat* Wu, float alpha, float act_in, float act_out, const us_mat* H, const us_mat* U,
                    const us_mat* A, void* ws, size_t ws_bytes, void* stream, uint32_t wait_limit, int starved, int served) {
  if (fn < US_FN_GELU || fn > US_FN_SILU || !valid_mat(X) || !valid_mat(Wg) || !valid_mat(Wu) || !valid_mat(A)) return US_ERR_INVALID_ARG;
  const int64_t M = X->rows, K = X->cols, N = Wg->cols;
  if (Wg->rows != K || Wu->rows != K || Wu->cols != N || Wu->dtype != Wg->dtype || A->rows != M || A->cols != N) return US_ERR_INVALID_ARG;
  if (given(H) != given(U)) return US_ERR_INVALID_ARG;
  if (given(H) && (!valid_mat(H) || !valid_mat(U) || H->rows != M || H->cols != N || U->rows != M || U->cols != N || U->dtype != H->dtype)) return US_ERR_INVALID_ARG;
  const us_mat *in[3] = {X, Wg, Wu}, *out[1] = {A};
  bool f8;
  const us_status s = check_common(in, 3, out, 1, H, U, ws, ws_bytes, f8);
  if (s != US_OK) return s;
  GatedParams p{};
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.scale = alpha; p.act_in = act_in; p.c0 = act_out; p.fn = fn;
  p.kept_dt = US_BF16;
  if (given(H)) {
    p.h = static_cast<uint8_t*>(H->ptr); p.h_ld = H->ld; p.u = static_cast<uint8_t*>(U->ptr); p.u_ld = U->ld;
    p.kept_dt = H->dtype; p.kept_sectors = aligned(H, 32) && aligned(U, 32);
  }
  p.o0 = static_cast<uint8_t*>(A->ptr); p.o0_ld = A->ld; p.out_dt = A->dtype; p.out_sectors = aligned(A, 32);
  p.status = static_cast<unsigned int*>(ws); p.wait_limit = wait_limit; p.starved = starved; p.served = served;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const GatedMats m{X, Wg, Wu, H, U, A, nullptr};
  return f8 ? pick_gated<false, 1>(m, p, st) : pick_gated<false, 2>(m, p, st);
}

us_status gated_bwd(int fn, const us_mat* G, const us_mat* W2, float beta_x, float act_in, float beta_h, float beta_u, const us_mat* H, const us_mat* U,
                    const us_mat* dH, const us_mat* dU, void* ws, size_t ws_bytes, void* stream, uint32_t wait_limit, int starved, int served) {
  if (fn < US_FN_GELU || fn > US_FN_SILU || !valid_mat(G) || !valid_mat(W2) || !valid_mat(H) || !valid_mat(U) || !valid_mat(dH) || !valid_mat(dU)) return US_ERR_INVALID_ARG;
  const int64_t M = G->rows, K = G->cols, N = W2->rows;
  if (W2->cols != K) return US_ERR_INVALID_ARG;
  const us_mat* same[4] = {H, U, dH, dU};
  for (const us_mat* m : same) if (m->rows != M || m->cols != N) return US_ERR_INVALID_ARG;
  if (U->dtype != H->dtype || dU->dtype != dH->dtype) return US_ERR_INVALID_ARG;
  const us_mat *in[2] = {G, W2}, *out[2] = {dH, dU};
  bool f8;
  const us_status s = check_common(in, 2, out, 2, H, U, ws, ws_bytes, f8);
  if (s != US_OK) return s;
  GatedParams p{};
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  p.scale = beta_x; p.act_in = act_in; p.c0 = beta_u; p.c1 = beta_h * act_in; p.fn = fn;
  p.kept_dt = H->dtype; p.out_dt = dH->dtype;
  p.status = static_cast<unsigned int*>(ws); p.wait_limit = wait_limit; p.starved = starved; p.served = served;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const GatedMats m{G, W2, W2, H, U, dH, dU};
  return f8 ? pick_gated<true, 1>(m, p, st) : pick_gated<true, 2>(m, p, st);
}

bool bad_hook(uint32_t wait_limit, int cta, int tiles) { return wait_limit == 0 || wait_limit > (1u << 16) || cta < -1 || cta > 1 || tiles < 0 || tiles > 1024; }

}  // namespace
}  // namespace us

extern "C" us_status us_ffn_gated_fwd(us_fn fn, const us_mat* X, const us_mat* Wg, const us_mat* Wu, float alpha, float act_in_scale, float act_out_scale,
                                      const us_mat* H, const us_mat* U, const us_mat* A, void* ws, size_t ws_bytes, void* stream) {
  return us::gated_fwd(fn, X, Wg, Wu, alpha, act_in_scale, act_out_scale, H, U, A, ws, ws_bytes, stream, us::kWaitLimit, 0, 0);
}
extern "C" us_status us_ffn_gated_bwd(us_fn fn, const us_mat* G, const us_mat* W2, float beta_x, float act_in_scale, float beta_h, float beta_u, const us_mat* H,
                                      const us_mat* U, const us_mat* dH, const us_mat* dU, void* ws, size_t ws_bytes, void* stream) {
  return us::gated_bwd(fn, G, W2, beta_x, act_in_scale, beta_h, beta_u, H, U, dH, dU, ws, ws_bytes, stream, us::kWaitLimit, 0, 0);
}
extern "C" us_status us_test_ffn_gated_fwd_starved(const us_mat* X, const us_mat* Wg, const us_mat* Wu, const us_mat* H, const us_mat* U, const us_mat* A, void* ws,
                                                   size_t ws_bytes, uint32_t wait_limit, int cta, int tiles, void* stream) {
  if (us::bad_hook(wait_limit, cta, tiles)) return US_ERR_INVALID_ARG;
  return us::gated_fwd(US_FN_SILU, X, Wg, Wu, 1.f, 1.f, 1.f, H, U, A, ws, ws_bytes, stream, wait_limit, cta + 2, tiles);
}
extern "C" us_status us_test_ffn_gated_bwd_starved(const us_mat* G, const us_mat* W2, const us_mat* H, const us_mat* U, const us_mat* dH, const us_mat* dU, void* ws,
                                                   size_t ws_bytes, uint32_t wait_limit, int cta, int tiles, void* stream) {
  if (us::bad_hook(wait_limit, cta, tiles)) return US_ERR_INVALID_ARG;
  return us::gated_bwd(US_FN_SILU, G, W2, 1.f, 1.f, 1.f, 1.f, H, U, dH, dU, ws, ws_bytes, stream, wait_limit, cta + 2, tiles);
}
