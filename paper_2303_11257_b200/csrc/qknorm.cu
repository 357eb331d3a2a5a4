// us_qk_norm_fwd / us_qk_norm_bwd: root-mean-square norms of queries and keys, head by head, with the rotation of their positions in the
// same pass, forward and backward; us_rotary_table: the angles' cosines and sines.
//
//   forward    r = 1 / sqrt(mean x^2 + eps),  n = w x r,  y = R n          R: each pair (a, b) of the rotated features -> (a c - b s, b c + a s)
//   backward   n' = R^T g,  u = w n',  dx = beta_x r (u - x r mean(u x r)),  dw = beta_w sum n' x r
//
// Every element is read once and written once.  The kernels are bound by the latency of what they issue (11 to 14 instructions a value) before they are by HBM: 59 % of the issue slots are used, with 16 warps
// an SM that wait for results of fixed latency, then for shared memory and shuffles, hardly for global memory.  8192 tokens of 16 + 16 heads of 64
// in BF16: forward 13.5 us (5.0 TB/s), backward 22.0 (4.6 TB/s), in float32 34.4 and 54.6 (3.9 and 3.7 TB/s); 16384 tokens of 32 + 8 heads of 128 into E4M3 58 us (4.5 TB/s).
// A head is held by a group of G lanes (a power of two), each with two chunks of eight features that hold whole pairs -- features i .. i + 7 and their partners half a
// rotation further, or sixteen neighbours -- so that the rotation needs no exchange and one group sum (forward) or two (backward) are all that lanes tell one another.  A warp's
// unit is some steps of 32 / G heads of one row, whose cosines and sines it holds in registers over all of them; the norm's weight it holds for the whole launch,
// since a CTA works for one part (queries or keys) only.  Weight gradients are summed in the registers of the lane that has the feature, then over groups, warps and, in a second
// launch, CTAs, in a fixed order without atomics.
// Rows that are not on 16-byte boundaries, widths that are no multiple of eight, matrices of several types and turns of a number of features that is no multiple of 16 (neighbours: 8) take the general kernels: a warp a head,
// through shared memory, one value a lane at a time (8192 tokens of 16 + 16 heads of 72 in BF16, all turned: forward 294 us, backward 430; with neighbouring pairs, which the vector kernels take, 26 and 43).
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "host.h"
#include "rowwise.cuh"
#include "sm100.cuh"

namespace us {
namespace {

constexpr int kMostParts = 4, kMostWidth = 1024, kMostVecWidth = 512;
constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBwdCtasPerSm = 2, kFwdCtasPerSm = 2;

struct QkPart {
  const void *x, *g, *w;
  void* y;                     // forward: output; backward: dX
  void* dw;
  int64_t x_ld, g_ld, y_ld;
  int x_dt, g_dt, w_dt, y_dt, dw_dt;
  int heads, blocks;           // heads, and warp units per row
  uint32_t step_rows, step_blocks, step_position;      // of the units of a warp: rows, blocks beyond them, rows modulo the period
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

__device__ __forceinline__ int64_t position_of(const QkArgs& p, int64_t row) {
  return p.positions ? (int64_t)__ldg(p.positions + row) : p.start + (p.period ? (int64_t)((uint32_t)row % p.period) : row);
}
// The table row of a position, nullptr where it is not in the table.
__device__ __forceinline__ const float* angles_at(const QkArgs& p, int64_t at) {
  return at >= 0 && at < p.table_rows ? p.table + at * p.table_ld : nullptr;
}

__device__ __forceinline__ float group_sum(float v, int group) {
  for (int o = group >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sixteen bytes to this lane's place in shared memory, asynchronously; waiting until at most N groups of them are under way.
__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A chunk of eight features in shared memory, 512 bytes of a warp (float32: twice that) in pieces of sixteen bytes a lane.  Widened to pairs of neighbours, for arithmetic
// on two values at a time.
template <int DT>
constexpr int kChunkBytes = DT == US_F32 ? 1024 : 512;
template <int DT>
__device__ __forceinline__ void fetch(uint32_t to, const char* from) {
  copy16(to, from);
  if (DT == US_F32) copy16(to + 512u, from + 16);
}
template <int DT>
__device__ __forceinline__ void widen(uint32_t from, f32x2 (&v)[4]) {
  const uint4 r = ptx::lds128(from);
  if constexpr (DT == US_F32) {
    const uint4 s = ptx::lds128(from + 512u);
    v[0] = pack2(__uint_as_float(r.x), __uint_as_float(r.y)); v[1] = pack2(__uint_as_float(r.z), __uint_as_float(r.w));
    v[2] = pack2(__uint_as_float(s.x), __uint_as_float(s.y)); v[3] = pack2(__uint_as_float(s.z), __uint_as_float(s.w));
  } else {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = DT == US_BF16 ? unpack_bf16x2(w[i]) : unpack_f16x2(w[i]);
      v[i] = pack2(f.x, f.y);
    }
  }
}
__device__ __forceinline__ float halves_sum(f32x2 v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}
// Eight features rounded to type DT, to an address with the chunk's alignment.
template <int DT>
__device__ __forceinline__ void put(char* to, const f32x2 (&y)[4]) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack2(y[i], v[2 * i], v[2 * i + 1]);
  if (DT == US_F32) {
    reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else if (DT == US_BF16) {
    *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
  } else if (DT == US_F16) {
    *reinterpret_cast<uint4*>(to) = make_uint4(pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]), pack_f16x2(v[4], v[5]), pack_f16x2(v[6], v[7]));
  } else {
    *reinterpret_cast<uint2*>(to) = make_uint2(cvt_fp8x4<DT == US_E5M2>(v[0], v[1], v[2], v[3]), cvt_fp8x4<DT == US_E5M2>(v[4], v[5], v[6], v[7]));
  }
}
// Calls g with the type of a part's results as a constant.
template <class G>
__device__ __forceinline__ void with_output(int dt, G g) {
  switch (dt) {
    case US_F32: g(std::integral_constant<int, US_F32>()); break;
    case US_BF16: g(std::integral_constant<int, US_BF16>()); break;
    case US_F16: g(std::integral_constant<int, US_F16>()); break;
    case US_E4M3: g(std::integral_constant<int, US_E4M3>()); break;
    default: g(std::integral_constant<int, US_E5M2>()); break;
  }
}
// 1 / sqrt(x), within 2 steps; of nothing infinite.
__device__ __forceinline__ float rsqrt_approx(float x) {
  float r;
  asm("rsqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Which features a lane has, and which of them are rotated.
struct Lane {
  int a, b;                    // first feature of each chunk
  bool has_a, has_b, rot_a, rot_b;
};
// FULL: every lane of a group has two chunks and every feature is rotated (widths of 16 to 512 that are a power of two), known when compiled: tests of a lane's share
// become selections between registers in the arithmetic, twice as many instructions in all.
template <bool NEIGHBOURS, bool FULL>
__device__ __forceinline__ Lane lane_of(const QkArgs& p, int j) {
  Lane l;
  if (FULL) {
    l.a = NEIGHBOURS ? 16 * j : 8 * j;
    l.b = NEIGHBOURS ? l.a + 8 : l.a + p.width / 2;
    l.has_a = l.has_b = l.rot_a = l.rot_b = true;
    return l;
  }
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
// Cosines and sines of a lane's pairs, eight from pair 8 j on, as a turn needs them.  Chunk a of a half turn: cos[0 .. 3] its cosines, two each, sin and minus the sines and their negatives.
// Neighbours: for pair i of chunk a (b: i + 4) cos[i] = (c, c), sin[i] = (-s, s).
template <bool NEIGHBOURS>
struct Turn { f32x2 cos[NEIGHBOURS ? 8 : 4], sin[NEIGHBOURS ? 8 : 4], minus[NEIGHBOURS ? 1 : 4]; };
// from: this lane's 64 bytes of the table's row
template <bool NEIGHBOURS, bool BACK>
__device__ __forceinline__ void read_turn(uint32_t from, const Lane& l, Turn<NEIGHBOURS>& t) {
  if (!(l.rot_a || l.rot_b)) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {                                // two pairs
    const uint4 r = ptx::lds128(from + 16u * i);
    float4 v = make_float4(__uint_as_float(r.x), __uint_as_float(r.y), __uint_as_float(r.z), __uint_as_float(r.w));
    if (BACK) { v.y = -v.y; v.w = -v.w; }
    if constexpr (NEIGHBOURS) {
      t.cos[2 * i] = pack2(v.x, v.x); t.cos[2 * i + 1] = pack2(v.z, v.z);
      t.sin[2 * i] = pack2(-v.y, v.y); t.sin[2 * i + 1] = pack2(-v.w, v.w);
    } else {
      t.cos[i] = pack2(v.x, v.z); t.sin[i] = pack2(v.y, v.w); t.minus[i] = pack2(-v.y, -v.w);
    }
  }
}
__device__ __forceinline__ f32x2 swapped(f32x2 v) {
  float a, b;
  unpack2(v, a, b);
  return pack2(b, a);
}
template <bool NEIGHBOURS>
__device__ __forceinline__ void rotate(f32x2 (&a)[4], f32x2 (&b)[4], const Turn<NEIGHBOURS>& t, const Lane& l) {
  if constexpr (NEIGHBOURS) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (l.rot_a) a[i] = fma2(swapped(a[i]), t.sin[i], mul2(a[i], t.cos[i]));
      if (l.rot_b) b[i] = fma2(swapped(b[i]), t.sin[4 + i], mul2(b[i], t.cos[4 + i]));
    }
  } else if (l.rot_a) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 ya = fma2(b[i], t.minus[i], mul2(a[i], t.cos[i]));
      b[i] = fma2(a[i], t.sin[i], mul2(b[i], t.cos[i]));
      a[i] = ya;
    }
  }
}

__device__ __forceinline__ int part_of(const QkArgs& p, int cta) {
  int k = 0;
  while (k + 1 < p.count && cta >= p.part[k + 1].first_cta) ++k;
  return k;
}
__device__ __forceinline__ void load_weight(const QkPart& q, const Lane& l, f32x2 (&wa)[4], f32x2 (&wb)[4]) {
  auto at = [&](bool has, int i) { return has ? (q.w ? load_one(q.w, q.w_dt, i) : 1.f) : 0.f; };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    wa[i] = pack2(at(l.has_a, l.a + 2 * i), at(l.has_a, l.a + 2 * i + 1));
    wb[i] = pack2(at(l.has_b, l.b + 2 * i), at(l.has_b, l.b + 2 * i + 1));
  }
}

// The vector kernels' walk over the units of a warp: STEPS steps of 32 / G heads of one row, which arrive in a ring of kStages slots of the warp's own in shared memory, ahead of the
// one that is worked on.  (us, 8192 tokens of 16 + 16 heads of 64 forward and backward, 16384 of 32 + 8 heads of 128 into E4M3; rings of two / three slots: 13.5 / 13.7, 22.0 / 23.0, 57.6 / 58.2;
// units of one step 14.4, 22.7, 69; of four 72 for the last.)
constexpr int kStages = 2;
// Bytes of a slot: both chunks of a step, of x and backward of the gradient, and the row of the table.
template <bool BWD, int DT, int STEPS>
__host__ __device__ constexpr int slot_bytes(int group) { return STEPS * (BWD ? 4 : 2) * kChunkBytes<DT> + 64 * group; }

// A unit of a warp, and its position where all rows' follow from their number.  Advanced by additions: 64-bit products and divisions for each unit were most of what
// the kernels issued (21 to 26 instructions a value).
struct Unit { uint32_t row, block, position; };
__device__ __forceinline__ Unit first_unit(const QkArgs& p, const QkPart& q, uint32_t number) {
  const uint32_t row = number / (uint32_t)q.blocks;
  return Unit{row, number - row * q.blocks, p.period ? row % p.period : row};
}
__device__ __forceinline__ bool advance(const QkArgs& p, const QkPart& q, Unit& u) {            // whether the blocks of a row were through
  const uint32_t carry = u.block + q.step_blocks >= (uint32_t)q.blocks;
  u.block += q.step_blocks - (carry ? q.blocks : 0);
  u.row += q.step_rows + carry;
  u.position += q.step_position + carry;
  if (p.period && u.position >= p.period) u.position -= p.period;
  return carry;
}
// (what is not in the table, negative ones too, is not below its number of rows, which are fewer than 2^31 here)
__device__ __forceinline__ uint32_t position_of(const QkArgs& p, const Unit& u) { return p.positions ? (uint32_t)__ldg(p.positions + u.row) : (uint32_t)p.start + u.position; }
// A lane's place in a matrix.  STEPPED: it goes from unit to unit by additions (forward; backward, where registers are short, by a product).
template <bool STEPPED>
struct Place {
  char* base;
  int64_t row_bytes, carried;                                   // STEPPED: bytes from unit to unit, and what is added where the blocks of a row are through
  int block_bytes;
  __device__ __forceinline__ Place(const void* to, const Unit& u, const QkPart& q, int64_t pitch, int block) : base(static_cast<char*>(const_cast<void*>(to))), row_bytes(pitch), block_bytes(block) {
    if (STEPPED) {
      base += u.row * pitch + (int64_t)u.block * block;
      row_bytes = q.step_rows * pitch + (int64_t)q.step_blocks * block;
      carried = pitch - (int64_t)q.blocks * block;
    }
  }
  __device__ __forceinline__ char* at(const Unit& u) const { return STEPPED ? base : base + u.row * row_bytes + (int64_t)u.block * block_bytes; }
  __device__ __forceinline__ void advance(bool carry) { if (STEPPED) { base += row_bytes; if (carry) base += carried; } }
};

template <bool BWD, int DT, int STEPS, class B, class G>
__device__ __forceinline__ void walk(const QkArgs& p, const QkPart& q, const Lane& l, uint32_t ring, int zero, B begin, G work) {
  constexpr int kC = kChunkBytes<DT>, kStep = (BWD ? 4 : 2) * kC, kEs = DT == US_F32 ? 4 : 2;
  const int lane = threadIdx.x & 31, j = lane & (p.group - 1), per = 32 / p.group, slot = slot_bytes<BWD, DT, STEPS>(p.group);
  const uint32_t rows = (uint32_t)p.rows;
  const int step_bytes = per * p.width * kEs, b_minus_a = (l.b - l.a) * kEs;
  const int first = lane / p.group * p.width + l.a;             // this lane's first feature among those of a step
  const bool turns = p.table != nullptr;
  const float* table = p.table + 16 * j;
  Unit now = first_unit(p, q, (blockIdx.x - q.first_cta) * kWarps + (threadIdx.x >> 5) + zero), next = now;
  Place<!BWD> x(static_cast<const char*>(q.x) + first * kEs, next, q, q.x_ld * kEs, step_bytes * STEPS), g(BWD ? static_cast<const char*>(q.g) + first * kEs : nullptr, next, q, q.g_ld * kEs, step_bytes * STEPS);
  // positions are read one unit before the copy of their angles is issued; one that is not in the table has NaN for angles
  uint32_t position = turns && next.row < rows ? position_of(p, next) : 0;
  auto issue = [&](int s) {
    if (next.row < rows) {
      const uint32_t to = ring + s * slot + lane * 16u;
      const char *px = x.at(next), *pg = BWD ? g.at(next) : nullptr;
      const int heads = q.heads - (int)next.block * (per * STEPS) - lane / p.group;        // left from this lane's first on
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        if (k * per >= heads) break;
        if (l.has_a) { fetch<DT>(to + k * kStep, px + k * step_bytes); if (BWD) fetch<DT>(to + k * kStep + 2 * kC, pg + k * step_bytes); }
        if (l.has_b) { fetch<DT>(to + k * kStep + kC, px + k * step_bytes + b_minus_a); if (BWD) fetch<DT>(to + k * kStep + 3 * kC, pg + k * step_bytes + b_minus_a); }
      }
      const uint32_t at = position;
      const bool carry = advance(p, q, next);
      x.advance(carry);
      if (BWD) g.advance(carry);
      if (turns) {
        if (lane < p.group) {
          const uint32_t angles = ring + s * slot + STEPS * kStep + 64u * j, none = 0x7fffffffu;
          if (at < (uint32_t)p.table_rows) {
            const float* t = table + (int64_t)at * p.table_ld;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (i < 2 ? l.rot_a : l.rot_b) copy16(angles + 16u * i, t + 4 * i);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) ptx::sts128(angles + 16u * i, make_uint4(none, none, none, none));
          }
        }
        if (next.row < rows) position = position_of(p, next);
      }
    }
    copies_commit();
  };
  if (!(l.has_a && l.has_b)) {                                  // chunks that a lane has not are zeros, which are never copied over
    for (uint32_t at = ring + lane * 16u; at < ring + kStages * slot; at += slot) {
#pragma unroll
      for (int c = 0; c < STEPS * kStep / 512; ++c)
        if (!(c / (kC / 512) & 1 ? l.has_b : l.has_a)) ptx::sts128(at + 512u * c, make_uint4(0u, 0u, 0u, 0u));
    }
  }
  for (int s = 0; s < kStages - 1; ++s) issue(s);
  begin();                                                      // what else has to be fetched, while those are on their way
  const int y_es = dtype_size(q.y_dt);
  const int y_step = per * p.width * y_es, y_b = (l.b - l.a) * y_es;
  Place<!BWD> y(static_cast<char*>(q.y) + first * y_es, now, q, q.y_ld * y_es, y_step * STEPS);
  for (int s = 0; now.row < rows; y.advance(advance(p, q, now))) {
    copies_wait<kStages - 2>();
    __syncwarp();
    issue(s == 0 ? kStages - 1 : s - 1);                        // the slot that the last unit was read from
    const uint32_t from = ring + s * slot;
    const int heads = q.heads - (int)now.block * (per * STEPS) - lane / p.group;
    work(heads, from + lane * 16u, from + STEPS * kStep + 64u * j, y.at(now), y_step, y_b);
    if (++s == kStages) s = 0;
  }
  copies_wait<0>();
}

// DT: type of the inputs.
template <int DT, int STEPS, bool NEIGHBOURS, bool FULL>
__global__ void __launch_bounds__(kThreads, kFwdCtasPerSm) qk_fwd_kernel(const __grid_constant__ QkArgs p) {
  extern __shared__ __align__(16) float smem[];
  const int zero = ptx::grid_wait_previous();
  const QkPart& q = p.part[part_of(p, blockIdx.x)];
  with_output(q.y_dt, [&](auto y_dt) {
  const int lane = threadIdx.x & 31, per = 32 / p.group;
  const Lane l = lane_of<NEIGHBOURS, FULL>(p, lane & (p.group - 1));
  f32x2 wa[4], wb[4];
  const uint32_t ring = ptx::smem_addr(smem) + (threadIdx.x >> 5) * kStages * slot_bytes<false, DT, STEPS>(p.group);
  walk<false, DT, STEPS>(p, q, l, ring, zero, [&] { load_weight(q, l, wa, wb); }, [&](int heads, uint32_t data, uint32_t angles, char* y, int y_step, int y_b) {
    Turn<NEIGHBOURS> turn;
    if (FULL || p.table) read_turn<NEIGHBOURS, false>(angles, l, turn);
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const uint32_t from = data + k * 2 * kChunkBytes<DT>;
      f32x2 a[4], b[4], ss = 0ull;
      widen<DT>(from, a);
      widen<DT>(from + kChunkBytes<DT>, b);
#pragma unroll
      for (int i = 0; i < 4; ++i) ss = fma2(a[i], a[i], fma2(b[i], b[i], ss));
      const f32x2 r = splat2(rsqrt_approx(fmaf(group_sum(halves_sum(ss), p.group), p.inv_width, p.eps)));
#pragma unroll
      for (int i = 0; i < 4; ++i) { a[i] = mul2(mul2(a[i], r), wa[i]); b[i] = mul2(mul2(b[i], r), wb[i]); }
      if (FULL || p.table) rotate<NEIGHBOURS>(a, b, turn, l);
      if (k * per < heads && l.has_a) put<decltype(y_dt)::value>(y + k * y_step, a);
      if (k * per < heads && l.has_b) put<decltype(y_dt)::value>(y + k * y_step + y_b, b);
    }
  });
  });
}

template <int DT, int STEPS, bool NEIGHBOURS, bool FULL>
__global__ void __launch_bounds__(kThreads, kBwdCtasPerSm) qk_bwd_kernel(const __grid_constant__ QkArgs p) {
  extern __shared__ __align__(16) float smem[];
  const int zero = ptx::grid_wait_previous();
  const QkPart& q = p.part[part_of(p, blockIdx.x)];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = 32 / p.group;
  const Lane l = lane_of<NEIGHBOURS, FULL>(p, lane & (p.group - 1));
  f32x2 wa[4], wb[4], da2[4] = {}, db2[4] = {};
  const uint32_t ring = ptx::smem_addr(smem) + warp * kStages * slot_bytes<true, DT, STEPS>(p.group);
  with_output(q.y_dt, [&](auto y_dt) {
  walk<true, DT, STEPS>(p, q, l, ring, zero, [&] { load_weight(q, l, wa, wb); }, [&](int heads, uint32_t data, uint32_t angles, char* y, int y_step, int y_b) {
    Turn<NEIGHBOURS> turn;
    if (FULL || p.table) read_turn<NEIGHBOURS, true>(angles, l, turn);
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const uint32_t from = data + k * 4 * kChunkBytes<DT>;
      f32x2 a[4], b[4], na[4], nb[4], ss2 = 0ull, dot2 = 0ull;
      widen<DT>(from, a);
      widen<DT>(from + kChunkBytes<DT>, b);
      widen<DT>(from + 2 * kChunkBytes<DT>, na);
      widen<DT>(from + 3 * kChunkBytes<DT>, nb);
      if (FULL || p.table) rotate<NEIGHBOURS>(na, nb, turn, l);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ss2 = fma2(a[i], a[i], fma2(b[i], b[i], ss2));
        dot2 = fma2(mul2(na[i], wa[i]), a[i], fma2(mul2(nb[i], wb[i]), b[i], dot2));
      }
      float ss = halves_sum(ss2), dot = halves_sum(dot2);
      for (int o = p.group >> 1; o > 0; o >>= 1) {
        ss += __shfl_xor_sync(0xffffffffu, ss, o);
        dot += __shfl_xor_sync(0xffffffffu, dot, o);
      }
      if (k * per >= heads) continue;                     // (what its slots hold is not of this unit)
      const float r = rsqrt_approx(fmaf(ss, p.inv_width, p.eps));
      // mean(u xhat) = r dot / width, times xhat = x r
      const f32x2 m = splat2(-dot * r * r * p.inv_width), br = splat2(p.beta_x * r), r2 = splat2(r);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        da2[i] = fma2(na[i], mul2(a[i], r2), da2[i]);
        db2[i] = fma2(nb[i], mul2(b[i], r2), db2[i]);
        a[i] = mul2(br, fma2(a[i], m, mul2(na[i], wa[i])));
        b[i] = mul2(br, fma2(b[i], m, mul2(nb[i], wb[i])));
      }
      if (l.has_a) put<decltype(y_dt)::value>(y + k * y_step, a);
      if (l.has_b) put<decltype(y_dt)::value>(y + k * y_step + y_b, b);
    }
  });
  });
  if (!q.dw) return;
  float da[8], db[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) { unpack2(da2[i], da[2 * i], da[2 * i + 1]); unpack2(db2[i], db[2 * i], db[2 * i + 1]); }
  for (int o = p.group; o < 32; o <<= 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      da[i] += __shfl_xor_sync(0xffffffffu, da[i], o);
      db[i] += __shfl_xor_sync(0xffffffffu, db[i], o);
    }
  }
  __syncthreads();                                        // every warp is through with its ring, which the sums take the place of
  if (lane < p.group) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (l.has_a) smem[warp * p.width + l.a + i] = da[i];
      if (l.has_b) smem[warp * p.width + l.b + i] = db[i];
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < p.width; c += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) v += smem[k * p.width + c];
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
    const float* t = p.table ? angles_at(p, position_of(p, row)) : nullptr;
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
    const int64_t span = period ? std::min(period, a.rows) : a.rows;                // (start + span may pass 2^63)
    if (!positions && a.rows > 0 && (span > table->rows || start > table->rows - span)) return US_ERR_INVALID_ARG;
    if (positions && reinterpret_cast<uintptr_t>(positions) % 4) return US_ERR_ALIGNMENT;
    a.table = static_cast<const float*>(table->ptr); a.table_ld = table->ld; a.table_rows = table->rows;
    a.positions = positions; a.start = start; a.period = period < a.rows ? (uint32_t)period : 0; a.rotated = (int)table->cols;
    c.vec = c.vec && table->rows < (1ll << 31) && aligned(*table, 16) && a.rotated % (neighbours ? 8 : 16) == 0;
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

// Deals the CTAs to the parts by their heads; returns the grid.  A part's work is its units, per_block heads each, so that parts get what they need where their heads fill units; one whose
// heads do not (a unit holds heads of one row only) has more units than its heads say, and ends last.  (8192 tokens in BF16, heads of 64, forward / backward us: 16 + 16 heads 13.4 / 22.2,
// 16 + 4 19.2 / 31.1, 16 + 1 54.7 / 82.9; of 128: 32 + 8 30.9 / 50.5, 32 + 4 37.9 / 59.8.)
int deal(QkArgs& a, int per_block, int most) {
  int64_t all = 0;
  for (int k = 0; k < a.count; ++k) {
    QkPart& q = a.part[k];
    q.blocks = std::max(1, (q.heads + per_block - 1) / per_block);
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
    const int64_t step = (int64_t)q.ctas * kWarps, blocks = q.blocks;
    q.step_rows = (uint32_t)(step / blocks); q.step_blocks = (uint32_t)(step % blocks);
    q.step_position = a.period ? q.step_rows % a.period : q.step_rows;
  }
  return grid;
}

template <bool BWD, int DT, int STEPS>
us_status launch_vec(Call& c, int neighbours, int sms, cudaStream_t st) {
  // as many CTAs an SM as their rings leave room for, and no more
  const size_t smem = (size_t)kWarps * kStages * slot_bytes<BWD, DT, STEPS>(c.a.group);
  constexpr size_t most = (size_t)kWarps * kStages * slot_bytes<BWD, DT, STEPS>(32);
  const int grid = deal(c.a, 32 / c.a.group * STEPS, sms * std::min(BWD ? kBwdCtasPerSm : kFwdCtasPerSm, (int)((227 << 10) / (smem + 1024))));
  const bool full = c.a.table && c.a.rotated == c.a.width && c.a.group * 16 == c.a.width;
  static std::atomic<uint64_t> smem_set[4];
  auto go = [&](auto kern) {
    if (!host::allow_smem(kern, smem_set[2 * full + neighbours], most)) return host::failed();
    return host::launch(kern, nullptr, grid, kThreads, smem, 1, st, c.a);
  };
  if constexpr (BWD) {
    if (full) return neighbours ? go(qk_bwd_kernel<DT, STEPS, true, true>) : go(qk_bwd_kernel<DT, STEPS, false, true>);
    return neighbours ? go(qk_bwd_kernel<DT, STEPS, true, false>) : go(qk_bwd_kernel<DT, STEPS, false, false>);
  } else {
    if (full) return neighbours ? go(qk_fwd_kernel<DT, STEPS, true, true>) : go(qk_fwd_kernel<DT, STEPS, false, true>);
    return neighbours ? go(qk_fwd_kernel<DT, STEPS, true, false>) : go(qk_fwd_kernel<DT, STEPS, false, false>);
  }
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
  if (c.dt == US_F32) return launch_vec<BWD, US_F32, 1>(c, neighbours, sms, st);
  return c.dt == US_BF16 ? launch_vec<BWD, US_BF16, 2>(c, neighbours, sms, st) : launch_vec<BWD, US_F16, 2>(c, neighbours, sms, st);
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
