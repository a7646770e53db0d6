// What stands between two blocks of a layer, in one pass over the rows: the norm behind the
// block (optional), its gate (optional), the scaled sum with the residual and the norm before
// the next block (optional).
//
// A row of H elements, y the block's output, r the residual, w_post and w_pre the norms'
// weights, o their offset, g the row's gate, a and b the scales:
//   u  = y                                     or  y / sqrt(mean(y^2) + eps) * (o + w_post)
//   r' = a r + b g u
//   h  = r' / sqrt(mean(r'^2) + eps) * (o + w_pre)
// in float32; r' rounded once as it is stored (h takes it unrounded), h once, to bf16.
//
// Bytes: y, r, r' and h once each; HBM bounds many rows, the launch and two dependent
// reductions a few.  A row's elements stay in the registers of its lanes between the
// reductions, so that nothing is read twice.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;

constexpr int kThreads = 256;

__device__ __forceinline__ f32x4 load4(const float* p, int64_t at) { return *reinterpret_cast<const f32x4*>(p + at); }
__device__ __forceinline__ f32x4 load4(const uint16_t* p, int64_t at) {
  const dev::u32x2 w = *reinterpret_cast<const dev::u32x2*>(p + at);
  return {dev::bf16_lo(w.x), dev::bf16_hi(w.x), dev::bf16_lo(w.y), dev::bf16_hi(w.y)};
}
__device__ __forceinline__ void store4(float* p, int64_t at, f32x4 x) { *reinterpret_cast<f32x4*>(p + at) = x; }
__device__ __forceinline__ void store4(uint16_t* p, int64_t at, f32x4 x) {
  const dev::u32x2 w = {dev::pack_bf16(x[0], x[1]), dev::pack_bf16(x[2], x[3])};
  *reinterpret_cast<dev::u32x2*>(p + at) = w;
}
// A weight or gate, float32 or bf16.
__device__ __forceinline__ f32x4 load4(const void* p, bool bf16, int64_t at) {
  return bf16 ? load4(static_cast<const uint16_t*>(p), at) : load4(static_cast<const float*>(p), at);
}

// The sum over a row's lanes, in every one of them.  sh: 4 floats that nothing else uses
// between two calls.
template <int kLanes>
__device__ __forceinline__ float row_sum(float x, float* sh) {
  x = dev::wave_sum(x);
  if constexpr (kLanes > 64) {
    const int wave = static_cast<int>(threadIdx.x) >> 6;
    if ((threadIdx.x & 63) == 0) sh[wave] = x;
    __syncthreads();
    x = (sh[0] + sh[1]) + (sh[2] + sh[3]);
  }
  return x;
}

__device__ __forceinline__ float dot4(f32x4 x) { return (x[0] * x[0] + x[1] * x[1]) + (x[2] * x[2] + x[3] * x[3]); }

// kLanes lanes a row (a wave or the workgroup), kU quadruples a lane.
template <typename Y, typename R, int kLanes, int kU>
__global__ __launch_bounds__(kThreads) void block_norm_kernel(const BlockNormArgs p) {
  constexpr int kRows = kThreads / kLanes;
  __shared__ float sh[2][4];
  const int lane = static_cast<int>(threadIdx.x) % kLanes;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + static_cast<int>(threadIdx.x) / kLanes;
  if (row >= p.M) return;                       // a whole wave, and only where a wave is a row
  const Y* y = static_cast<const Y*>(p.y);
  const R* r = static_cast<const R*>(p.residual);
  R* r_out = static_cast<R*>(p.residual_out);

  f32x4 u[kU], x[kU];
#pragma unroll
  for (int i = 0; i < kU; ++i) {
    const int at = 4 * (lane + i * kLanes);
    u[i] = x[i] = 0.f;
    if (at < p.H) {
      if (y) u[i] = load4(y, row * p.ld_y + at);
      if (r) x[i] = load4(r, row * p.ld_r + at);
    }
  }
  int64_t gate_row = p.gate ? 0 : -1;
  if (p.gate) gate_row = p.gate_index ? p.gate_index[row] : p.gate_rows > 1 ? row : 0;
  const bool gated = gate_row >= 0 && gate_row < p.gate_rows;     // a row that names none has none

  if (p.post) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kU; ++i) s += dot4(u[i]);
    const float inv = 1.0f / sqrtf(row_sum<kLanes>(s, sh[0]) / static_cast<float>(p.H) + p.eps);
#pragma unroll
    for (int i = 0; i < kU; ++i) {
      const int at = 4 * (lane + i * kLanes);
      if (at < p.H) u[i] *= inv * (load4(p.post, p.w_bf16, at) + p.offset);
    }
  }
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kU; ++i) {
    const int at = 4 * (lane + i * kLanes);
    if (at < p.H) {
      if (gated) u[i] *= load4(p.gate, p.gate_bf16, gate_row * p.ld_gate + at);
      x[i] = p.a * x[i] + p.b * u[i];
      if (r_out) store4(r_out, row * p.ld_ro + at, x[i]);
    }
    s += dot4(x[i]);
  }
  if (!p.pre) return;
  const float inv = 1.0f / sqrtf(row_sum<kLanes>(s, sh[1]) / static_cast<float>(p.H) + p.eps);
#pragma unroll
  for (int i = 0; i < kU; ++i) {
    const int at = 4 * (lane + i * kLanes);
    if (at < p.H) store4(p.h, row * p.ld_h + at, x[i] * inv * (load4(p.pre, p.w_bf16, at) + p.offset));
  }
}

template <typename Y, typename R, int kLanes>
void launch(const BlockNormArgs& p, hipStream_t stream) {
  constexpr int kRows = kThreads / kLanes;
  const int grid = static_cast<int>((p.M + kRows - 1) / kRows);
  const int per = (p.H + 4 * kLanes - 1) / (4 * kLanes);
  auto go = [&](auto u) {
    block_norm_kernel<Y, R, kLanes, decltype(u)::value><<<grid, kThreads, 0, stream>>>(p);
  };
  if (per <= 1) go(std::integral_constant<int, 1>{});
  else if (per <= 2) go(std::integral_constant<int, 2>{});
  else if (per <= 3) go(std::integral_constant<int, 3>{});
  else if (per <= 4) go(std::integral_constant<int, 4>{});
  else if (per <= 6) go(std::integral_constant<int, 6>{});
  else if (per <= 8) go(std::integral_constant<int, 8>{});
  else if (per <= 10) go(std::integral_constant<int, 10>{});
  else go(std::integral_constant<int, 16>{});
}

}  // namespace

hipError_t launch_block_norm(const BlockNormArgs& p, bool y_bf16, bool r_bf16, int num_cus, hipStream_t stream) {
  // A wave a row where the rows fill the chip, else the workgroup.
  const bool waves = p.M >= 8 * num_cus && p.H <= 10 * 256;
  auto go = [&](auto y, auto r) {
    using Y = decltype(y);
    using R = decltype(r);
    waves ? launch<Y, R, 64>(p, stream) : launch<Y, R, kThreads>(p, stream);
  };
  if (y_bf16) r_bf16 ? go(uint16_t{}, uint16_t{}) : go(uint16_t{}, float{});
  else r_bf16 ? go(float{}, uint16_t{}) : go(float{}, float{});
  return hipGetLastError();
}

}  // namespace prq
