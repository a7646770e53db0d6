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
// reductions, so that nothing is read twice.  8192 rows of 2560, float32: 48.6 us, 293 MB at
// 6.0 TB/s (a large copy here 5.4, a sum of two tensors 5.9); one row of 2048: 2.0 us.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;

constexpr int kThreads = 256;
template <int kValue>
using Int = std::integral_constant<int, kValue>;

// Four elements as they lie in memory; their values are made where they are used, so that no load is
// waited for among the others.
template <typename T>
using Raw = std::conditional_t<std::is_same_v<T, float>, f32x4, dev::u32x2>;
template <bool kOnce, typename T>
__device__ __forceinline__ Raw<T> load4(const T* p, int64_t at) {
  const Raw<T>* from = reinterpret_cast<const Raw<T>*>(p + at);
  if constexpr (kOnce) return __builtin_nontemporal_load(from);
  else return *from;
}
__device__ __forceinline__ f32x4 values(f32x4 x) { return x; }
__device__ __forceinline__ f32x4 values(dev::u32x2 w) {
  return {dev::bf16_lo(w.x), dev::bf16_hi(w.x), dev::bf16_lo(w.y), dev::bf16_hi(w.y)};
}
template <bool kOnce, typename T>
__device__ __forceinline__ void store4(T* p, int64_t at, f32x4 x) {
  Raw<T> v;
  if constexpr (std::is_same_v<T, float>) v = x;
  else v = Raw<T>{dev::pack_bf16(x[0], x[1]), dev::pack_bf16(x[2], x[3])};
  Raw<T>* to = reinterpret_cast<Raw<T>*>(p + at);
  if constexpr (kOnce) __builtin_nontemporal_store(v, to);
  else *to = v;
}
// The same of a weight or a gate, whose type the call says.
struct Weight {
  dev::u32x4v raw;
  __device__ __forceinline__ void load(const void* p, bool bf16, int64_t at) {
    if (bf16) {
      const dev::u32x2 w = *reinterpret_cast<const dev::u32x2*>(static_cast<const uint16_t*>(p) + at);
      raw[0] = w.x;
      raw[1] = w.y;
    } else {
      raw = *reinterpret_cast<const dev::u32x4v*>(static_cast<const float*>(p) + at);
    }
  }
  __device__ __forceinline__ f32x4 get(bool bf16) const {
    return bf16 ? values(dev::u32x2{raw[0], raw[1]}) : __builtin_bit_cast(f32x4, raw);
  }
};

// The sum over a row's lanes, in every one of them.  sh: 4 floats that nothing else uses
// between two calls.
template <int kLanes>
__device__ __forceinline__ float row_sum(float x, float* sh) {
  x = dev::wave_sum(x);
  if constexpr (kLanes > 64) {
    const int wave = static_cast<int>(threadIdx.x) >> 6;
    if ((threadIdx.x & 63) == 0) sh[wave] = x;
    __syncthreads();
    x = kLanes == kThreads ? (sh[0] + sh[1]) + (sh[2] + sh[3]) : sh[wave & 2] + sh[wave | 1];
  }
  return x;
}

__device__ __forceinline__ float dot4(f32x4 x) { return (x[0] * x[0] + x[1] * x[1]) + (x[2] * x[2] + x[3] * x[3]); }

// kLanes lanes a row (a wave, two or the workgroup), kU quadruples a lane.  kOnce: what is more than the
// caches keep is loaded and stored past them.
template <typename Y, typename R, int kLanes, int kU, bool kOnce>
__global__ __launch_bounds__(kThreads) void block_norm_kernel(const BlockNormArgs p) {
  constexpr int kRows = kThreads / kLanes;
  constexpr bool kEarly = kU <= 4;              // weights and gate in registers from the start
  __shared__ float sh[2][4];
  const int lane = static_cast<int>(threadIdx.x) % kLanes;
  // Past the last row: nothing to wait for where a wave is a row, else that row again, not stored.
  const int64_t own = static_cast<int64_t>(blockIdx.x) * kRows + static_cast<int>(threadIdx.x) / kLanes;
  if (kLanes == 64 && own >= p.M) return;
  const int64_t row = min(own, p.M - 1);
  const bool live = own < p.M;
  const Y* y = static_cast<const Y*>(p.y);
  const R* r = static_cast<const R*>(p.residual);
  R* r_out = static_cast<R*>(p.residual_out);
  // A lane's i-th quadruple; past the end the row's last one, whose values are made zeros.
  auto place = [&](int i) { return min(4 * (lane + i * kLanes), p.H - 4); };
  auto in = [&](int i) { return 4 * (lane + i * kLanes) < p.H; };

  Raw<Y> y_raw[kU];
  Raw<R> r_raw[kU];
  if (y) {
#pragma unroll
    for (int i = 0; i < kU; ++i) y_raw[i] = load4<kOnce>(y, row * p.ld_y + place(i));
  }
  if (r) {
#pragma unroll
    for (int i = 0; i < kU; ++i) r_raw[i] = load4<kOnce>(r, row * p.ld_r + place(i));
  }
  int64_t gate_row = p.gate ? 0 : -1;
  if (p.gate) gate_row = p.gate_index ? p.gate_index[row] : p.gate_rows > 1 ? row : 0;
  const bool gated = gate_row >= 0 && gate_row < p.gate_rows;     // a row that names none has none
  Weight post[kU], gate[kU], pre[kU];
  auto weights = [&](Weight (&w)[kU], const void* from, bool bf16, int64_t at) {
#pragma unroll
    for (int i = 0; i < kU; ++i) w[i].load(from, bf16, at + place(i));
  };
  if constexpr (kEarly) {
    if (p.post) weights(post, p.post, p.w_bf16, 0);
    if (p.pre) weights(pre, p.pre, p.w_bf16, 0);
    if (gated) weights(gate, p.gate, p.gate_bf16, gate_row * p.ld_gate);
  }
  f32x4 u[kU], x[kU];
#pragma unroll
  for (int i = 0; i < kU; ++i) u[i] = y && in(i) ? values(y_raw[i]) : f32x4{};
#pragma unroll
  for (int i = 0; i < kU; ++i) x[i] = r && in(i) ? values(r_raw[i]) : f32x4{};

  if (p.post) {
    if constexpr (!kEarly) weights(post, p.post, p.w_bf16, 0);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kU; ++i) s += dot4(u[i]);
    const float inv = 1.0f / sqrtf(row_sum<kLanes>(s, sh[0]) / static_cast<float>(p.H) + p.eps);
#pragma unroll
    for (int i = 0; i < kU; ++i) u[i] *= inv * (post[i].get(p.w_bf16) + p.offset);
  }
  if (gated) {
    if constexpr (!kEarly) weights(gate, p.gate, p.gate_bf16, gate_row * p.ld_gate);
#pragma unroll
    for (int i = 0; i < kU; ++i) u[i] *= gate[i].get(p.gate_bf16);
  }
  if constexpr (!kEarly)
    if (p.pre) weights(pre, p.pre, p.w_bf16, 0);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kU; ++i) {
    x[i] = p.a * x[i] + p.b * u[i];
    if (r_out && live && in(i)) store4<kOnce>(r_out, row * p.ld_ro + place(i), x[i]);
    if (in(i)) s += dot4(x[i]);
  }
  if (!p.pre) return;
  const float inv = 1.0f / sqrtf(row_sum<kLanes>(s, sh[1]) / static_cast<float>(p.H) + p.eps);
#pragma unroll
  for (int i = 0; i < kU; ++i)
    if (live && in(i)) store4<kOnce>(p.h, row * p.ld_h + place(i), x[i] * inv * (pre[i].get(p.w_bf16) + p.offset));
}

}  // namespace

NormPlan plan_block_norm(const BlockNormArgs& p, bool y_bf16, bool r_bf16) {
  NormPlan c;
  // A wave a row up to 512 elements, else the workgroup: few quadruples a lane beat rows without a
  // barrier (us, a wave / the workgroup: 61 rows of 2560 9.6 / 4.4, 1537 of 1056 8.7 / 7.6, 8192 of 2560
  // in float32 71 / 52).  Many rows of up to 1536, three quadruples a lane, by half a workgroup each (the
  // workgroup / half: 512 rows of 1024 2.9 / 3.0, 1537 of 1056 6.9 / 6.35, 4096 of 1024 9.7 / 8.5, 20000 38 / 31,
  // 4096 of 1536 13.2 / 12.7; but of 2048 14.2 / 14.5).
  c.lanes = p.H <= 512 ? 64 : p.H <= 1536 && p.M >= 1024 ? 128 : kThreads;
  const int per = (p.H + 4 * c.lanes - 1) / (4 * c.lanes);
  c.quads = per <= 4 ? per : per <= 8 ? 8 : 16;
  // What does not fit the last cache (256 MB) goes past it: 8192 rows of 2560 in float32 51.8 -> 48.6 us;
  // less than that the next kernel finds there.
  const int64_t each = (p.y ? (y_bf16 ? 2 : 4) : 0) +
                       (r_bf16 ? 2 : 4) * ((p.residual != nullptr) + (p.residual_out != nullptr)) + (p.h ? 2 : 0);
  c.once = p.M * p.H * each > (int64_t{256} << 20);
  return c;
}

hipError_t launch_block_norm(const BlockNormArgs& p, bool y_bf16, bool r_bf16, hipStream_t stream) {
  const NormPlan c = plan_block_norm(p, y_bf16, r_bf16);
  auto of_types = [&](auto y, auto r) {
    using Y = decltype(y);
    using R = decltype(r);
    auto go = [&](auto kernel) {
      const int rows = kThreads / c.lanes;
      kernel<<<static_cast<int>((p.M + rows - 1) / rows), kThreads, 0, stream>>>(p);
      return hipGetLastError();
    };
    auto with = [&](auto lanes, auto quads) {
      constexpr int kLanes = decltype(lanes)::value, kU = decltype(quads)::value;
      if constexpr (kLanes == kThreads && kU == 1)             // (fewer than 1024 rows of 1024)
        return go(&block_norm_kernel<Y, R, kLanes, kU, false>);
      else
        return go(c.once ? &block_norm_kernel<Y, R, kLanes, kU, true> : &block_norm_kernel<Y, R, kLanes, kU, false>);
    };
    const Int<64> wave{};
    const Int<128> half{};
    const Int<kThreads> whole{};
    if (c.lanes == 64) return c.quads == 1 ? with(wave, Int<1>{}) : with(wave, Int<2>{});
    if (c.lanes == 128) return c.quads == 2 ? with(half, Int<2>{}) : with(half, Int<3>{});
    switch (c.quads) {
      case 1: return with(whole, Int<1>{});
      case 2: return with(whole, Int<2>{});
      case 3: return with(whole, Int<3>{});
      case 4: return with(whole, Int<4>{});
      case 8: return with(whole, Int<8>{});
      default: return with(whole, Int<16>{});
    }
  };
  if (y_bf16) return r_bf16 ? of_types(uint16_t{}, uint16_t{}) : of_types(uint16_t{}, float{});
  return r_bf16 ? of_types(float{}, uint16_t{}) : of_types(float{}, float{});
}

}  // namespace prq
