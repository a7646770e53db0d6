// The router of a mixture-of-experts layer: every token's scores, the experts it goes to and
// their weights, in one launch.
//
//   l = x W^T                                     x [M, H], W [E, H] bf16, float32 sums
//   s = softmax(l)  or  1 / (1 + exp(-l))
//   the k experts with the largest s (+ bias, with the sigmoid), descending, the lower index
//   first among equals, NaN behind everything
//   w = s (or s divided by the sum of the chosen) times `scale`
// softmax keeps the order of l, so l itself is compared; the sigmoid does not in 32 bits (scores
// near 1 meet) and a bias moves borders, so that key, like the sigmoid's weights, is computed
// in 64 bits.
//
// The product is MFMA work with 16 experts as rows and 16 tokens as columns.  A wave owns a tile of
// experts, or a part of H where there are fewer tiles than waves.  Many tokens: a workgroup takes
// 32 of them and all experts, and its waves choose from the logits in LDS.  Few tokens: a
// workgroup a tile of experts, so that W is read by as many CUs as there are tiles; the last one
// to arrive of a block of 16 tokens reads the block's logits back and chooses.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;
using dev::u32x4v;

constexpr int kWaves = 8, kThreads = 64 * kWaves;

// Unsigned integers in the order of the numbers, 0 for none, NaN below everything.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);           // -0 is 0
  return x != x ? 1u : u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t u = __double_as_longlong(x + 0.0);
  return x != x ? 1u : u ^ (u >> 63 ? ~uint64_t{0} : uint64_t{1} << 63);
}

// A lane's value at other lanes of its wave by a row shift or broadcast, 0 from outside.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t shifted(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, kRows, 0xF, false));
}
template <int kCtrl, int kRows>
__device__ __forceinline__ uint64_t shifted(uint64_t x) {
  return static_cast<uint64_t>(shifted<kCtrl, kRows>(static_cast<uint32_t>(x >> 32))) << 32 |
         shifted<kCtrl, kRows>(static_cast<uint32_t>(x));
}
__device__ __forceinline__ uint32_t at_lane(uint32_t x, int lane) {
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), lane));
}
__device__ __forceinline__ uint64_t at_lane(uint64_t x, int lane) {
  return static_cast<uint64_t>(at_lane(static_cast<uint32_t>(x >> 32), lane)) << 32 |
         at_lane(static_cast<uint32_t>(x), lane);
}
template <typename T>
__device__ __forceinline__ T wave_most(T x) {
  x = max(x, shifted<0x111, 0xF>(x));
  x = max(x, shifted<0x112, 0xF>(x));
  x = max(x, shifted<0x114, 0xF>(x));
  x = max(x, shifted<0x118, 0xF>(x));
  x = max(x, shifted<0x142, 0xA>(x));
  x = max(x, shifted<0x143, 0xC>(x));
  return at_lane(x, 63);
}

__device__ __forceinline__ double wave_sum64(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}

__device__ __forceinline__ double sigmoid64(float l) { return 1.0 / (1.0 + exp(-static_cast<double>(l))); }

// One token by a wave.  Lane i holds experts kR i .. kR i + kR - 1, so that the first lane with
// the largest key has the lowest index of equal ones.  logit(e): expert e's.
template <int kR, bool kSigmoid, typename Logit>
__device__ __forceinline__ void choose(const RouteArgs& p, int token, Logit logit) {
  using Key = std::conditional_t<kSigmoid, uint64_t, uint32_t>;
  const int lane = static_cast<int>(threadIdx.x) & 63;
  float l[kR];
  Key key[kR];
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    const int e = lane * kR + i;
    l[i] = e < p.E ? logit(e) : -__builtin_inff();
    key[i] = 0;
    if (e < p.E) {
      if constexpr (kSigmoid) key[i] = ordered(sigmoid64(l[i]) + static_cast<double>(p.bias ? p.bias[e] : 0.f));
      else key[i] = ordered(l[i]);
      if (p.logits) p.logits[token * p.ld_logits + e] = l[i];
    }
  }
  int id = 0;                                   // lane j: the j-th expert
  float mine = 0.f, first = 0.f;
  for (int j = 0; j < p.k; ++j) {
    Key best = key[0];
    int at = 0;
    float best_l = l[0];
#pragma unroll
    for (int i = 1; i < kR; ++i)
      if (key[i] > best) best = key[i], at = i, best_l = l[i];
    const Key most = wave_most(best);
    const int from = __builtin_ctzll(__ballot(best == most));
    const int e = __builtin_amdgcn_readlane(lane * kR + at, from);
    const float chosen = __uint_as_float(at_lane(__float_as_uint(best_l), from));
#pragma unroll
    for (int i = 0; i < kR; ++i)
      if (lane == from && at == i) key[i] = 0;
    if (lane == j) id = e, mine = chosen;
    if (j == 0) first = chosen;
  }
  float w = 0.f;
  if constexpr (kSigmoid) {
    double s = lane < p.k ? sigmoid64(mine) : 0.0;
    if (p.renormalize) s /= wave_sum64(s);
    w = static_cast<float>(s * p.scale);
  } else {
    const float s = lane < p.k ? expf(mine - first) : 0.f;
    float total = s;
    if (!p.renormalize) {
      total = 0.f;
#pragma unroll
      for (int i = 0; i < kR; ++i)
        if (lane * kR + i < p.E) total += expf(l[i] - first);
    }
    w = s / dev::wave_sum(total) * p.scale;
  }
  if (lane < p.k) {
    p.ids[static_cast<int64_t>(token) * p.k + lane] = id;
    p.weights[static_cast<int64_t>(token) * p.k + lane] = w;
  }
}

template <typename Logit>
__device__ __forceinline__ void choose_any(const RouteArgs& p, int token, Logit logit) {
  auto go = [&](auto sigmoid) {
    constexpr bool kS = decltype(sigmoid)::value;
    if (p.E <= 64) choose<1, kS>(p, token, logit);
    else if (p.E <= 128) choose<2, kS>(p, token, logit);
    else if (p.E <= 256) choose<4, kS>(p, token, logit);
    else if (p.E <= 512) choose<8, kS>(p, token, logit);
    else choose<16, kS>(p, token, logit);
  };
  if (p.sigmoid) go(std::true_type{});
  else go(std::false_type{});
}

// Floats between two tokens' logits in LDS: 4 past a multiple of 32, so that the 16 tokens of a
// tile's float4 stores lie in different banks.
__host__ __device__ inline int pitch_of(int experts) { return ((experts + 31) & ~31) + 4; }

// kG blocks of 16 tokens and kTw tiles of 16 experts a workgroup at a time, kWaves / kTw parts of H.
template <int kG, int kTw, bool kSplit>
__global__ __launch_bounds__(kThreads) void moe_route_kernel(const RouteArgs p, float* parts, uint32_t* arrived) {
  constexpr int kKs = kWaves / kTw, kRows = 16 * kG;
  extern __shared__ __align__(16) float sh[];   // [kKs][kRows][pitch]
  __shared__ int sh_last;
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int c = lane & 15, q = lane >> 4;
  const int token0 = static_cast<int>(blockIdx.x) * kRows;
  const int tiles = (p.E + 15) >> 4;
  const int first = kSplit ? static_cast<int>(blockIdx.y) : 0, last = kSplit ? first + 1 : tiles;
  const int pitch = pitch_of(kSplit ? 16 : p.E);
  const int part = wave / kTw;
  const int steps = (p.H + 127) >> 7;           // of 128: lane group q has elements 32 q .. 32 q + 31 of each

  const uint16_t* x[kG];
#pragma unroll
  for (int g = 0; g < kG; ++g)                  // columns past M: the last token's again, not stored
    x[g] = p.x + static_cast<int64_t>(min(token0 + 16 * g + c, p.M - 1)) * p.ld_x;
  for (int t = first + wave % kTw; t < last; t += kTw) {
    const uint16_t* w = p.w + static_cast<int64_t>(min(16 * t + c, p.E - 1)) * p.ld_w;
    f32x4 acc[kG] = {};
#pragma unroll 2
    for (int s = part; s < steps; s += kKs) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = 128 * s + 32 * q + 8 * j;
        u32x4v a = 0u;
        if (at < p.H) a = *reinterpret_cast<const u32x4v*>(w + at);
#pragma unroll
        for (int g = 0; g < kG; ++g) {
          u32x4v b = 0u;
          if (at < p.H) b = *reinterpret_cast<const u32x4v*>(x[g] + at);
          acc[g] = dev::mfma_bf16(a, b, acc[g]);
        }
      }
    }
#pragma unroll
    for (int g = 0; g < kG; ++g)
      *reinterpret_cast<f32x4*>(sh + (part * kRows + 16 * g + c) * pitch + 16 * (t - first) + 4 * q) = acc[g];
  }
  __syncthreads();
  if constexpr (!kSplit) {
    for (int i = wave; i < kRows && token0 + i < p.M; i += kWaves)
      choose_any(p, token0 + i, [&](int e) {
        float l = sh[i * pitch + e];
#pragma unroll
        for (int ks = 1; ks < kKs; ++ks) l += sh[(ks * kRows + i) * pitch + e];
        return l;
      });
  } else {
    // The tile's logits for whoever arrives last: device-scope accesses, since that may be another
    // XCD with an L2 of its own.
    if (tid < 256) {
      const int i = tid >> 4, e = tid & 15;
      float l = 0.f;
#pragma unroll
      for (int ks = 0; ks < kKs; ++ks) l += sh[(ks * kRows + i) * pitch + e];
      if (token0 + i < p.M && 16 * first + e < p.E)
        __hip_atomic_store(parts + static_cast<int64_t>(token0 + i) * p.E + 16 * first + e, l, __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // what this wave has stored is there
    __syncthreads();
    if (tid == 0)
      sh_last = __hip_atomic_fetch_add(arrived + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                static_cast<uint32_t>(tiles - 1);
    __syncthreads();
    if (!sh_last) return;
    if (tid == 0) __hip_atomic_store(arrived + blockIdx.x, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int i = wave; i < kRows && token0 + i < p.M; i += kWaves)
      choose_any(p, token0 + i, [&](int e) {
        return __hip_atomic_load(parts + static_cast<int64_t>(token0 + i) * p.E + e, __ATOMIC_RELAXED,
                                 __HIP_MEMORY_SCOPE_AGENT);
      });
  }
}

}  // namespace

RoutePlan plan_moe_route(int M, int E, int H, int num_cus) {
  RoutePlan c;
  const int tiles = (E + 15) / 16;
  c.split = tiles > 1 && M <= 16 * num_cus / 4;
  c.rows = c.split ? 16 : 32;
  c.blocks = (static_cast<int64_t>(M) + c.rows - 1) / c.rows;
  return c;
}

size_t route_workspace_bytes(const RoutePlan& c, int M, int E) {
  return c.split ? kWorkspaceStateBytes + static_cast<size_t>(M) * E * 4 : 0;
}

hipError_t launch_moe_route(const RoutePlan& c, const RouteArgs& p, void* workspace, hipStream_t stream) {
  const int tiles = (p.E + 15) / 16, grid = static_cast<int>(c.blocks);
  if (c.split) {
    static_assert(kWaves * 16 * (32 + 4) * 4 <= 64 * 1024, "LDS");
    float* parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + kWorkspaceStateBytes);
    moe_route_kernel<1, 1, true><<<dim3(grid, tiles), kThreads, kWaves * 16 * pitch_of(16) * 4, stream>>>(
        p, parts, static_cast<uint32_t*>(workspace));
    return hipGetLastError();
  }
  auto go = [&](auto tw) {
    constexpr int kTw = decltype(tw)::value;
    const void* fn = reinterpret_cast<const void*>(&moe_route_kernel<2, kTw, false>);
    const int lds = kWaves / kTw * 32 * pitch_of(p.E) * 4;
    if (lds > 64 * 1024) {
      const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e != hipSuccess) return e;
    }
    moe_route_kernel<2, kTw, false><<<grid, kThreads, lds, stream>>>(p, nullptr, nullptr);
    return hipGetLastError();
  };
  if (tiles > 4) return go(std::integral_constant<int, 8>{});
  if (tiles > 2) return go(std::integral_constant<int, 4>{});
  if (tiles > 1) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 1>{});
}

}  // namespace prq
