// All experts of a few tokens (up to 64), in two launches: MXFP4 weights, bf16 activations.
//
// Token t with experts e_j and weights w_j, expert e's gate, up and down weights G, U (I x H) and
// D (N x (I + k_tail)):
//   h_e = SiLU(G_e x) * (U_e x),  SiLU(z) = z / (1 + exp(-z))
//   y   = sum_j w_j D_{e_j} [h; the last k_tail of h again]
// Sums are float32.  w h is rounded to bf16 between the launches (the operand of the second
// product's matrix instructions), y to bf16 at the end: two roundings of 2^-9 relative, the second
// of them the output's own.  A token that names an expert twice gets it with both weights; an id
// outside [0, E) names none.
//
// The weights of the experts that are reached are most of the bytes, and what bounds both
// launches; a CU has 80 cycles of matrix work free for every kilobyte of them, so the
// activations stay in bf16 at no cost and the weights are brought to bf16 in registers (a 4-bit
// value times a power of two is exact there).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;
using dev::u32x4v;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kMaxExperts = 4096;
constexpr int kMaxPairs = kMaxLayerTokens * kMaxLayerTop;

// What a workgroup knows about the routing: every pair's expert, and the experts that some token
// goes to in ascending order.
struct Routing {
  int ids[kMaxPairs];
  uint32_t reached[kMaxExperts / 32];
  int experts[kMaxPairs];
};

// Fills `r` and returns the number of experts.  All threads of the workgroup.
__device__ __forceinline__ int read_routing(const MoeArgs& p, Routing& r) {
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63;
  const int pairs = p.M * p.k;
  for (int i = tid; i < kMaxExperts / 32; i += kThreads) r.reached[i] = 0;
  __syncthreads();
  for (int i = tid; i < pairs; i += kThreads) {
    const int e = p.ids[i];
    r.ids[i] = e;
    if (e >= 0 && e < p.E) atomicOr(&r.reached[e >> 5], 1u << (e & 31));
  }
  __syncthreads();
  // Lane i: experts 64 i .. 64 i + 63, and how many are reached before them.
  const int n = __popc(r.reached[2 * lane]) + __popc(r.reached[2 * lane + 1]);
  const int upto = dev::prefix_sum(n);
  for (int e = tid; e < ((p.E + 63) & ~63); e += kThreads) {     // a wave's lanes: the 64 experts of one such group
    const int group = __builtin_amdgcn_readfirstlane(e >> 6);
    const int before = __builtin_amdgcn_readlane(upto, group) - __builtin_amdgcn_readlane(n, group);
    const uint64_t mask = static_cast<uint64_t>(r.reached[2 * group + 1]) << 32 | r.reached[2 * group];
    if (mask >> lane & 1) r.experts[before + __popcll(mask & ((uint64_t{1} << lane) - 1))] = e;
  }
  __syncthreads();
  return __builtin_amdgcn_readlane(upto, 63);
}

// A lane's 32 weights of a K step (the 16 bytes of an MXFP4 block, its E8M0 code) as the four
// bf16 operands of the matrix instruction.
__device__ __forceinline__ void to_bf16(u32x4v w, uint32_t code, u32x4v (&out)[4]) {
  const float scale = __uint_as_float(code << 23);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    out[j][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], scale, 0));
    out[j][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], scale, 1));
    out[j][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], scale, 2));
    out[j][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[j], scale, 3));
  }
}

// A tile of 16 rows of a packed weight: kilobyte s and the dwords that hold its scales.
struct Tile {
  const uint8_t* codes;
  const uint32_t* scales;
  __device__ __forceinline__ Tile(const uint8_t* Wp, const uint8_t* Wps, int64_t tile, int steps) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    codes = Wp + (tile * steps * 64 + lane) * 16;
    scales = reinterpret_cast<const uint32_t*>(Wps) + tile * ((steps + 3) >> 2) * 64 + lane;
  }
  __device__ __forceinline__ u32x4v code(int s) const {
    return *reinterpret_cast<const u32x4v*>(codes + static_cast<int64_t>(s) * 1024);
  }
  __device__ __forceinline__ uint32_t scale(int s) const { return scales[(s >> 2) * 64] >> (8 * (s & 3)) & 255u; }
};

// First launch: one expert's 16 intermediate features (a gate tile and an up tile) for all of its
// tokens; the waves share the steps of H.  kG: blocks of 16 tokens that an expert can have.
template <int kG>
__global__ __launch_bounds__(kThreads) void moe_up_kernel(const MoeArgs p, uint16_t* __restrict__ hidden) {
  extern __shared__ __align__(16) float red[];       // [kWaves][2][kG][64][4]
  __shared__ Routing routing;
  __shared__ int token_of[64], row_of[64];
  __shared__ float weight_of[64];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int c = lane & 15, q = lane >> 4;
  const int n = read_routing(p, routing);
  if (static_cast<int>(blockIdx.y) >= n) return;
  const int e = routing.experts[blockIdx.y], tile = static_cast<int>(blockIdx.x);

  if (wave == 0) {                                   // lane t: token t's share of the expert
    int slot = -1;
    float w = 0.f;
    if (lane < p.M)
      for (int j = 0; j < p.k; ++j)
        if (routing.ids[lane * p.k + j] == e) {
          w += p.weights[lane * p.k + j];
          if (slot < 0) slot = j;
        }
    const uint64_t mine = __ballot(slot >= 0);
    const int at = __popcll(mine & ((uint64_t{1} << lane) - 1));
    token_of[lane] = -1;
    dev::wave_lds_barrier();
    if (slot >= 0) {
      token_of[at] = lane;
      row_of[at] = lane * p.k + slot;
      weight_of[at] = w;
    }
  }
  __syncthreads();

  const int steps = (p.H + 127) >> 7, tiles = p.I >> 4;
  const int64_t first = static_cast<int64_t>(e) * 2 * tiles + tile;
  const Tile gate(p.up_codes, p.up_scales, first, steps), up(p.up_codes, p.up_scales, first + tiles, steps);
  const uint16_t* x[kG];
  int groups = 0;
#pragma unroll
  for (int g = 0; g < kG; ++g) {
    const int t = token_of[16 * g + c];
    x[g] = t < 0 ? nullptr : p.x + t * p.ld_x;
    if (token_of[16 * g] >= 0) groups = g + 1;
  }
  f32x4 acc[2][kG] = {};
  for (int s = wave; s < steps; s += kWaves) {
    u32x4v a[2][4];
    to_bf16(gate.code(s), gate.scale(s), a[0]);
    to_bf16(up.code(s), up.scale(s), a[1]);
    const int at = 128 * s + 32 * q;
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      if (g >= groups) break;
      u32x4v b[4] = {};
      if (x[g] && at < p.H) {
        const u32x4v* from = reinterpret_cast<const u32x4v*>(x[g] + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = from[j];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[0][g] = dev::mfma_bf16(a[0][j], b[j], acc[0][g]);
        acc[1][g] = dev::mfma_bf16(a[1][j], b[j], acc[1][g]);
      }
    }
  }
  f32x4* sums = reinterpret_cast<f32x4*>(red);
#pragma unroll
  for (int g = 0; g < kG; ++g)
    if (g < groups) {
      sums[((wave * 2 + 0) * kG + g) * 64 + lane] = acc[0][g];
      sums[((wave * 2 + 1) * kG + g) * 64 + lane] = acc[1][g];
    }
  __syncthreads();
  for (int g = wave; g < groups; g += kWaves) {
    f32x4 a = 0.f, b = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      a += sums[((w * 2 + 0) * kG + g) * 64 + lane];
      b += sums[((w * 2 + 1) * kG + g) * 64 + lane];
    }
    if (token_of[16 * g + c] >= 0) {                 // column c's features 4 q .. 4 q + 3 of the tile
      const float w = weight_of[16 * g + c];
      float h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = a[i] / (1.f + expf(-a[i])) * b[i] * w;
      const dev::u32x2 v = {dev::pack_bf16(h[0], h[1]), dev::pack_bf16(h[2], h[3])};
      *reinterpret_cast<dev::u32x2*>(hidden + static_cast<int64_t>(row_of[16 * g + c]) * p.I + 16 * tile + 4 * q) = v;
    }
  }
}

// Second launch: 16 output features of all tokens, over the experts that are reached.  Column c of
// block g is token 16 g + c, so that all experts add into the same registers; the units (an
// expert's kilobyte of the tile) are dealt evenly to the waves of the tile's workgroups, in
// order.  The workgroups' sums are added in their order by the one that arrives last.
template <int kG>
__global__ __launch_bounds__(kThreads) void moe_down_kernel(const MoeArgs p, const uint16_t* __restrict__ hidden,
                                                             float* parts, uint32_t* arrived) {
  __shared__ Routing routing;
  __shared__ __align__(16) float red[kWaves * kG * 64 * 4];
  __shared__ int sh_last;
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int c = lane & 15, q = lane >> 4;
  const int n = read_routing(p, routing);
  const int tile = static_cast<int>(blockIdx.x), splits = static_cast<int>(gridDim.y), part = static_cast<int>(blockIdx.y);
  const int K = p.I + p.k_tail, steps = (K + 127) >> 7;
  const int units = n * steps, shares = splits * kWaves, share = part * kWaves + wave;
  int u = static_cast<int>(static_cast<int64_t>(units) * share / shares);
  const int end = static_cast<int>(static_cast<int64_t>(units) * (share + 1) / shares);

  f32x4 acc[kG] = {};
  while (u < end) {
    const int e = routing.experts[u / steps];
    int s = u % steps;
    const int stop = min(steps, s + end - u);
    u += stop - s;
    const Tile down(p.down_codes, p.down_scales, static_cast<int64_t>(e) * (p.N >> 4) + tile, steps);
    int row = -1;                                    // lane t: where token t's share of the expert is
    if (lane < p.M)
      for (int j = p.k - 1; j >= 0; --j)
        if (routing.ids[lane * p.k + j] == e) row = lane * p.k + j;
    const uint64_t mine = __ballot(row >= 0);
    const uint16_t* h[kG];
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      const int at = __shfl(row, 16 * g + c, 64);
      h[g] = at < 0 ? nullptr : hidden + static_cast<int64_t>(at) * p.I;
    }
    for (; s < stop; ++s) {
      u32x4v a[4];
      to_bf16(down.code(s), down.scale(s), a);
      int at = 128 * s + 32 * q;
      const bool in = at < K;
      if (at >= p.I) at -= p.k_tail;                 // the tail meets the last values again
#pragma unroll
      for (int g = 0; g < kG; ++g) {
        if (!(mine >> (16 * g) & 0xFFFF)) continue;
        u32x4v b[4] = {};
        if (h[g] && in) {
          const u32x4v* from = reinterpret_cast<const u32x4v*>(h[g] + at);
#pragma unroll
          for (int j = 0; j < 4; ++j) b[j] = from[j];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[g] = dev::mfma_bf16(a[j], b[j], acc[g]);
      }
    }
  }
  f32x4* sums = reinterpret_cast<f32x4*>(red);
#pragma unroll
  for (int g = 0; g < kG; ++g) sums[(wave * kG + g) * 64 + lane] = acc[g];
  __syncthreads();
  const int g = wave;                                // wave g: block g
  const int t = 16 * g + c;
  f32x4 y = 0.f;
  if (g < kG) {
#pragma unroll
    for (int w = 0; w < kWaves; ++w) y += sums[(w * kG + g) * 64 + lane];
  }
  const bool here = g < kG && t < p.M;
  const int64_t at = static_cast<int64_t>(t) * p.N + 16 * tile + 4 * q;
  if (splits > 1) {
    const int64_t all = static_cast<int64_t>(p.M) * p.N;
    if (here) {
      // device scope: the last workgroup may be on another XCD with an L2 of its own
      for (int i = 0; i < 4; i += 2)
        __hip_atomic_store(reinterpret_cast<uint64_t*>(parts + part * all + at + i),
                           static_cast<uint64_t>(__float_as_uint(y[i + 1])) << 32 | __float_as_uint(y[i]),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // what this wave has stored is there
    __syncthreads();
    if (tid == 0)
      sh_last = __hip_atomic_fetch_add(arrived + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                static_cast<uint32_t>(splits - 1);
    __syncthreads();
    if (!sh_last) return;
    if (tid == 0) __hip_atomic_store(arrived + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (here) {
      y = 0.f;
      for (int w = 0; w < splits; ++w)
        for (int i = 0; i < 4; i += 2) {
          const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(parts + w * all + at + i),
                                               __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          y[i] += __uint_as_float(static_cast<uint32_t>(v));
          y[i + 1] += __uint_as_float(static_cast<uint32_t>(v >> 32));
        }
    }
  }
  if (here) {
    const dev::u32x2 v = {dev::pack_bf16(y[0], y[1]), dev::pack_bf16(y[2], y[3])};
    *reinterpret_cast<dev::u32x2*>(p.out + t * p.ld_out + 16 * tile + 4 * q) = v;
  }
}

size_t hidden_bytes(const MoeArgs& p) { return (static_cast<size_t>(p.M) * p.k * p.I * 2 + 255) & ~size_t{255}; }

}  // namespace

MoePlan plan_moe_layer(const MoeArgs& p, int num_cus) {
  MoePlan c;
  c.slots = std::min(p.E, p.M * p.k);
  const int64_t units = static_cast<int64_t>(c.slots) * ((p.I + p.k_tail + 127) / 128);
  while (c.splits < 8 && static_cast<int64_t>(p.N / 16) * c.splits < 2 * num_cus && units >= 2 * c.splits * kWaves * 4)
    c.splits *= 2;
  return c;
}

size_t moe_workspace_bytes(const MoePlan& c, const MoeArgs& p) {
  return kWorkspaceStateBytes + hidden_bytes(p) +
         (c.splits > 1 ? static_cast<size_t>(c.splits) * p.M * p.N * 4 : 0);
}

hipError_t launch_moe_layer(const MoePlan& c, const MoeArgs& p, void* workspace, hipStream_t stream) {
  char* at = static_cast<char*>(workspace);
  uint32_t* arrived = reinterpret_cast<uint32_t*>(at);
  uint16_t* hidden = reinterpret_cast<uint16_t*>(at + kWorkspaceStateBytes);
  float* parts = reinterpret_cast<float*>(at + kWorkspaceStateBytes + hidden_bytes(p));
  auto go = [&](auto blocks) {
    constexpr int kG = decltype(blocks)::value;
    const int lds = kWaves * 2 * kG * 64 * 16;
    if (lds > 32 * 1024) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&moe_up_kernel<kG>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (e != hipSuccess) return e;
    }
    moe_up_kernel<kG><<<dim3(p.I / 16, c.slots), kThreads, lds, stream>>>(p, hidden);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    moe_down_kernel<kG><<<dim3(p.N / 16, c.splits), kThreads, 0, stream>>>(p, hidden, parts, arrived);
    return hipGetLastError();
  };
  if (p.M <= 16) return go(std::integral_constant<int, 1>{});
  if (p.M <= 32) return go(std::integral_constant<int, 2>{});
  return go(std::integral_constant<int, 4>{});
}

}  // namespace prq
