// The router of a mixture-of-experts layer: every token's scores, the experts it goes to and
// their weights, in one launch.
//
//   l = x W^T                                     x [M, H], W [E, H] bf16, float32 sums
//   s = softmax(l)  or  1 / (1 + exp(-l))
//   the k experts with the largest s (or s + bias), descending, the lower index first among
//   equals, NaN behind everything
//   w = s (or s divided by the sum of the chosen, for which a softmax needs the chosen logits only)
//     times `scale`
// Both scores keep the order of l, so without a bias l itself is compared.  A bias moves borders: its
// key, and the sigmoid's weights, are computed in 64 bits.
//
// The product is MFMA work with experts as rows and tokens as columns; the operands' rows are loaded
// whole and brought into operand order through LDS (loaded in operand order, 16 rows at once, a load
// takes four times as long: 8192 tokens of 128 experts 53 us).  Few tokens: a workgroup has 16 of them
// and 16 experts, and its waves share H, so that W is read by as many CUs as possible.  The last
// one of a block of tokens to arrive reads the block's logits back.  Many: a workgroup has 32 tokens and
// all experts, in two stages of LDS, or of many experts a group of 128.  Choosing, a token has 16 lanes (or a
// wave).
//
// Bounds.  One token of 128 experts, H = 2048, 6.6 us: launch 2, one trip to memory and the product 2,
// arrival 1, choosing 1.5.  8192 of them 16.5 us: their bytes are 6.4, but one workgroup a CU loads 640 KB in
// 16 chunks at 0.5 to 0.6 us (16 to 20 TB/s over the card, most of it W from L2; LDS is active a third of
// the time, deeper rings change nothing), behind a launch of 3 and in front of 3 of choosing.  1537 tokens of
// 250 experts, H = 1024, 19.6 us: the same on 49 CUs with two groups of experts.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;
using dev::u32x4v;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
// Experts past which a block's logits do not fit beside the stages of route_many_kernel (512: 158 of 160 KB).
constexpr int kMaxManyExperts = 512;

// Unsigned integers in the order of the numbers, above 0, NaN below everything; and back.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);           // -0 is 0
  return x != x ? 1u : u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float number(uint32_t u) {
  return u == 1u ? __builtin_nanf("") : __uint_as_float(u ^ (u >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t u = __double_as_longlong(x + 0.0);
  return x != x ? 1u : u ^ (u >> 63 ? ~uint64_t{0} : uint64_t{1} << 63);
}

__device__ __forceinline__ double sigmoid64(float l) { return 1.0 / (1.0 + exp(-static_cast<double>(l))); }

// fold(both) for the exchanges after which every lane of a group of kLanes has met every other: each
// neighbour, pair, quad and octet, then each 16 and 32.  both(x): x of the two lanes that meet, in one
// order or the other.
template <int kLanes, typename Fold>
__device__ __forceinline__ void over_group(Fold fold) {
  struct Both {
    uint32_t a, b;
  };
  auto by = [](auto ctrl) {
    return [](uint32_t x) {
      return Both{x, static_cast<uint32_t>(
                         __builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(ctrl)::value, 0xF, 0xF, false))};
    };
  };
  fold(by(std::integral_constant<int, 0xB1>{}));         // quad_perm 1 0 3 2
  fold(by(std::integral_constant<int, 0x4E>{}));         // quad_perm 2 3 0 1
  fold(by(std::integral_constant<int, 0x141>{}));        // row_half_mirror
  fold(by(std::integral_constant<int, 0x140>{}));        // row_mirror
  if constexpr (kLanes == 64) {                          // (an exchange through LDS takes a hundred cycles)
    fold([](uint32_t x) {
      const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
      return Both{r[0], r[1]};
    });
    fold([](uint32_t x) {
      const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
      return Both{r[0], r[1]};
    });
  }
}
template <int kLanes>
__device__ __forceinline__ float group_sum(float x) {
  over_group<kLanes>([&](auto both) {
    const auto v = both(__float_as_uint(x));
    x = __uint_as_float(v.a) + __uint_as_float(v.b);
  });
  return x;
}
template <int kLanes>
__device__ __forceinline__ double group_sum(double x) {
  over_group<kLanes>([&](auto both) {
    const uint64_t u = __double_as_longlong(x);
    const auto high = both(static_cast<uint32_t>(u >> 32)), low = both(static_cast<uint32_t>(u));
    x = __longlong_as_double(static_cast<uint64_t>(high.a) << 32 | low.a) +
        __longlong_as_double(static_cast<uint64_t>(high.b) << 32 | low.b);
  });
  return x;
}

template <int kLanes>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  over_group<kLanes>([&](auto both) {
    const auto v = both(x);
    x = max(v.a, v.b);
  });
  return x;
}

// A token by a group of kLanes lanes, of which lane i has experts kR i .. kR i + kR - 1 and keeps choices
// i, kLanes + i, ...  live: the group has a token.  logit(e): expert e's.  A choice is the largest key
// (of two words, with a bias) and the lowest index that has it: steps of 32 bits, since a
// comparison of 64 takes four times as long.
template <int kLanes, int kR, bool kBias, typename Logit>
__device__ __forceinline__ void choose(const RouteArgs& p, int token, bool live, Logit logit) {
  constexpr int kKept = (kMaxRouteTop + kLanes - 1) / kLanes;
  const int mine = static_cast<int>(threadIdx.x) % kLanes;
  float l[kR];
#pragma unroll
  for (int i = 0; i < kR; ++i) l[i] = live && mine * kR + i < p.E ? logit(mine * kR + i) : -__builtin_inff();
  uint32_t key[kR], low[kBias ? kR : 1];         // 0: no expert
#pragma unroll
  for (int i = 0; i < kR; ++i) {
    const int e = mine * kR + i;
    const bool in = live && e < p.E;
    if (in && p.logits) p.logits[token * p.ld_logits + e] = l[i];
    if constexpr (kBias) {
      const uint64_t both = in ? ordered(sigmoid64(l[i]) + static_cast<double>(p.bias[e])) : 0;
      key[i] = static_cast<uint32_t>(both >> 32);
      low[i] = static_cast<uint32_t>(both);
    } else {
      key[i] = in ? ordered(l[i]) : 0;
    }
  }
  int ids[kKept];
  float chosen[kKept], first = 0.f;
  for (int j = 0; j < p.k; ++j) {
    uint32_t most = key[0];
#pragma unroll
    for (int i = 1; i < kR; ++i) most = max(most, key[i]);
    most = group_max<kLanes>(most);
    uint32_t most_low = 0;
    if constexpr (kBias) {
#pragma unroll
      for (int i = 0; i < kR; ++i) most_low = max(most_low, key[i] == most ? low[i] : 0u);
      most_low = group_max<kLanes>(most_low);
    }
    uint32_t above = 0;                          // ~ the lowest index
#pragma unroll
    for (int i = kR - 1; i >= 0; --i)
      if (key[i] == most && (!kBias || low[i] == most_low)) above = ~static_cast<uint32_t>(mine * kR + i);
    const int e = static_cast<int>(~group_max<kLanes>(above));
    float of_e = 0.f;
    if constexpr (kBias) {
      uint32_t u = 0;
#pragma unroll
      for (int i = 0; i < kR; ++i)
        if (e == mine * kR + i) u = ordered(l[i]);
      of_e = number(group_max<kLanes>(u));
    } else {
      of_e = number(most);
    }
#pragma unroll
    for (int i = 0; i < kR; ++i)
      if (e == mine * kR + i) {
        key[i] = 0;
        if constexpr (kBias) low[i] = 0;
      }
    if (j == 0) first = of_e;
#pragma unroll
    for (int i = 0; i < kKept; ++i)
      if (j == mine + i * kLanes) ids[i] = e, chosen[i] = of_e;
  }
  auto kept = [&](int i) { return mine + i * kLanes < p.k; };
  float w[kKept];
  if (p.sigmoid) {
    double s[kKept], total = 0.0;
#pragma unroll
    for (int i = 0; i < kKept; ++i) total += s[i] = kept(i) ? sigmoid64(chosen[i]) : 0.0;
    total = p.renormalize ? group_sum<kLanes>(total) : 1.0;
#pragma unroll
    for (int i = 0; i < kKept; ++i) w[i] = static_cast<float>(s[i] / total * p.scale);
  } else {
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < kKept; ++i) total += w[i] = kept(i) ? expf(chosen[i] - first) : 0.f;
    if (!p.renormalize) {
      float each[kR];
#pragma unroll
      for (int i = 0; i < kR; ++i) each[i] = mine * kR + i < p.E ? expf(l[i] - first) : 0.f;
#pragma unroll
      for (int n = kR / 2; n; n /= 2)            // in pairs: five roundings of a lane's 32
#pragma unroll
        for (int i = 0; i < n; ++i) each[i] += each[i + n];
      total = each[0];
    }
    total = group_sum<kLanes>(total);
#pragma unroll
    for (int i = 0; i < kKept; ++i) w[i] = w[i] / total * p.scale;
  }
#pragma unroll
  for (int i = 0; i < kKept; ++i)
    if (live && kept(i)) {
      const int64_t at = static_cast<int64_t>(token) * p.k + mine + i * kLanes;
      p.ids[at] = ids[i];
      p.weights[at] = w[i];
    }
}

// choose with as many keys a lane as E takes, of a kernel that takes kMost experts at most.
template <int kLanes, int kR, int kMost, bool kBias, typename Logit>
__device__ __forceinline__ void choose_of(const RouteArgs& p, int token, bool live, Logit logit) {
  if constexpr (kLanes * kR >= kMost) {
    choose<kLanes, kR, kBias>(p, token, live, logit);
  } else {
    if (p.E <= kLanes * kR) choose<kLanes, kR, kBias>(p, token, live, logit);
    else choose_of<kLanes, 2 * kR, kMost, kBias>(p, token, live, logit);
  }
}

// Tokens token0 .. token0 + rows - 1 by the workgroup: 16 lanes each, or 64 where there are no more tokens
// than waves or more experts than 32 a lane.  us, 16 / 64 lanes (H = 2048): 512 experts 300 tokens 25.1 / 23.9, 1100
// 30.0 / 30.5, 2000 34.6 / 31.5, 8192 54.3 / 56.4; 300 experts (H = 1024) 8192 29.4 / 32.8.  logit(row, e).
template <bool kBias, int kMost, typename Logit>
__device__ __forceinline__ void choose_rows(const RouteArgs& p, int token0, int rows, Logit logit) {
  constexpr int kMostOf16 = 512;
  const int wave = static_cast<int>(threadIdx.x) >> 6;
  if ((kMost > kMostOf16 && p.E > kMostOf16) || rows <= kWaves) {
    for (int r = wave; r < rows; r += kWaves)
      choose_of<64, 2, kMost, kBias>(p, token0 + r, true, [&](int e) { return logit(r, e); });
  } else {
    for (int r0 = 4 * wave; r0 < rows; r0 += 4 * kWaves) {
      const int r = r0 + (static_cast<int>(threadIdx.x) >> 4 & 3);
      choose_of<16, 4, (kMost < kMostOf16 ? kMost : kMostOf16), kBias>(p, token0 + r, r < rows,
                                                                       [&](int e) { return logit(r, e); });
    }
  }
}

// A workgroup's logits (value(row, e) of its experts e0 .. e0 + experts - 1) to where the last one to
// arrive of a block finds them, and whether this is it: device-scope accesses, since that may be
// another XCD with an L2 of its own.
template <typename Value>
__device__ __forceinline__ bool arrive(const RouteArgs& p, float* parts, uint32_t* arrived, int row0, int rows, int e0,
                                       int experts, int groups, Value value) {
  __shared__ int sh_last;
  const int tid = static_cast<int>(threadIdx.x);
  for (int i = tid; i < rows * experts; i += kThreads) {
    const int r = i / experts, e = i % experts;
    if (e0 + e < p.E)
      __hip_atomic_store(parts + static_cast<int64_t>(row0 + r) * p.E + e0 + e, value(r, e), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // what this wave has stored is there
  __syncthreads();
  if (tid == 0)
    sh_last = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
              static_cast<uint32_t>(groups - 1);
  __syncthreads();
  if (!sh_last) return false;
  if (tid == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}
__device__ __forceinline__ float arrived_logit(const RouteArgs& p, const float* parts, int row, int e) {
  return __hip_atomic_load(parts + static_cast<int64_t>(row) * p.E + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Rows in LDS: 32 bytes past a multiple of 128, at which 16 rows' octets at one place meet different
// banks (16, 48 or 64 past it: twelve times the conflicts, 16.8 -> 17.6 us).
__host__ __device__ constexpr int pitch_of(int elements) { return 2 * elements + 32; }
// The two stages, or the parts' sums, of 32 tokens and 32 kE experts.
__host__ __device__ constexpr int stages_bytes(int kE) {
  const int rows = 2 * (32 + 32 * kE) * pitch_of(64 * kWaves / kE), sums = kWaves / kE * 32 * (32 * kE + 4) * 4;
  return rows > sums ? rows : sums;
}

// 16 tokens and 16 experts; the waves share H by steps of 128, each with LDS of its own.
template <bool kBias>
__global__ __launch_bounds__(kThreads) void route_few_kernel(const RouteArgs p, int first, float* parts, uint32_t* arrived) {
  constexpr int kPitch = pitch_of(128);
  __shared__ __align__(16) unsigned char rows[kWaves][32 * kPitch];
  __shared__ f32x4 sums[kWaves][64];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int c = lane & 15, q = lane >> 4;
  const int token0 = first + static_cast<int>(blockIdx.x) * 16, e0 = static_cast<int>(blockIdx.y) * 16;
  const int steps = (p.H + 127) >> 7, count = min(p.M - token0, 16);

  f32x4 acc = 0.f;
  u32x4v x[4], w[4];                             // rows 4 j + q, octet c
  auto ask = [&](int s) {
    const int k = 128 * s + 8 * c;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = w[j] = 0u;
      const int r = 4 * j + q;
      if (k < p.H) {
        if (r < count) x[j] = *reinterpret_cast<const u32x4v*>(p.x + (token0 + r) * p.ld_x + k);
        if (e0 + r < p.E) w[j] = *reinterpret_cast<const u32x4v*>(p.w + (e0 + r) * p.ld_w + k);
      }
    }
  };
  ask(wave);
  unsigned char* const mine = rows[wave];
  for (int s = wave; s < steps; s += kWaves) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      *reinterpret_cast<u32x4v*>(mine + (4 * j + q) * kPitch + 16 * c) = x[j];
      *reinterpret_cast<u32x4v*>(mine + (16 + 4 * j + q) * kPitch + 16 * c) = w[j];
    }
    dev::wave_lds_barrier();
    if (s + kWaves < steps) ask(s + kWaves);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32x4v b = *reinterpret_cast<const u32x4v*>(mine + c * kPitch + (4 * j + q) * 16);
      const u32x4v a = *reinterpret_cast<const u32x4v*>(mine + (16 + c) * kPitch + (4 * j + q) * 16);
      acc = dev::mfma_bf16(a, b, acc);
    }
    dev::wave_lds_barrier();
  }
  sums[wave][lane] = acc;
  __syncthreads();
  auto sum = [&](int r, int e) {                 // token r's, of expert e0 + e
    float l = 0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) l += sums[v][(e >> 2) * 16 + r][e & 3];
    return l;
  };
  if (gridDim.y == 1) return choose_rows<kBias, 16>(p, token0, count, sum);
  if (arrive(p, parts, arrived + blockIdx.x, token0 - first, count, e0, 16, static_cast<int>(gridDim.y), sum))
    choose_rows<kBias, kMaxRouteExperts>(p, token0, count, [&](int r, int e) {
      return arrived_logit(p, parts, token0 - first + r, e);
    });
}

// 32 tokens and all experts, 32 kE at a time (kSplit: the grid's 32 kE); wave (g, part) has 32 of those, all
// tokens and 64 elements of every chunk of H.  Chunks come by way of registers, kAhead of them under way,
// into two stages of LDS.
__host__ __device__ inline int logits_pitch(int E, int kE) { return (E + 32 * kE - 1) / (32 * kE) * 32 * kE + 4; }

template <int kE, bool kBias, bool kSplit>
__global__ __launch_bounds__(kThreads, 2) void route_many_kernel(const RouteArgs p, float* parts, uint32_t* arrived) {
  constexpr int kParts = kWaves / kE, kChunk = 64 * kParts, kPitch = pitch_of(kChunk);
  constexpr int kRows = 32 + 32 * kE, kOctets = kChunk / 8, kEach = kThreads / kOctets;      // rows a pass
  constexpr int kLoads = kRows / kEach, kAhead = kE == 4 ? 4 : kE == 2 ? 3 : 2;
  constexpr int kSums = 32 * kE + 4;             // floats between two tokens' sums
  extern __shared__ __align__(16) unsigned char smem[];      // [2][kRows][kPitch] or [kParts][32][kSums], and the logits
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int c = lane & 15, q = lane >> 4;
  const int token0 = static_cast<int>(blockIdx.x) * 32;
  const int count = min(p.M - token0, 32);
  float* const sums = reinterpret_cast<float*>(smem);
  float* const logits = reinterpret_cast<float*>(smem + stages_bytes(kE));
  const int pitch = logits_pitch(p.E, kE);

  const int octet = tid % kOctets, row = tid / kOctets;
  const int part = wave / kE, g = wave % kE;
  for (int e0 = kSplit ? static_cast<int>(blockIdx.y) * 32 * kE : 0; e0 < p.E; e0 += 32 * kE) {
    const uint16_t* from[kLoads];                // rows past the end: the last one's again, not stored
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = row + i * kEach;
      from[i] = (r < 32 ? p.x + min(token0 + r, p.M - 1) * p.ld_x : p.w + min(e0 + r - 32, p.E - 1) * p.ld_w) + 8 * octet;
    }
    u32x4v ring[kAhead][kLoads];
    // (loads without conditions, so that every wait counts exactly the loads behind it)
    auto ask = [&](int chunk, u32x4v (&to)[kLoads]) {      // chunk: its first element
      const int k = min(chunk, p.H - 8 - 8 * octet);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) to[i] = *reinterpret_cast<const u32x4v*>(from[i] + k);
    };
    auto put = [&](const u32x4v (&v)[kLoads], int chunk, int stage) {
      unsigned char* to = smem + stage * kRows * kPitch + row * kPitch + 16 * octet;
      const bool in = chunk + 8 * octet < p.H;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) *reinterpret_cast<u32x4v*>(to + i * kEach * kPitch) = in ? v[i] : u32x4v{};
    };
    f32x4 acc[2][2] = {};
    u32x4v a[2][2], b[2][2];
    auto read = [&](int stage) {
      const unsigned char* at = smem + stage * kRows * kPitch + c * kPitch + (part * 8 + q) * 16;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          b[s][m] = *reinterpret_cast<const u32x4v*>(at + 16 * m * kPitch + 64 * s);
          a[s][m] = *reinterpret_cast<const u32x4v*>(at + (32 + 32 * g + 16 * m) * kPitch + 64 * s);
        }
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ask(i * kChunk, ring[i]);
    __syncthreads();                             // the sums before have been read
    put(ring[0], 0, 0);
    ask(kAhead * kChunk, ring[0]);
    constexpr int kRound = kAhead % 2 ? 2 * kAhead : kAhead;
    for (int i0 = 0; i0 < p.H; i0 += kRound * kChunk) {      // (chunks past the end are zeros)
#pragma unroll
      for (int r = 0; r < kRound; ++r) {
        // A stage is written while the other is read: the next chunk's LDS writes overlap this one's reads.
        const int next = i0 + (r + 1) * kChunk;
        __syncthreads();
        read(r % 2);
        put(ring[(r + 1) % kAhead], next, (r + 1) % 2);
        ask(next + kAhead * kChunk, ring[(r + 1) % kAhead]);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int t = 0; t < 2; ++t) acc[m][t] = dev::mfma_bf16(a[s][m], b[s][t], acc[m][t]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        *reinterpret_cast<f32x4*>(sums + (part * 32 + 16 * t + c) * kSums + 32 * g + 16 * m + 4 * q) = acc[m][t];
    __syncthreads();
    if constexpr (kSplit) {
      auto sum = [&](int r, int e) {
        float l = sums[r * kSums + e];
#pragma unroll
        for (int v = 1; v < kParts; ++v) l += sums[(v * 32 + r) * kSums + e];
        return l;
      };
      if (!arrive(p, parts, arrived + blockIdx.x, token0, count, e0, 32 * kE, static_cast<int>(gridDim.y), sum)) return;
      break;
    }
    for (int i = tid; i < 32 * 8 * kE; i += kThreads) {
      const int r = i / (8 * kE), e = i % (8 * kE) * 4;
      f32x4 l = *reinterpret_cast<const f32x4*>(sums + r * kSums + e);
#pragma unroll
      for (int v = 1; v < kParts; ++v) l += *reinterpret_cast<const f32x4*>(sums + (v * 32 + r) * kSums + e);
      *reinterpret_cast<f32x4*>(logits + r * pitch + e0 + e) = l;
    }
  }
  __syncthreads();
  choose_rows<kBias, kE == 4 ? kMaxManyExperts : 32 * kE>(p, token0, count, [&](int r, int e) {
    return kSplit ? arrived_logit(p, parts, token0 + r, e) : logits[r * pitch + e];
  });
}

// Tokens in a launch of the other kernel: what the state's counters and a modest workspace hold.
constexpr int kMaxFewTokens = 8192;
static_assert(kMaxFewTokens / 16 <= static_cast<int>(kWorkspaceStateBytes / 4), "a counter a block");

}  // namespace

RoutePlan plan_moe_route(int M, int E, int H, int num_cus) {
  RoutePlan c;
  // A workgroup for 16 experts while there are no more than two a CU, or four past 128 experts, where the
  // other kernel's workgroups take two groups of them in turn.  us, this one / the other: 128 experts
  // (H = 2048) 600 tokens 12.1 / 15.1, 1024 12.9 / 15.1, 2000 23.3 / 15.2; 64 (2560) 1000 tokens 10.4 / 14.0,
  // 2048 13.0 / 14.4, 4000 22.9 / 13.2; 250 (1024) 700 tokens 16.3 / 18.6, 1000 20.4 / 18.9, 1537 27.6 / 18.9.
  const int64_t few = (static_cast<int64_t>(M) + 15) / 16 * ((E + 15) / 16);
  if (E > kMaxManyExperts || few <= (E > 128 ? 4 : 2) * num_cus) return c;
  c.groups = E > 64 ? 4 : E > 32 ? 2 : 1;
  // Three and four groups of a block go to workgroups of their own while those are at most two a CU, and
  // meet in the workspace.  us, 16 experts / groups apart / groups in turn (H = 2048): 512 experts 400 tokens
  // 27.4 / 27.9 / 51.9, 1100 50.7 / 30.2 / 52.0, 4096 130 / 44.7 / 52.2, 8192 257 / 72.5 / 54.4; 384 and a bias 600
  // tokens 38.9 / 41.2 / 54.9, 1000 50.7 / 40.6 / 55.2.  Two groups gain less than the room for all logits
  // is worth (250 experts, 4096 tokens 70.6 / 29.7 / 33.5).
  const int64_t apart = (static_cast<int64_t>(M) + 31) / 32 * ((E + 127) / 128);
  c.split = E > 256 && apart <= 2 * num_cus;
  return c;
}

size_t route_workspace_bytes(const RoutePlan& c, int M, int E) {
  if (c.groups ? !c.split : E <= 16) return 0;
  return kWorkspaceStateBytes + static_cast<size_t>(c.split ? M : std::min(M, kMaxFewTokens)) * E * 4;
}

hipError_t launch_moe_route(const RoutePlan& c, const RouteArgs& p, void* workspace, hipStream_t stream) {
  uint32_t* const arrived = static_cast<uint32_t*>(workspace);
  float* const parts = workspace ? reinterpret_cast<float*>(arrived + kWorkspaceStateBytes / 4) : nullptr;
  auto many = [&](auto kernel, int kE) {
    const int lds = stages_bytes(kE) + (c.split ? 0 : 32 * logits_pitch(p.E, kE) * 4);
    const int apart = c.split ? (p.E + 32 * kE - 1) / (32 * kE) : 1;
    kernel<<<dim3((p.M + 31) / 32, apart), kThreads, lds, stream>>>(p, parts, arrived);
    return hipGetLastError();
  };
  auto go = [&](auto bias) {
    constexpr bool kBias = decltype(bias)::value;
    if (c.split) return many(LargeLds<&route_many_kernel<4, kBias, true>>::kernel(), 4);
    if (c.groups == 4) return many(LargeLds<&route_many_kernel<4, kBias, false>>::kernel(), 4);
    if (c.groups == 2) return many(LargeLds<&route_many_kernel<2, kBias, false>>::kernel(), 2);
    if (c.groups == 1) return many(LargeLds<&route_many_kernel<1, kBias, false>>::kernel(), 1);
    const int tiles = (p.E + 15) / 16, most = tiles > 1 ? kMaxFewTokens : p.M;
    for (int first = 0; first < p.M; first += most) {
      route_few_kernel<kBias><<<dim3((std::min(p.M - first, most) + 15) / 16, tiles), kThreads, 0, stream>>>(
          p, first, parts, arrived);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  };
  return p.bias ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace prq
