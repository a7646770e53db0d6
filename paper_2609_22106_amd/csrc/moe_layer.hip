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
// value times a power of two is exact there).  A wave asks for four K steps of its weights and
// the activations that meet them at once; enough waves a CU keep the memory busy meanwhile.
//
// A slot is an expert (its number), or where there are fewer pairs of a token and an expert than
// experts a pair (its first occurrence), so that a launch of `slots` workgroups in y reaches every
// expert that is named.  An expert's tokens are gathered into columns in ascending order, 16 to a
// block.  The first launch finds them with a lane a token, and leaves the second a table.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;
using dev::u32x4v;

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kSteps = 2;                            // K steps of 128 in a wave's unit

// What the first launch leaves: of every slot the number of its tokens (0: none, or the expert is
// another slot's), its expert, and for column i the row of `hidden` times 64 plus the token, -1 past
// the last.
struct Table {
  int32_t* counts;
  int32_t* experts;
  int32_t* columns;                                  // [slots][64]
};

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

// kSteps steps of a packed weight's tile of 16 rows, from a multiple of kSteps on: their kilobytes
// (the last one's again past the end, for which the activations are zeros) and the dword of their
// scales.
struct Unit {
  u32x4v codes[kSteps];
  uint32_t scales;
  __device__ __forceinline__ void load(const uint8_t* Wp, const uint8_t* Wps, int64_t tile, int steps, int unit) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    const u32x4v* from = reinterpret_cast<const u32x4v*>(Wp) + tile * steps * 64 + lane;
    scales = reinterpret_cast<const uint32_t*>(Wps)[(tile * ((steps + 3) >> 2) + (kSteps * unit >> 2)) * 64 + lane] >>
             (8 * (kSteps * unit & 3));
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      codes[i] = __builtin_nontemporal_load(from + min(kSteps * unit + i, steps - 1) * 64);
  }
};

// The columns' activations of a unit: lane (c, q) gets elements 32 q .. 32 q + 31 of each step, zeros
// for a column without a token (row null).  whole: a row's elements; K: the weight's, of which those
// past `whole` meet the row's last ones again, and zeros are behind.
__device__ __forceinline__ void load_columns(const uint16_t* row, int unit, int whole, int K, u32x4v (&b)[kSteps][4]) {
  const int q = (static_cast<int>(threadIdx.x) >> 4) & 3;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int k = 128 * (kSteps * unit + i) + 32 * q;
    const bool in = row && k < K;
    const u32x4v* from = reinterpret_cast<const u32x4v*>(row + (k < whole ? k : k - (K - whole)));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      b[i][j] = 0u;
      if (in) b[i][j] = from[j];
    }
  }
}

// A lane's token's share of expert e: whether it has one, the first of its k ids that names it, and
// the sum of the weights that do.
struct Share {
  bool has = false;
  int first = 0;
  float weight = 0.f;
  __device__ __forceinline__ Share(const MoeArgs& p, int e) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    if (lane >= p.M) return;
    const int32_t* ids = p.ids + lane * p.k;
    for (int j0 = 0; j0 < p.k; j0 += 8) {
      int id[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) id[j] = j0 + j < p.k ? ids[j0 + j] : -1;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (id[j] == e) {                            // (e >= 0)
          weight += p.weights[lane * p.k + j0 + j];
          if (!has) first = j0 + j;
          has = true;
        }
    }
  }
};

// First launch: a wave has 16 intermediate features of one expert (a gate tile and an up tile) for
// all of its tokens, and of the steps of H every kS-th unit.
template <int kS>
__global__ __launch_bounds__(kThreads, 4) void moe_up_kernel(const MoeArgs p, bool by_expert,
                                                              uint16_t* __restrict__ hidden, const Table table) {
  constexpr int kTiles = kWaves / kS;
  __shared__ f32x4 sums[kS > 1 ? kWaves * 2 * 64 : 1];
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int slot = static_cast<int>(blockIdx.y);
  const int tile = static_cast<int>(blockIdx.x) * kTiles + wave / kS, part = wave % kS;
  const int steps = (p.H + 127) >> 7, tiles = p.I >> 4, units = (steps + kSteps - 1) / kSteps;

  const int e = by_expert ? slot : p.ids[slot];
  const bool reached = e >= 0 && e < p.E;
  const Share share(p, reached ? e : -2);
  const uint64_t mine = __ballot(share.has);
  int n = __popcll(mine);
  if (!by_expert) {                                  // an earlier pair of the same expert has it
    const int token = slot / p.k;
    if (__ballot(share.has && (lane < token || (lane == token && lane * p.k + share.first < slot)))) n = 0;
  }
  // Column i: the i-th token.  Lanes without a share go behind the others.
  const uint64_t below = (uint64_t{1} << lane) - 1;
  const int at = share.has ? __popcll(mine & below) : __popcll(mine) + __popcll(~mine & below);
  const int row = share.has ? lane * p.k + share.first : -1;
  const int entry = share.has ? row * 64 + lane : -1;
  const int column = __builtin_amdgcn_ds_permute(4 * at, entry);
  if (blockIdx.x == 0 && wave == 0) {
    if (lane == 0) {
      table.counts[slot] = n;
      table.experts[slot] = e;
    }
    table.columns[slot * 64 + lane] = column;
  }
  if (n == 0) return;                                // the whole workgroup
  const float weight = __int_as_float(__builtin_amdgcn_ds_permute(4 * at, __float_as_int(share.weight)));

  const int64_t first = static_cast<int64_t>(e) * 2 * tiles + tile;
  for (int g = 0; 16 * g < n; ++g) {                 // (more than 16 tokens: the weights come from L2 again)
    const int col = __shfl(column, 16 * g + c, 64);
    f32x4 z = 0.f, y = 0.f;
    if (tile < tiles) {
      const uint16_t* x = col < 0 ? nullptr : p.x + (col & 63) * p.ld_x;
      for (int u = part; u < units; u += kS) {
        Unit gate, up;
        gate.load(p.up_codes, p.up_scales, first, steps, u);
        up.load(p.up_codes, p.up_scales, first + tiles, steps, u);
        u32x4v b[kSteps][4];
        load_columns(x, u, p.H, p.H, b);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          u32x4v a[4];
          to_bf16(gate.codes[i], gate.scales >> (8 * i) & 255u, a);
#pragma unroll
          for (int j = 0; j < 4; ++j) z = dev::mfma_bf16(a[j], b[i][j], z);
          to_bf16(up.codes[i], up.scales >> (8 * i) & 255u, a);
#pragma unroll
          for (int j = 0; j < 4; ++j) y = dev::mfma_bf16(a[j], b[i][j], y);
        }
      }
    }
    if constexpr (kS > 1) {
      if (g) __syncthreads();
      sums[(wave * 2) * 64 + lane] = z;
      sums[(wave * 2 + 1) * 64 + lane] = y;
      __syncthreads();
      if (part) continue;
#pragma unroll
      for (int w = 1; w < kS; ++w) {
        z += sums[((wave + w) * 2) * 64 + lane];
        y += sums[((wave + w) * 2 + 1) * 64 + lane];
      }
    }
    // column c's features 4 q .. 4 q + 3 of the tile
    const float w = __shfl(weight, 16 * g + c, 64);
    if (col >= 0 && tile < tiles) {
      float h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = z[i] / (1.f + expf(-z[i])) * y[i] * w;
      const dev::u32x2 v = {dev::pack_bf16(h[0], h[1]), dev::pack_bf16(h[2], h[3])};
      *reinterpret_cast<dev::u32x2*>(hidden + static_cast<int64_t>(col >> 6) * p.I + 16 * tile + 4 * q) = v;
    }
  }
}

// Second launch: 16 output features of all tokens.  The units of the experts that are reached are
// dealt evenly, in order, to the waves of the tile's workgroups.  A unit's columns are its expert's
// tokens; their sums are added to the tokens' in LDS, of which each wave has its own.  The waves'
// sums are added in their order, the workgroups' in theirs, by the one that arrives last.
__global__ __launch_bounds__(kThreads, 4) void moe_down_kernel(const MoeArgs p, const uint16_t* __restrict__ hidden,
                                                                const Table table, int slots, float* parts,
                                                                uint32_t* arrived) {
  extern __shared__ __align__(16) float own[];       // [kWaves][M][16]
  __shared__ int sh_last;
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int tile = static_cast<int>(blockIdx.x), splits = static_cast<int>(gridDim.y), part = static_cast<int>(blockIdx.y);
  const int K = p.I + p.k_tail, steps = (K + 127) >> 7, units = (steps + kSteps - 1) / kSteps;
  f32x4* mine = reinterpret_cast<f32x4*>(own) + wave * p.M * 4;
  for (int i = lane; i < p.M * 4; i += 64) mine[i] = 0.f;
  dev::wave_lds_barrier();

  // The slots with tokens, 64 at a time.
  auto there = [&](int base) { return __ballot(base + lane < slots && table.counts[min(base + lane, slots - 1)] > 0); };
  int n = 0;
  for (int base = 0; base < slots; base += 64) n += __popcll(there(base));
  const int64_t all = static_cast<int64_t>(n) * units;
  const int shares = splits * kWaves, share = part * kWaves + wave;
  int u = static_cast<int>(all * share / shares);
  const int end = static_cast<int>(all * (share + 1) / shares);

  if (u < end) {
    int skip = u / units, base = 0;
    uint64_t left = there(0);
    for (; __popcll(left) <= skip; left = there(base)) skip -= __popcll(left), base += 64;
    for (; skip; --skip) left &= left - 1;
    while (true) {
      const int slot = base + __builtin_ctzll(left);
      const int e = table.experts[slot];
      const int64_t first = static_cast<int64_t>(e) * (p.N >> 4) + tile;
      const int column = table.columns[slot * 64 + lane];
      const int blocks = (table.counts[slot] + 15) >> 4;
      const int stop = min(u / units * units + units, end);
      for (; u < stop; ++u) {
        Unit down;
        down.load(p.down_codes, p.down_scales, first, steps, u % units);
        for (int g = 0; g < blocks; ++g) {
          const int col = __shfl(column, 16 * g + c, 64);
          u32x4v b[kSteps][4];
          load_columns(col < 0 ? nullptr : hidden + static_cast<int64_t>(col >> 6) * p.I, u % units, p.I, K, b);
          f32x4 acc = 0.f;
#pragma unroll
          for (int i = 0; i < kSteps; ++i) {
            u32x4v a[4];
            to_bf16(down.codes[i], down.scales >> (8 * i) & 255u, a);
#pragma unroll
            for (int j = 0; j < 4; ++j) acc = dev::mfma_bf16(a[j], b[i][j], acc);
          }
          if (col >= 0) mine[(col & 63) * 4 + q] += acc;
          dev::wave_lds_barrier();
        }
      }
      if (u >= end) break;
      left &= left - 1;
      while (!left) base += 64, left = there(base);
    }
  }
  __syncthreads();
  // Thread (t, i): token t's features 4 i .. 4 i + 3.
  const int t = tid >> 2, i = tid & 3;
  const bool here = t < p.M;
  const f32x4* sums = reinterpret_cast<const f32x4*>(own);
  f32x4 y = 0.f;
  if (here) {
#pragma unroll
    for (int w = 0; w < kWaves; ++w) y += sums[(w * p.M + t) * 4 + i];
  }
  const int64_t at = static_cast<int64_t>(t) * p.N + 16 * tile + 4 * i;
  if (splits > 1) {
    const int64_t stride = static_cast<int64_t>(p.M) * p.N;
    if (here) {
      // device scope: the last workgroup may be on another XCD with an L2 of its own
#pragma unroll
      for (int j = 0; j < 4; j += 2)
        __hip_atomic_store(reinterpret_cast<uint64_t*>(parts + part * stride + at + j),
                           static_cast<uint64_t>(__float_as_uint(y[j + 1])) << 32 | __float_as_uint(y[j]),
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
      for (int w = 0; w < splits; ++w) {
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(parts + w * stride + at + j),
                                               __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          y[j] += __uint_as_float(static_cast<uint32_t>(v));
          y[j + 1] += __uint_as_float(static_cast<uint32_t>(v >> 32));
        }
      }
    }
  }
  if (here) {
    const dev::u32x2 v = {dev::pack_bf16(y[0], y[1]), dev::pack_bf16(y[2], y[3])};
    *reinterpret_cast<dev::u32x2*>(p.out + t * p.ld_out + 16 * tile + 4 * i) = v;
  }
}

size_t up16(size_t n) { return (n + 15) & ~size_t{15}; }
size_t hidden_bytes(const MoeArgs& p) { return up16(static_cast<size_t>(p.M) * p.k * p.I * 2); }
size_t table_bytes(const MoePlan& c) { return up16(static_cast<size_t>(c.slots) * 4 * (2 + 64)); }

}  // namespace

MoePlan plan_moe_layer(const MoeArgs& p, int num_cus) {
  MoePlan c;
  c.slots = std::min(p.E, p.M * p.k);
  c.by_expert = c.slots == p.E;
  // The first launch: 16 waves a CU, by parts of H where the tiles are fewer.
  const int64_t tiles = static_cast<int64_t>(p.I / 16) * c.slots;
  const int up_units = (p.H + 128 * kSteps - 1) / (128 * kSteps);
  while (c.parts < kWaves && c.parts < up_units && tiles * c.parts < 16 * num_cus) c.parts *= 2;
  const int64_t units = static_cast<int64_t>(c.slots) * ((p.I + p.k_tail + 128 * kSteps - 1) / (128 * kSteps));
  while (c.splits < 8 && static_cast<int64_t>(p.N / 16) * c.splits < 2 * num_cus && units >= 4 * c.splits * kWaves)
    c.splits *= 2;
  return c;
}

size_t moe_workspace_bytes(const MoePlan& c, const MoeArgs& p) {
  return kWorkspaceStateBytes + hidden_bytes(p) + table_bytes(c) +
         (c.splits > 1 ? static_cast<size_t>(c.splits) * p.M * p.N * 4 : 0);
}

hipError_t launch_moe_layer(const MoePlan& c, const MoeArgs& p, void* workspace, hipStream_t stream) {
  char* at = static_cast<char*>(workspace);
  uint32_t* arrived = reinterpret_cast<uint32_t*>(at);
  uint16_t* hidden = reinterpret_cast<uint16_t*>(at += kWorkspaceStateBytes);
  int32_t* const ints = reinterpret_cast<int32_t*>(at += hidden_bytes(p));
  const Table table{ints, ints + c.slots, ints + 2 * c.slots};
  float* parts = reinterpret_cast<float*>(at += table_bytes(c));
  auto up = [&](auto shared) {
    constexpr int kS = decltype(shared)::value, kTiles = kWaves / kS;
    moe_up_kernel<kS><<<dim3((p.I / 16 + kTiles - 1) / kTiles, c.slots), kThreads, 0, stream>>>(p, c.by_expert, hidden,
                                                                                                 table);
  };
  if (c.parts == 1) up(std::integral_constant<int, 1>{});
  else if (c.parts == 2) up(std::integral_constant<int, 2>{});
  else if (c.parts == 4) up(std::integral_constant<int, 4>{});
  else up(std::integral_constant<int, 8>{});
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  moe_down_kernel<<<dim3(p.N / 16, c.splits), kThreads, kWaves * p.M * 16 * 4, stream>>>(p, hidden, table, c.slots,
                                                                                         parts, arrived);
  return hipGetLastError();
}

}  // namespace prq
