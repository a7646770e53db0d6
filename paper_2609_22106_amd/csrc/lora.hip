// Low-rank adapters of many requests beside a shared projection: rows sorted by
// segment, segment s with the adapter of_s of rank r (or none),
//   out_row = Y_row + scale_a * B_a (A_a x_row),   A_a [r, K], B_a [N, r] bf16,
// Y and out float32 [M, N] (out may be Y), x bf16 [M, K].
//
// Two products with the rank between them, in two kernels: `down` forms
// t = A_a x over ranges of K (a workgroup per 16 rows of one segment and range, so
// that a few decoding rows still occupy the chip; partial sums in the workspace) and
// `up` adds them in order, scales and multiplies by B_a.  The bytes of Y and out bound
// long prompts; the adapters' own bytes and the two launches a decoding step.
//
// t stays float32: `up` splits each value into three bf16 terms (8 + 8 + 8 bits, the
// remainders exact), and three bf16 MFMAs add their products with B_a, so that the
// delta carries no rounding but those of the float32 sums.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;
using dev::u32x4v;

constexpr int kWaves = 4, kThreads = 64 * kWaves;

struct LoraArgs {
  const uint16_t* x;
  int64_t ld_x;
  const uint16_t *A, *B;
  const int32_t* rank_offsets;
  const float* scales;
  const int32_t *offsets, *of;
  const float* Y;
  float* out;
  int64_t ld_y, ld_out;
  float* t;                              // [splits][M][max_rank]
  int adapters, rank_rows, segments, M, N, K, max_rank, splits, k_per;
};

// The adapter of a segment: its first rank row and its rank, 0 where it has none (or
// where the tables name one that A and B do not hold).
struct Adapter {
  int index, first, rank;
};

__device__ __forceinline__ Adapter adapter_of(const LoraArgs& p, int segment) {
  Adapter a{p.of[segment], 0, 0};
  if (a.index < 0 || a.index >= p.adapters) return a;
  const int first = p.rank_offsets[a.index], end = p.rank_offsets[a.index + 1];
  if (first < 0 || end > p.rank_rows || end - first > p.max_rank || ((first | end) & 7)) return a;
  a.first = first;
  a.rank = end - first;
  return a;
}

// t of 16 rows over one range of K.  The waves take every fourth 32-element step, all
// ranks each, and are joined through LDS.
template <int kRankTiles>
__global__ __launch_bounds__(kThreads) void lora_down_kernel(const LoraArgs p) {
  __shared__ f32x4 sh[kWaves][kRankTiles][64];
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const dev::TileAt at = dev::find_tile(p.offsets, p.of, p.segments, p.M, static_cast<int>(blockIdx.y), 1, 16);
  if (at.segment < 0) return;
  const Adapter ad = adapter_of(p, at.segment);
  if (ad.rank <= 0) return;
  const int rows = min(at.rows - 16 * at.tile, 16);
  const int64_t row0 = at.first + 16 * at.tile;
  const int k0 = static_cast<int>(blockIdx.x) * p.k_per, k1 = min(k0 + p.k_per, p.K);
  // A operand: x's rows; B operand: the adapter's rank rows.  Rows and ranks past the
  // end read the last one and are not stored.
  const uint16_t* xp = p.x + (row0 + min(r, rows - 1)) * p.ld_x + 8 * g;
  const uint16_t* ap[kRankTiles];
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j)
    ap[j] = p.A + static_cast<int64_t>(ad.first + min(16 * j + r, ad.rank - 1)) * p.K + 8 * g;
  f32x4 acc[kRankTiles];
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j) acc[j] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int k = k0 + 32 * wave; k < k1; k += 32 * kWaves) {
    const u32x4v none = {0, 0, 0, 0};
    const bool in = k + 8 * g < k1;      // K % 8 == 0: a group of 8 is whole or absent
    const u32x4v xa = in ? *reinterpret_cast<const u32x4v*>(xp + k) : none;
#pragma unroll
    for (int j = 0; j < kRankTiles; ++j) {
      const u32x4v b = in ? *reinterpret_cast<const u32x4v*>(ap[j] + k) : none;
      acc[j] = dev::mfma_bf16(xa, b, acc[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < kRankTiles; ++j) sh[wave][j][lane] = acc[j];
  __syncthreads();
  // sh[.][j][16 g + c][i] is row 4 g + i, rank 16 j + c
  float* const t = p.t + (static_cast<int64_t>(blockIdx.x) * p.M + row0) * p.max_rank;
  for (int e = static_cast<int>(threadIdx.x); e < 256 * kRankTiles; e += kThreads) {
    const int rank = e % (16 * kRankTiles), row = e / (16 * kRankTiles);
    if (row < rows && rank < ad.rank) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum += sh[w][rank >> 4][16 * (row >> 2) + (rank & 15)][row & 3];
      t[row * p.max_rank + rank] = sum;
    }
  }
}

// x's three bf16 terms: x = a + b + c up to 2^-24 of x.  An infinity or a NaN is a's alone.
__device__ __forceinline__ void split3(float x, float (&part)[3]) {
  const float a = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
  const float rest = x - a;
  const float b = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u);
  const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
  part[0] = x != x ? x : a;
  part[1] = finite ? b : 0.f;
  part[2] = finite ? rest - b : 0.f;
}

// Y's rows of kRowTiles * 16 rows of one segment, columns of one slice: A operand
// B_a's rows (16 columns of Y), B operand t's rows, so that a lane holds 4
// neighbouring columns of one row.
template <int kSteps, int kRowTiles>
__global__ __launch_bounds__(kThreads) void lora_up_kernel(const LoraArgs p, int n_per) {
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const dev::TileAt at =
      dev::find_tile(p.offsets, p.of, p.segments, p.M, static_cast<int>(blockIdx.y), 1, 16 * kRowTiles);
  if (at.segment < 0) return;
  const Adapter ad = adapter_of(p, at.segment);
  const int rows = min(at.rows - 16 * kRowTiles * at.tile, 16 * kRowTiles);
  const int64_t row0 = at.first + 16 * kRowTiles * at.tile;
  const int n0 = static_cast<int>(blockIdx.x) * n_per, n1 = min(n0 + n_per, p.N);
  if (ad.rank <= 0 && p.out == p.Y) return;

  u32x4v t[kRowTiles][kSteps][3];
  const float scale = ad.rank > 0 ? p.scales[ad.index] : 0.f;
#pragma unroll
  for (int a = 0; a < kRowTiles; ++a) {
    const int64_t row = row0 + min(16 * a + r, rows - 1);
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
      if (32 * k + 8 * g < ad.rank) {    // ranks are multiples of 8
        for (int s = 0; s < p.splits; ++s) {
          const f32x4* tp = reinterpret_cast<const f32x4*>(p.t + (static_cast<int64_t>(s) * p.M + row) * p.max_rank +
                                                           32 * k + 8 * g);
          lo += tp[0];
          hi += tp[1];
        }
        lo *= scale;
        hi *= scale;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float one[3], two[3];
        split3(e < 2 ? lo[2 * e] : hi[2 * e - 4], one);
        split3(e < 2 ? lo[2 * e + 1] : hi[2 * e - 3], two);
#pragma unroll
        for (int w = 0; w < 3; ++w) t[a][k][w][e] = dev::pack_bf16(one[w], two[w]);
      }
    }
  }
  const uint16_t* const B = p.B + static_cast<int64_t>(p.N) * ad.first;
  for (int n = n0 + 16 * wave; n < n1; n += 16 * kWaves) {
    // N % 16 == 0: the tile's columns are all there
    f32x4 y[kRowTiles];
#pragma unroll
    for (int a = 0; a < kRowTiles; ++a) {
      const int64_t row = row0 + min(16 * a + r, rows - 1);
      y[a] = *reinterpret_cast<const f32x4*>(p.Y + row * p.ld_y + n + 4 * g);
    }
    u32x4v b[kSteps];
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      b[k] = u32x4v{0, 0, 0, 0};
      if (32 * k + 8 * g < ad.rank)
        b[k] = *reinterpret_cast<const u32x4v*>(B + static_cast<int64_t>(n + r) * ad.rank + 32 * k + 8 * g);
    }
    f32x4 acc[kRowTiles];
#pragma unroll
    for (int a = 0; a < kRowTiles; ++a) {
      acc[a] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 2; w >= 0; --w)       // the small terms first
#pragma unroll
        for (int k = 0; k < kSteps; ++k) acc[a] = dev::mfma_bf16(b[k], t[a][k][w], acc[a]);
    }
#pragma unroll
    for (int a = 0; a < kRowTiles; ++a)
      if (16 * a + r < rows)
        *reinterpret_cast<f32x4*>(p.out + (row0 + 16 * a + r) * p.ld_out + n + 4 * g) = y[a] + acc[a];
  }
}

template <int kRankTiles>
void launch_down(const LoraArgs& p, int64_t tiles, hipStream_t stream) {
  lora_down_kernel<kRankTiles><<<dim3(p.splits, static_cast<unsigned>(tiles)), kThreads, 0, stream>>>(p);
}

template <int kSteps, int kRowTiles>
void launch_up(const LoraArgs& p, int64_t tiles, int n_per, hipStream_t stream) {
  lora_up_kernel<kSteps, kRowTiles>
      <<<dim3((p.N + n_per - 1) / n_per, static_cast<unsigned>(tiles)), kThreads, 0, stream>>>(p, n_per);
}

}  // namespace

LoraPlan plan_lora(int M, int segments, int N, int K, int max_rank, int num_cus) {
  LoraPlan c;
  c.tiles = most_tiles(M, segments, 1, 16);
  const int steps = (K + 31) / 32;
  const int64_t want = (2 * static_cast<int64_t>(num_cus) + c.tiles - 1) / c.tiles;
  const int most = std::max(1, steps / 16);            // at least four steps a wave
  int splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({want, most, 16})));
  c.k_per = (steps + splits - 1) / splits * 32;
  c.splits = (K + c.k_per - 1) / c.k_per;
  const int64_t mean = M / std::max(1, std::min(M, segments));
  c.row_tiles = mean >= 64 && max_rank <= 64 ? 4 : 1;
  c.up_tiles = most_tiles(M, segments, 1, 16 * c.row_tiles);
  const int64_t slices = std::max<int64_t>(1, (4 * static_cast<int64_t>(num_cus) + c.up_tiles - 1) / c.up_tiles);
  c.n_per = static_cast<int>((N + slices - 1) / slices + 16 * kWaves - 1) / (16 * kWaves) * (16 * kWaves);
  return c;
}

size_t lora_workspace_bytes(const LoraPlan& c, int M, int max_rank) {
  return static_cast<size_t>(c.splits) * M * max_rank * 4;
}

hipError_t launch_lora(const LoraPlan& c, const uint16_t* x, int64_t ld_x, int M, int K, const uint16_t* A,
                       const uint16_t* B, const int32_t* rank_offsets, const float* scales, int adapters,
                       int rank_rows, int max_rank, const int32_t* offsets, const int32_t* of, int segments, int N, const float* Y,
                       int64_t ld_y, float* out, int64_t ld_out, void* workspace, hipStream_t stream) {
  const LoraArgs p{x, ld_x, A, B, rank_offsets, scales, offsets, of, Y, out, ld_y, ld_out,
                   static_cast<float*>(workspace), adapters, rank_rows, segments, M, N, K, max_rank, c.splits, c.k_per};
  if (max_rank <= 16) launch_down<1>(p, c.tiles, stream);
  else if (max_rank <= 32) launch_down<2>(p, c.tiles, stream);
  else if (max_rank <= 64) launch_down<4>(p, c.tiles, stream);
  else if (max_rank <= 128) launch_down<8>(p, c.tiles, stream);
  else launch_down<16>(p, c.tiles, stream);
  if (c.row_tiles == 4) {
    if (max_rank <= 32) launch_up<1, 4>(p, c.up_tiles, c.n_per, stream);
    else launch_up<2, 4>(p, c.up_tiles, c.n_per, stream);
  } else {
    if (max_rank <= 32) launch_up<1, 1>(p, c.up_tiles, c.n_per, stream);
    else if (max_rank <= 64) launch_up<2, 1>(p, c.up_tiles, c.n_per, stream);
    else if (max_rank <= 128) launch_up<4, 1>(p, c.up_tiles, c.n_per, stream);
    else launch_up<8, 1>(p, c.up_tiles, c.n_per, stream);
  }
  return hipGetLastError();
}

}  // namespace prq
