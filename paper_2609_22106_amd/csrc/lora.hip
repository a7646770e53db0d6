// Low-rank adapters of many requests beside a shared projection: rows sorted by
// segment, segment s with the adapter of_s of rank r (or none),
//   out_row = Y_row + scale_a * B_a (A_a x_row),   A_a [r, K], B_a [N, r] bf16,
// Y and out float32 [M, N] (out may be Y), x bf16 [M, K].
//
// Two products with the rank between them, in two kernels: `down` forms
// t = A_a x over ranges of K (a workgroup per 16 or 32 rows of one segment, or of one
// adapter, and range, so that a few decoding rows still occupy the chip; partial sums in the
// workspace) and `up` adds them in order, scales and multiplies by B_a.  The bytes of Y and
// out bound long prompts; the adapters' own bytes and the two launches a decoding step.
//
// An operand's neighbouring lanes hold different rows, so operands loaded straight from
// rows in memory use 16 of the 64 bytes a clock of a CU's first cache: rows are loaded
// whole and pass through LDS instead (64 requests, ranks up to 64, K = 9728: `down` 13.3
// -> 8.4 us), and `up` of many rows lays its columns out so that 16 lanes load and store 256
// bytes of a row of Y (8192 rows x 9728 columns: 167 -> 126 us).
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

constexpr int kWaves = 4, kThreads = 64 * kWaves, kSmallWaves = 8;
constexpr int kMaxRanges = 8;            // of K

struct LoraArgs {
  const uint16_t* x;
  int64_t ld_x;
  const uint16_t *A, *B;
  const int32_t *rank_offsets, *ranks;
  const float* scales;
  const int32_t *offsets, *of;
  const float* Y;
  float* out;
  int64_t ld_y, ld_out;
  float* t;                              // [splits][M][max_rank]
  int adapters, rank_rows, segments, M, N, K, max_rank, splits, k_per;
};

// An adapter: its first rank row and its rank as A and B hold it, 0 where it has none (or
// where the tables name one that they do not hold), and how many of those ranks are its own.
// The others pad it: their t is 0 whatever x holds (0 x infinity is not).
struct Adapter {
  int index, first, rank, own;
};

__device__ __forceinline__ Adapter adapter_of(const LoraArgs& p, int index) {
  Adapter a{index, 0, 0, 0};
  if (a.index < 0 || a.index >= p.adapters) return a;
  const int first = p.rank_offsets[a.index], end = p.rank_offsets[a.index + 1];
  if (first < 0 || end > p.rank_rows || end - first > p.max_rank || ((first | end) & 7)) return a;
  a.own = p.ranks ? min(p.ranks[a.index], end - first) : end - first;
  if (a.own <= 0) return a;
  a.first = first;
  a.rank = end - first;
  return a;
}

// 16 rows that have an adapter (or none) in common.
struct Tile {
  int with, rows, mine;                  // its index; the rows; row lane % 16 of them (the last one past the end)
};

// Tile y of the launch: 16 neighbouring rows of one segment, or (kGrouped, M <= 64) of all rows
// with one adapter, wherever they are: lane i asks for row i, and the adapters are taken in the
// order of their first rows.  owner: 64 words of LDS of the wave's own.  false: there is none.
template <bool kGrouped>
__device__ __forceinline__ bool find_rows(const LoraArgs& p, int* owner, Tile* out) {
  const int lane = static_cast<int>(threadIdx.x) & 63;
  int t = static_cast<int>(blockIdx.y);
  if constexpr (!kGrouped) {
    const dev::TileAt at = dev::find_tile(p.offsets, p.of, p.segments, p.M, t, 1, 16);
    if (at.segment < 0) return false;
    const int rows = min(at.rows - 16 * at.tile, 16);
    *out = {at.with, rows, at.first + 16 * at.tile + min(lane & 15, rows - 1)};
    return true;
  }
  constexpr int kNobody = -2;
  owner[lane] = kNobody;
  dev::wave_lds_barrier();
  for (int base = 0; base < p.segments; base += 64) {
    const int s = base + lane;
    if (s < p.segments) {
      const int with = p.of[s], first = min(max(p.offsets[s], 0), p.M), end = min(max(p.offsets[s + 1], 0), p.M);
      for (int row = first; row < end; ++row) owner[row] = with >= 0 && with < p.adapters ? with : -1;
    }
  }
  dev::wave_lds_barrier();
  const int own = lane < p.M ? owner[lane] : kNobody;
  // The rows with the lane's adapter, bit by bit of its index; the first of them counts their tiles.
  uint64_t same = __ballot(own != kNobody);
  for (int b = 0; p.adapters >> b; ++b) {
    const bool bit = (own + 1) >> b & 1;
    const uint64_t set = __ballot(bit);
    same &= bit ? set : ~set;
  }
  const bool leads = own != kNobody && __builtin_ctzll(same) == lane;
  const int tiles = leads ? (__builtin_popcountll(same) + 15) / 16 : 0, sum = dev::prefix_sum(tiles);
  const uint64_t past = __ballot(sum > t);
  if (!past) return false;
  const int at = __builtin_ctzll(past);
  t -= __builtin_amdgcn_readlane(sum - tiles, at);
  const uint64_t rows = static_cast<uint64_t>(static_cast<uint32_t>(
                            __builtin_amdgcn_readlane(static_cast<int>(same >> 32), at))) << 32 |
                        static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(same), at));
  const int with = __builtin_amdgcn_readlane(own, at);
  const int n = min(__builtin_popcountll(rows) - 16 * t, 16);
  const int rank = __builtin_popcountll(rows & ((uint64_t{1} << lane) - 1)) - 16 * t;
  const bool in = (rows >> lane & 1) && rank >= 0 && rank < 16;
  const int sent = __builtin_amdgcn_ds_permute(4 * (in ? rank : 63), lane);     // lane 63's is not used
  *out = {with, n, __shfl(sent, min(lane & 15, n - 1))};
  return true;
}

// t of 16 kRowTiles rows over K's elements [k0, end), for up to 16 kTiles ranks from `rank0`
// on, by kN waves: emit(row, rank, value), by any thread.  The waves take every kN-th step
// of 64 elements.  A row's 128 bytes of a step are loaded by 8 neighbouring lanes -- an
// operand's own lanes, each on another row, would take the first cache four times as long
// -- and reach their operand's place through a part of LDS of the wave's own (unit u of row k
// at u ^ (k / 2 & 7): no conflicts).
template <int kRowTiles, int kTiles, int kN, typename RowAt, typename Emit>
__device__ __forceinline__ void down_rows(const LoraArgs& p, const Adapter& ad, RowAt row_at, int rows, int rank0,
                                          int k0, int end, u32x4v* sh, Emit emit) {
  constexpr int kLoads = 2 * (kRowTiles + kTiles);           // of 8 rows, a step
  // steps under way: the small kernel has the registers for all of K = 2560 at up to 32 ranks
  constexpr int kAtOnce = kN == kSmallWaves ? (kLoads <= 6 ? 5 : 3) : kLoads <= 6 ? 4 : 2;
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int lr = lane >> 3, unit = lane & 7;
  // rows and ranks past the end read the last one and are not used
  const uint16_t* src[kLoads];
#pragma unroll
  for (int i = 0; i < 2 * kRowTiles; ++i) src[i] = p.x + row_at(min(8 * i + lr, rows - 1)) * p.ld_x;
#pragma unroll
  for (int i = 0; i < 2 * kTiles; ++i)
    src[2 * kRowTiles + i] = p.A + static_cast<int64_t>(ad.first + min(rank0 + 8 * i + lr, ad.rank - 1)) * p.K;
  u32x4v* const mine = sh + wave * kLoads * 64;
  f32x4 acc[kRowTiles][kTiles];
#pragma unroll
  for (int a = 0; a < kRowTiles; ++a)
#pragma unroll
    for (int j = 0; j < kTiles; ++j) acc[a][j] = {0.f, 0.f, 0.f, 0.f};
  const u32x4v none = {0, 0, 0, 0};
  for (int k = k0 + 64 * wave; k < end; k += kAtOnce * 64 * kN) {
    u32x4v in[kAtOnce][kLoads];
#pragma unroll
    for (int s = 0; s < kAtOnce; ++s) {
      const int at = k + s * 64 * kN + 8 * unit;             // K % 8 == 0: a unit is whole or absent
      if (kN == kSmallWaves && s && k + s * 64 * kN >= end) break;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) in[s][i] = *reinterpret_cast<const u32x4v*>(src[i] + (at < end ? at : 0));
    }
#pragma unroll
    for (int s = 0; s < kAtOnce; ++s) {
      if (s && k + s * 64 * kN >= end) break;
      const bool here = k + s * 64 * kN + 8 * unit < end;
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        mine[(8 * i + lr) * 8 + (unit ^ ((8 * i + lr) >> 1 & 7))] = here ? in[s][i] : none;
      dev::wave_lds_barrier();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4v x[kRowTiles];
#pragma unroll
        for (int a = 0; a < kRowTiles; ++a) x[a] = mine[(16 * a + r) * 8 + ((4 * h + g) ^ (r >> 1))];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          const u32x4v w = mine[(16 * (kRowTiles + j) + r) * 8 + ((4 * h + g) ^ (r >> 1))];
#pragma unroll
          for (int a = 0; a < kRowTiles; ++a) acc[a][j] = dev::mfma_bf16(x[a], w, acc[a][j]);
        }
      }
      dev::wave_lds_barrier();
    }
  }
  // Join the waves, 16 rows at a time: sum[w][j][16 g + c][i] is row 4 g + i, rank 16 j + c.
  f32x4* const sum = reinterpret_cast<f32x4*>(sh);
#pragma unroll
  for (int a = 0; a < kRowTiles; ++a) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kTiles; ++j) sum[(wave * kTiles + j) * 64 + lane] = acc[a][j];
    __syncthreads();
#pragma unroll
    for (int e = static_cast<int>(threadIdx.x); e < 256 * kTiles; e += 64 * kN) {
      const int rank = e % (16 * kTiles), row = e / (16 * kTiles);
      if (16 * a + row < rows && rank0 + rank < ad.rank) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kN; ++w)
          x += sum[(w * kTiles + (rank >> 4)) * 64 + 16 * (row >> 2) + (rank & 15)][row & 3];
        emit(16 * a + row, rank0 + rank, rank0 + rank < ad.own ? x : 0.f);
      }
    }
  }
}

// The same for all of an adapter's ranks, up to 16 kMost of them at a time: the adapter's
// own rank, not the largest one, says what is read.
template <int kRowTiles, int kMost, int kN, typename RowAt, typename Emit>
__device__ __forceinline__ void down_ranks(const LoraArgs& p, const Adapter& ad, RowAt row_at, int rows, int k0,
                                           int end, u32x4v* sh, Emit emit) {
  int rank0 = 0;
  if constexpr (kMost == 4)
    for (; ad.rank - rank0 > 32; rank0 += 64) {
      if (rank0) __syncthreads();
      down_rows<kRowTiles, 4, kN>(p, ad, row_at, rows, rank0, k0, end, sh, emit);
    }
  if (ad.rank <= rank0) return;
  if (rank0) __syncthreads();
  if constexpr (kMost >= 2)
    if (ad.rank - rank0 > 16) return down_rows<kRowTiles, 2, kN>(p, ad, row_at, rows, rank0, k0, end, sh, emit);
  down_rows<kRowTiles, 1, kN>(p, ad, row_at, rows, rank0, k0, end, sh, emit);
}

template <int kRowTiles, int kMost, bool kGrouped>
__global__ __launch_bounds__(kThreads, kRowTiles == 1 ? 3 : 2) void lora_down_kernel(const LoraArgs p) {
  __shared__ u32x4v sh[kWaves * 2 * (kRowTiles + kMost) * 64];
  const int k0 = static_cast<int>(blockIdx.x) * p.k_per, end = min(k0 + p.k_per, p.K);
  float* const t = p.t + static_cast<int64_t>(blockIdx.x) * p.M * p.max_rank;
  if constexpr (kGrouped) {
    __shared__ int owner[kWaves][64], row[16];
    Tile at;
    if (!find_rows<true>(p, owner[threadIdx.x >> 6], &at)) return;
    const Adapter ad = adapter_of(p, at.with);
    if (ad.rank <= 0) return;
    if (threadIdx.x < 16) row[threadIdx.x] = at.mine;        // (down_rows has barriers before it is read)
    down_ranks<1, kMost, kWaves>(
        p, ad, [&](int k) { return static_cast<int64_t>(__shfl(at.mine, k)); }, at.rows, k0, end, sh,
        [&](int k, int rank, float x) { t[static_cast<int64_t>(row[k]) * p.max_rank + rank] = x; });
  } else {
    const dev::TileAt at = dev::find_tile(p.offsets, p.of, p.segments, p.M, static_cast<int>(blockIdx.y), 1,
                                          16 * kRowTiles);
    if (at.segment < 0) return;
    const Adapter ad = adapter_of(p, at.with);
    if (ad.rank <= 0) return;
    const int64_t row0 = at.first + 16 * kRowTiles * at.tile;
    down_ranks<kRowTiles, kMost, kWaves>(
        p, ad, [&](int k) { return row0 + k; }, min(at.rows - 16 * kRowTiles * at.tile, 16 * kRowTiles), k0, end, sh,
        [&](int k, int rank, float x) { t[(row0 + k) * p.max_rank + rank] = x; });
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

// lo, hi: ranks 8 g .. + 7 of one 32-rank step, scaled -> the step's three B operands.
__device__ __forceinline__ void split_operand(f32x4 lo, f32x4 hi, u32x4v (&out)[3]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float one[3], two[3];
    split3(e < 2 ? lo[2 * e] : hi[2 * e - 4], one);
    split3(e < 2 ? lo[2 * e + 1] : hi[2 * e - 3], two);
#pragma unroll
    for (int w = 0; w < 3; ++w) out[w][e] = dev::pack_bf16(one[w], two[w]);
  }
}

// 8 ranks of t, 0 where there are none, as operands.
__device__ __forceinline__ void load_operand(const float* sh, bool here, u32x4v (&out)[3]) {
  const f32x4 none = {0.f, 0.f, 0.f, 0.f};
  const f32x4* in = reinterpret_cast<const f32x4*>(sh);
  const f32x4 lo = in[0], hi = in[1];
  split_operand(here ? lo : none, here ? hi : none, out);
}

// t of the tile's rows, the ranges of K added in order, scaled, into sh (rows `pitch`
// apart); what lies past the rows and the rank is left as it is.
template <int kAtOnce, typename RowAt>
__device__ __forceinline__ void join_ranges(const LoraArgs& p, const Adapter& ad, RowAt row_at, int rows, float* sh,
                                            int pitch) {
  if (ad.rank <= 0) return;
  const float scale = p.scales[ad.index];
  const int quads = ad.rank >> 2, all = rows * quads;
  const int64_t next_range = static_cast<int64_t>(p.M) * p.max_rank;
#pragma unroll kAtOnce
  for (int e = static_cast<int>(threadIdx.x); e < all; e += kThreads) {
    const int row = e / quads, quad = e - row * quads;
    const float* tp = p.t + row_at(row) * p.max_rank + 4 * quad;
    f32x4 in[kMaxRanges];
#pragma unroll
    for (int s = 0; s < kMaxRanges; ++s)
      in[s] = *reinterpret_cast<const f32x4*>(tp + min(s, p.splits - 1) * next_range);
    f32x4 sum = in[0];
#pragma unroll
    for (int s = 1; s < kMaxRanges; ++s)
      if (s < p.splits) sum += in[s];
    *reinterpret_cast<f32x4*>(sh + row * pitch + 4 * quad) = sum * scale;
  }
}

// A tile's 16 rows, 32 columns of Y at a time: A operand B_a's rows (16 columns),
// straight from memory, B operand t's rows, so that a lane holds 4 neighbouring columns of
// one row.
template <int kSteps>
struct Up {
  const LoraArgs& p;
  int64_t row;                           // row lane % 16
  int rows;
  struct In {
    f32x4 y[2];
    u32x4v b[2][kSteps];
  } now, next;
  u32x4v t[kSteps][3];

  // N % 16 == 0: a tile's columns are all there, or none (then the last tile is read)
  __device__ __forceinline__ void load_y(int n, In* in) const {
    const int lane = static_cast<int>(threadIdx.x) & 63, g = lane >> 4;
    const float* const yp = p.Y + row * p.ld_y + 4 * g;
#pragma unroll
    for (int j = 0; j < 2; ++j) in->y[j] = *reinterpret_cast<const f32x4*>(yp + min(n + 16 * j, p.N - 16));
  }
  __device__ __forceinline__ void load_b(const Adapter& ad, int n, In* in) const {
    const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
    const uint16_t* const B = p.B + static_cast<int64_t>(p.N) * ad.first;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        in->b[j][k] = u32x4v{0, 0, 0, 0};
        if (32 * k + 8 * g < ad.rank)    // ranks are multiples of 8
          in->b[j][k] = *reinterpret_cast<const u32x4v*>(
              B + static_cast<int64_t>(min(n + 16 * j, p.N - 16) + r) * ad.rank + 32 * k + 8 * g);
      }
  }
  // t's rows, pitch floats apart, scaled; rows past the last are not stored, whatever they hold.
  __device__ __forceinline__ void operands(const Adapter& ad, const float* sh, int pitch) {
    const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int k = 0; k < kSteps; ++k) load_operand(sh + r * pitch + 32 * k + 8 * g, 32 * k + 8 * g < ad.rank, t[k]);
  }
  // Columns n, n + stride, .. below n1, the next ones' Y and B_a under way; `now` holds n's.
  __device__ __forceinline__ void columns(const Adapter& ad, int n, int n1, int stride) {
    const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
    for (; n < n1; n += stride) {
      if (n + stride < n1) {
        load_y(n + stride, &next);
        load_b(ad, n + stride, &next);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 2; w >= 0; --w)     // the small terms first
#pragma unroll
          for (int k = 0; k < kSteps; ++k) acc = dev::mfma_bf16(now.b[j][k], t[k][w], acc);
        if (r < rows && n + 16 * j < n1)
          *reinterpret_cast<f32x4*>(p.out + row * p.ld_out + n + 16 * j + 4 * g) = now.y[j] + acc;
      }
      now = next;
    }
  }
};

// Few rows, `up`: a tile of 16 rows, the columns of one slice.
template <int kSteps, bool kGrouped>
__global__ __launch_bounds__(kThreads) void lora_up_kernel(const LoraArgs p, int n_per) {
  __shared__ int owner[kWaves][kGrouped ? 64 : 1], row[16];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  Tile at;
  if (!find_rows<kGrouped>(p, owner[wave], &at)) return;
  Up<kSteps> up{p, at.mine, at.rows};
  const int n0 = static_cast<int>(blockIdx.x) * n_per, n1 = min(n0 + n_per, p.N), n = n0 + 32 * wave;
  if (n < n1) up.load_y(n, &up.now);
  const Adapter ad = adapter_of(p, at.with);
  if (ad.rank <= 0 && p.out == p.Y) return;
  if (n < n1) up.load_b(ad, n, &up.now);
  constexpr int kPitch = 32 * kSteps + 4;
  __shared__ __align__(16) float sh[16 * kPitch];
  if constexpr (kGrouped) {
    if (threadIdx.x < 16) row[threadIdx.x] = at.mine;
    __syncthreads();
    join_ranges<1>(p, ad, [&](int k) { return static_cast<int64_t>(row[k]); }, at.rows, sh, kPitch);
  } else {
    const int64_t row0 = __builtin_amdgcn_readfirstlane(at.mine);
    join_ranges<1>(p, ad, [&](int k) { return row0 + k; }, at.rows, sh, kPitch);
  }
  __syncthreads();
  up.operands(ad, sh, kPitch);
  up.columns(ad, n, n1, 32 * kWaves);
}

// Both products in one launch: a workgroup of a tile and a slice of columns forms all of
// the rows' t for itself.
template <int kMost, bool kGrouped>
__global__ __launch_bounds__(64 * kSmallWaves) void lora_small_kernel(const LoraArgs p, int n_per) {
  constexpr int kSteps = kMost <= 2 ? 1 : 2, kPitch = 32 * kSteps + 4;
  __shared__ u32x4v sh[kSmallWaves * 2 * (1 + kMost) * 64];
  __shared__ __align__(16) float sh_t[16 * kPitch];
  __shared__ int owner[kSmallWaves][kGrouped ? 64 : 1];
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  Tile at;
  if (!find_rows<kGrouped>(p, owner[wave], &at)) return;
  Up<kSteps> up{p, at.mine, at.rows};
  const int n0 = static_cast<int>(blockIdx.x) * n_per, n1 = min(n0 + n_per, p.N), n = n0 + 32 * wave;
  if (n < n1) up.load_y(n, &up.now);
  const Adapter ad = adapter_of(p, at.with);
  if (ad.rank <= 0 && p.out == p.Y) return;
  if (n < n1) up.load_b(ad, n, &up.now);
  const float scale = ad.rank > 0 ? p.scales[ad.index] : 0.f;
  down_ranks<1, kMost, kSmallWaves>(
      p, ad, [&](int k) { return static_cast<int64_t>(__shfl(at.mine, k)); }, at.rows, 0, p.K, sh,
      [&](int k, int rank, float x) { sh_t[k * kPitch + rank] = x * scale; });
  __syncthreads();
  up.operands(ad, sh_t, kPitch);
  up.columns(ad, n, n1, 32 * kSmallWaves);
}

// Many rows: 64 rows of one segment, 16 a wave, the columns of one slice, 64 at a time.  A
// operand t's rows, B operand B_a's rows, column c of the product's tile j being column
// 4 c + j of the 64, so that a lane holds 4 neighbouring columns of 4 rows and 16 lanes load
// and store 256 bytes of a row.  B_a's rows come whole and through LDS, once for the four
// waves, at most 64 ranks at a time (kMany: more than 64; t's operands are then made again
// for every 64).
template <bool kMany>
__global__ __launch_bounds__(kThreads) void lora_up_wide_kernel(const LoraArgs p, int n_per) {
  constexpr int kRows = 16 * kWaves, kCols = 64;
  constexpr int kPitch = (kMany ? 256 : 64) + 4;
  __shared__ __align__(16) float sh_t[kRows][kPitch];
  __shared__ u32x4v sh_b[kCols * 8];
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int my_row = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6) * 16;
  const dev::TileAt at = dev::find_tile(p.offsets, p.of, p.segments, p.M, static_cast<int>(blockIdx.y), 1, kRows);
  if (at.segment < 0) return;
  const int rows = min(at.rows - kRows * at.tile, kRows);
  const int64_t row0 = at.first + kRows * at.tile;
  const int n0 = static_cast<int>(blockIdx.x) * n_per, n1 = min(n0 + n_per, p.N);
  // N % 16 == 0: a lane's columns are all there, or none (then the last ones are read)
  const float* yp[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) yp[i] = p.Y + (row0 + min(my_row + 4 * g + i, rows - 1)) * p.ld_y;
  f32x4 y[4];
  auto load_y = [&](int n) {
    const int c = min(n + 4 * r, p.N - 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = *reinterpret_cast<const f32x4*>(yp[i] + c);
  };
  load_y(n0);
  const Adapter ad = adapter_of(p, at.with);
  if (ad.rank <= 0 && p.out == p.Y) return;
  // Ranks rank0 .. + 63 of B_a's rows n .. + 63: thread's rows bk and bk + 32, unit bu (of
  // 16 bytes).  Row k's unit u lies in LDS at row k ^ (k / 4 & 1), unit u ^ (k / 8 & 7), so
  // that the operand's rows 4 c + j do not conflict.
  const int bk = static_cast<int>(threadIdx.x) >> 3, bu = static_cast<int>(threadIdx.x) & 7;
  u32x4v b_in[2];
  auto load_b = [&](int n, int rank0) {
    const uint16_t* const B = p.B + static_cast<int64_t>(p.N) * ad.first + rank0 + 8 * bu;
    if (rank0 + 8 * bu < ad.rank)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        b_in[x] = *reinterpret_cast<const u32x4v*>(B + static_cast<int64_t>(min(n + bk + 32 * x, p.N - 1)) * ad.rank);
  };
  if (ad.rank > 0) load_b(n0, 0);
  join_ranges<2>(p, ad, [&](int k) { return row0 + k; }, rows, &sh_t[0][0], kPitch);
  __syncthreads();
  u32x4v t[2][3];
  auto operands = [&](int rank0) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      load_operand(&sh_t[my_row + r][rank0 + 32 * k + 8 * g], rank0 + 32 * k + 8 * g < ad.rank, t[k]);
  };
  if (ad.rank > 0) operands(0);
  for (int n = n0; n < n1; n += kCols) {
    f32x4 acc[4], y_now[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      acc[j] = {0.f, 0.f, 0.f, 0.f};
      y_now[j] = y[j];
    }
    for (int rank0 = 0; rank0 < ad.rank; rank0 += 64) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int k = bk + 32 * x;
        sh_b[(k ^ (k >> 2 & 1)) * 8 + (bu ^ (k >> 3 & 7))] = b_in[x];
      }
      __syncthreads();
      if (kMany && rank0 + 64 < ad.rank) {
        load_b(n, rank0 + 64);
      } else if (n + kCols < n1) {
        load_y(n + kCols);
        load_b(n + kCols, 0);
      }
      if (kMany) operands(rank0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = 4 * r + j;
        u32x4v b[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          b[s] = sh_b[(k ^ (k >> 2 & 1)) * 8 + ((4 * s + g) ^ (k >> 3 & 7))];
          if (rank0 + 32 * s + 8 * g >= ad.rank) b[s] = u32x4v{0, 0, 0, 0};
        }
#pragma unroll
        for (int w = 2; w >= 0; --w)     // the small terms first
#pragma unroll
          for (int s = 0; s < 2; ++s) acc[j] = dev::mfma_bf16(t[s][w], b[s], acc[j]);
      }
      __syncthreads();
    }
    if (ad.rank <= 0 && n + kCols < n1) load_y(n + kCols);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (my_row + 4 * g + i < rows && n + 4 * r < n1)
        *reinterpret_cast<f32x4*>(p.out + (row0 + my_row + 4 * g + i) * p.ld_out + n + 4 * r) =
            y_now[i] + f32x4{acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
  }
}

template <int kRowTiles, int kMost>
void launch_down(const LoraArgs& p, int64_t tiles, bool grouped, hipStream_t stream) {
  const dim3 grid(p.splits, static_cast<unsigned>(tiles));
  if (kRowTiles == 1 && grouped) lora_down_kernel<1, kMost, true><<<grid, kThreads, 0, stream>>>(p);
  else lora_down_kernel<kRowTiles, kMost, false><<<grid, kThreads, 0, stream>>>(p);
}

template <int kSteps>
void launch_up(const LoraArgs& p, int64_t tiles, int n_per, bool grouped, hipStream_t stream) {
  const dim3 grid((p.N + n_per - 1) / n_per, static_cast<unsigned>(tiles));
  if (grouped) lora_up_kernel<kSteps, true><<<grid, kThreads, 0, stream>>>(p, n_per);
  else lora_up_kernel<kSteps, false><<<grid, kThreads, 0, stream>>>(p, n_per);
}

template <int kMost>
void launch_small(const LoraArgs& p, int64_t tiles, int n_per, bool grouped, hipStream_t stream) {
  const dim3 grid((p.N + n_per - 1) / n_per, static_cast<unsigned>(tiles));
  if (grouped) lora_small_kernel<kMost, true><<<grid, 64 * kSmallWaves, 0, stream>>>(p, n_per);
  else lora_small_kernel<kMost, false><<<grid, 64 * kSmallWaves, 0, stream>>>(p, n_per);
}

template <bool kMany>
void launch_up_wide(const LoraArgs& p, int64_t tiles, int n_per, hipStream_t stream) {
  lora_up_wide_kernel<kMany>
      <<<dim3((p.N + n_per - 1) / n_per, static_cast<unsigned>(tiles)), kThreads, 0, stream>>>(p, n_per);
}

}  // namespace

LoraPlan plan_lora(int M, int segments, int adapters, int N, int K, int max_rank, int num_cus) {
  LoraPlan c;
  c.tiles = most_tiles(M, segments, 1, 16);
  // Few rows in more segments than there are adapters: the rows of an adapter together, which
  // reads it once.  us, 64 requests of a row, by segments / by adapters: 24 adapters of ranks up
  // to 64, K = 9728 17.0 / 14.2; of ranks up to 16, K = 2560, N = 4096 8.8 / 8.9, 8 of those
  // 7.8 / 6.4.
  const int64_t groups = std::min<int64_t>(M, int64_t{adapters} + 1 + M / 16);
  c.grouped = M <= 64 && groups < std::min(M, segments);
  // One launch while what every slice forms again, all of its rows' t, costs less than a
  // launch: us, one / two launches, rank 16, K = 2560, N = 4096: 1 row 6.2 / 6.9, 64 requests
  // of a row 8.0 / 11.4, 3000 rows 25.7 / 32.3; N = 9728: 2000 rows 45 / 51, 3000 rows 79 / 60;
  // K = 9728, 1 row: 11.6 / 7.8; rank 64, K = 4096, 8 requests: 14 / 9.2.
  if (max_rank <= 64 && K <= 4096 && max_rank * K <= 32 * 4096 && c.tiles <= num_cus &&
      (N <= 4096 || 2 * c.tiles <= num_cus)) {
    c.small = true;
    const int cols = 32 * kSmallWaves;
    if (c.grouped) c.tiles = groups;
    const int64_t slices = std::max<int64_t>(1, num_cus / c.tiles);
    c.n_per = static_cast<int>(((N + slices - 1) / slices + cols - 1) / cols * cols);
    return c;
  }
  // Rows share an adapter's loads where segments have them to share.
  const int64_t mean = M / std::max(1, std::min(M, segments));
  c.row_tiles = mean >= 32 ? 2 : 1;
  c.row_waves = mean >= 32 ? kWaves : 1;
  c.tiles = most_tiles(M, segments, 1, 16 * c.row_tiles);
  c.up_tiles = most_tiles(M, segments, 1, 16 * c.row_waves);
  // Ranges of K until there are four workgroups a CU, or the two that its registers hold of 32 rows
  // and more than 32 ranks (4 / 2 a CU: 8192 rows, K = 2560, N = 9728, rank 64 138.5 / 135.3 us, 4096
  // rows, K = 9728, N = 2560, rank 64 59.0 / 57.5, rank 32 50.7 / 53.5), two steps a wave at least.
  const int steps = (K + 63) / 64;
  const int64_t at_once = (c.row_tiles == 2 && max_rank > 32 ? 2 : 4) * static_cast<int64_t>(num_cus);
  const int64_t want = (at_once + c.tiles - 1) / c.tiles;
  const int64_t most = std::min(std::max(1, steps / (2 * kWaves)), kMaxRanges);
  const int splits = static_cast<int>(std::max<int64_t>(1, std::min(want, most)));
  if (c.grouped) c.tiles = c.up_tiles = groups;        // (the workspace is the same either way)
  c.k_per = (steps + splits - 1) / splits * 64;
  c.splits = (K + c.k_per - 1) / c.k_per;
  // Short slices: many workgroups a CU hide each other's start (8192 rows x 9728 columns,
  // slices for 4 / 8 / 24 workgroups a CU: 161 / 155 / 145 us).
  const int64_t slices = std::max<int64_t>(1, (24 * static_cast<int64_t>(num_cus) + c.up_tiles - 1) / c.up_tiles);
  const int cols = c.row_waves == 1 ? 32 * kWaves : 64;
  c.n_per = static_cast<int>((N + slices - 1) / slices + cols - 1) / cols * cols;
  return c;
}

size_t lora_workspace_bytes(const LoraPlan& c, int M, int max_rank) {
  return c.small ? 0 : static_cast<size_t>(c.splits) * M * max_rank * 4;
}

hipError_t launch_lora(const LoraPlan& c, const uint16_t* x, int64_t ld_x, int M, int K, const uint16_t* A,
                       const uint16_t* B, const int32_t* rank_offsets, const int32_t* ranks, const float* scales,
                       int adapters, int rank_rows, int max_rank, const int32_t* offsets, const int32_t* of,
                       int segments, int N, const float* Y, int64_t ld_y, float* out, int64_t ld_out,
                       void* workspace, hipStream_t stream) {
  const LoraArgs p{x, ld_x, A, B, rank_offsets, ranks, scales, offsets, of, Y, out, ld_y, ld_out,
                   static_cast<float*>(workspace), adapters, rank_rows, segments, M, N, K, max_rank, c.splits,
                   c.k_per};
  if (c.small) {
    if (max_rank <= 16) launch_small<1>(p, c.tiles, c.n_per, c.grouped, stream);
    else if (max_rank <= 32) launch_small<2>(p, c.tiles, c.n_per, c.grouped, stream);
    else launch_small<4>(p, c.tiles, c.n_per, c.grouped, stream);
    return hipGetLastError();
  }
  if (c.row_tiles == 2) {
    if (max_rank <= 16) launch_down<2, 1>(p, c.tiles, false, stream);
    else if (max_rank <= 32) launch_down<2, 2>(p, c.tiles, false, stream);
    else launch_down<2, 4>(p, c.tiles, false, stream);
  } else {
    if (max_rank <= 16) launch_down<1, 1>(p, c.tiles, c.grouped, stream);
    else if (max_rank <= 32) launch_down<1, 2>(p, c.tiles, c.grouped, stream);
    else launch_down<1, 4>(p, c.tiles, c.grouped, stream);
  }
  if (c.row_waves == kWaves) {
    if (max_rank <= 64) launch_up_wide<false>(p, c.up_tiles, c.n_per, stream);
    else launch_up_wide<true>(p, c.up_tiles, c.n_per, stream);
  } else {
    if (max_rank <= 32) launch_up<1>(p, c.up_tiles, c.n_per, c.grouped, stream);
    else if (max_rank <= 64) launch_up<2>(p, c.up_tiles, c.n_per, c.grouped, stream);
    else if (max_rank <= 128) launch_up<4>(p, c.up_tiles, c.n_per, c.grouped, stream);
    else launch_up<8>(p, c.up_tiles, c.n_per, c.grouped, stream);
  }
  return hipGetLastError();
}

}  // namespace prq
