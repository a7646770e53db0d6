// Device-side bf16 helpers of the attention block's kernels (norm_rope.hip,
// tree_attention.hip, lora.hip) for gfx950.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace prq {
namespace dev {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

// bf16 pair (low half first) of two floats, round to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float bf16_float(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }

// D (16 x 16, float32) += A (16 x 32) B (32 x 16), bf16.  Lane l: A row l % 16 and
// B column l % 16, both at k = 8 (l / 16) .. + 7; D column l % 16, rows
// 4 (l / 16) .. + 3.
__device__ __forceinline__ f32x4 mfma_bf16(u32x4v a, u32x4v b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                 0, 0, 0);
}

// Between LDS accesses by which the lanes of one wave hand values to each other.  The wave's
// LDS operations are done in order, so nothing waits; but the barrier builtin orders no memory
// for the compiler, and the places that a lane writes and reads itself may be different ones.
__device__ __forceinline__ void wave_lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Every lane's sum over itself and the lanes before it.
__device__ __forceinline__ int prefix_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);    // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);    // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}

// The wave's largest value, and its sum (lane 63's, in the same order for every wave).
template <int kCtrl, int kRows>
__device__ __forceinline__ float moved(float old, float x) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), kCtrl, kRows, 0xF, false));
}
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, moved<0x111, 0xF>(x, x));
  x = fmaxf(x, moved<0x112, 0xF>(x, x));
  x = fmaxf(x, moved<0x114, 0xF>(x, x));
  x = fmaxf(x, moved<0x118, 0xF>(x, x));
  x = fmaxf(x, moved<0x142, 0xA>(x, x));
  x = fmaxf(x, moved<0x143, 0xC>(x, x));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ float wave_sum(float x) {
  x += moved<0x111, 0xF>(0.f, x);
  x += moved<0x112, 0xF>(0.f, x);
  x += moved<0x114, 0xF>(0.f, x);
  x += moved<0x118, 0xF>(0.f, x);
  x += moved<0x142, 0xA>(0.f, x);
  x += moved<0x143, 0xC>(0.f, x);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// Segment tables on the device: segment s holds rows [offsets[s], offsets[s + 1]),
// per_row units each, cut into tiles of per_tile units.  find_tile: the segment that
// holds tile `t` (counted over all segments), the tile's number in it, and the
// segment's entry of `with` (loaded beside the offsets: one round trip to memory);
// segment -1 past the last.  Offsets outside [0, M] or descending are clamped to empty
// segments, so no table makes a kernel leave its buffers.  Every lane of the wave calls
// it.
struct TileAt {
  int segment, tile, first, rows, with;
};

__device__ __forceinline__ TileAt find_tile(const int32_t* __restrict__ offsets, const int32_t* __restrict__ with,
                                            int segments, int M, int t, int per_row, int per_tile) {
  const int lane = static_cast<int>(threadIdx.x) & 63;
  int before = 0, base = 0, at = -1;
  int lo = 0, n = 0, tiles = 0, entry = 0, sum = 0;
  for (; base < segments; base += 64) {
    const int s = base + lane;
    lo = n = tiles = entry = 0;
    if (s < segments) {
      lo = offsets[s];
      n = offsets[s + 1];
      entry = with[s];
      lo = min(max(lo, 0), M);
      n = max(min(max(n, 0), M) - lo, 0);
      tiles = (n * per_row + per_tile - 1) / per_tile;
    }
    sum = prefix_sum(tiles);
    const uint64_t past = __ballot(before + sum > t);
    if (past) {
      at = __builtin_ctzll(past);
      break;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  TileAt r;
  r.segment = at < 0 ? -1 : base + at;
  at = max(at, 0);
  r.tile = t - before - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(tiles, at));
  r.first = __builtin_amdgcn_readlane(lo, at);
  r.rows = __builtin_amdgcn_readlane(n, at);
  r.with = __builtin_amdgcn_readlane(entry, at);
  return r;
}

}  // namespace dev

// The most tiles that find_tile counts for `rows` rows in `segments` segments.
inline int64_t most_tiles(int64_t rows, int64_t segments, int64_t per_row, int64_t per_tile) {
  const int64_t used = segments < rows ? segments : rows;
  return (rows * per_row + (per_tile - 1) * used) / per_tile;
}

}  // namespace prq
