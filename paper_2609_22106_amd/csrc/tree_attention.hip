// Attention of each request's tokens -- one, a tree of drafted ones, or a chunk of a
// prompt -- over that request's pages of the cache.
//
// Request b has `cached` tokens that all its rows see, then its n rows' own tokens
// (in the cache too), seen as the tree mask says (no mask: a row and those before
// it).  Row i, query head h, kv head h / G:
//   s_j = scale q . k_j,  p = softmax of the visible s,  o = sum_j p_j v_j,
// o = 0 and lse = -inf for a row that sees nothing.
//
// One pass over K and V with the running maximum and sum: a wave takes 32 keys at a
// time and holds everything in registers.  Scores are computed transposed, keys x
// queries (A = K rows, B = Q rows), so that a lane ends with 8 keys of one query:
// rounded to bf16 they are its operand of the second product, O^T = V^T P^T, as they
// stand.  That product's A operand needs 8 keys of one column of V: a lane group loads
// whole rows of its 8 keys, 16 lanes a row, and pairs up halves of registers
// (32 v_perm per 32 x 128 tile).  The 16 queries of a product's column side are the G
// query heads of the kv head for 16 / G tokens.  Up to 16 columns a request, the waves
// take keys of their own, straight from memory into registers, and join their results
// through LDS; more columns are dealt to the waves, one or two tiles each, and K and V go
// through LDS once for all of them (trees of up to 64 nodes over 8 x 32 k tokens: four tiles
// a wave straight from memory 714 us, through LDS 303).
//
// The maximum is kept per lane group and only joined across the groups when a score
// passes it by 8 (powers of two): until then the stale maximum serves, P up to 2^8.
// Scores, statistics and O are float32; P is rounded to bf16 for its product (relative
// error 2^-9 each, as large as the rounding of the output; the sum that divides takes
// the unrounded P).
//
// Few rows leave most CUs idle, so each request's keys are split into equal parts over
// workgroups and the partial (m, l, O) joined by a second kernel in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;
using dev::u32x4v;

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kStep = 32 * kWaves;       // keys a narrow workgroup takes at a time
constexpr int kMaxSplits = 64;
constexpr float kSlack = 8.0f;           // log2 a score may pass the maximum by before it is renewed
constexpr float kNone = -INFINITY;

struct TreeArgs {
  const uint16_t* q;
  int64_t ld_q;
  const uint16_t *K, *V;
  int64_t page_stride;
  int page_shift, num_pages;
  const int32_t* pages;
  int64_t ld_pages;
  int max_keys;                          // keys the page table has room for
  const int32_t *cached, *offsets;
  const uint8_t* mask;
  int64_t ld_mask;
  int mask_wide;
  float scale, slack;                    // scale times log2 e, positive; kSlack / scale
  uint32_t flip;                         // sign bits to turn in q (a negative scale)
  uint16_t* out;
  float *lse, *part_o;
  float2* part_ml;
  int M, B, Hq, Hk, G, tiles, splits;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// exp2(scale (a - b)), 0 where a is -inf (b may be, too).
__device__ __forceinline__ float exp2_from(float a, float b, float scale) {
  return a == kNone ? 0.f : exp2_fast((a - b) * scale);
}

// The largest; a NaN stays one (its column is NaN whatever the maximum), which takes an
// instruction less than dropping it.
__device__ __forceinline__ float max_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float max_of(float a, float b, float c) { return max_of(max_of(a, b), c); }

__device__ __forceinline__ bool word_finite(uint32_t w) {
  return (w & 0x7F80u) != 0x7F80u && (w & 0x7F800000u) != 0x7F800000u;
}

// K and V of two 16-key blocks, as a lane (g = l / 16, r = l % 16) holds them.
template <int D>
struct Tile {
  static constexpr int kChunks = D / 32, kWords = D / 32;
  u32x4v keys[2][kChunks];               // key r of each block, dims 32 c + 8 g ..
  uint32_t values[8][kWords];            // keys 4 g .. + 3 of each block, dims (D / 16) r ..

  __device__ __forceinline__ void k(int b, u32x4v (&out)[kChunks]) const {
#pragma unroll
    for (int c = 0; c < kChunks; ++c) out[c] = keys[b][c];
  }
  __device__ __forceinline__ void v(int, uint32_t (&out)[8][kWords]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int x = 0; x < kWords; ++x) out[e][x] = values[e][x];
  }
};

// A lane's part of one row of V.
template <int D>
__device__ __forceinline__ void load_v(const uint16_t* at, uint32_t (&v)[D / 32]) {
  if constexpr (D == 64) {
    const dev::u32x2 w = *reinterpret_cast<const dev::u32x2*>(at);
    v[0] = w.x;
    v[1] = w.y;
  } else {
#pragma unroll
    for (int c = 0; c < D / 128; ++c) {
      const u32x4v w = *reinterpret_cast<const u32x4v*>(at + 8 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * c + e] = w[e];
    }
  }
}

template <int D>
__device__ __forceinline__ void load_tile(const TreeArgs& p, const int64_t (&base)[2], Tile<D>* t) {
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint16_t* kp = p.K + base[b] + r * D + 8 * g;
#pragma unroll
    for (int c = 0; c < Tile<D>::kChunks; ++c) t->keys[b][c] = *reinterpret_cast<const u32x4v*>(kp + 32 * c);
  }
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint16_t* vp = p.V + base[b] + 4 * g * D + r * (D / 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) load_v<D>(vp + i * D, t->values[4 * b + i]);
  }
}

// What a workgroup works on: a tile of one request's query columns (column c is token
// c / G, head h G + c % G), and a range of its keys.
struct Part {
  dev::TileAt at;
  int h, split, c0, cols, cached, lo, hi;
};

// false: nothing to do (where the keys are split, the join is told so).
__device__ __forceinline__ bool find_part(const TreeArgs& p, int per_tile, Part* w) {
  w->h = static_cast<int>(blockIdx.x) % p.Hk;
  const int rest = static_cast<int>(blockIdx.x) / p.Hk;
  w->split = rest / p.tiles;
  w->at = dev::find_tile(p.offsets, p.cached, p.B, p.M, rest % p.tiles, p.G, per_tile);
  if (w->at.segment < 0) return false;
  w->c0 = w->at.tile * per_tile;
  w->cols = min(w->at.rows * p.G - w->c0, per_tile);
  w->cached = min(max(w->at.with, 0), p.max_keys);
  const int keys = min(w->at.rows, p.max_keys - w->cached) + w->cached;
  // equal parts of this request's own keys, whole steps
  const int part = ((keys + p.splits - 1) / p.splits + kStep - 1) / kStep * kStep;
  w->lo = min(w->split * part, keys);
  w->hi = min(w->lo + part, keys);
  if (p.splits == 1 || w->hi > w->lo) return true;
  for (int x = static_cast<int>(threadIdx.x); x < w->cols; x += kThreads) {
    const int c = w->c0 + x;
    const int64_t row = w->at.first + c / p.G;
    p.part_ml[(w->split * static_cast<int64_t>(p.M) + row) * p.Hq + w->h * p.G + c % p.G] = {kNone, 0.f};
  }
  return false;
}

// Element offset of the 16-key block with key `key` on page `page` of the pool.  A block
// past the keys, or on a page outside the pool (-1), reads the pool's first page, and its
// keys are not seen.
template <int D>
__device__ __forceinline__ int64_t block_base(const TreeArgs& p, int h, int page, int key) {
  return max(page, 0) * p.page_stride +
         ((static_cast<int64_t>(h) << p.page_shift) + (key & ((1 << p.page_shift) - 1))) * D;
}

// A wave's T tiles of 16 query columns: operands, running maximum (of q . k, the same
// in the four lanes of a column), sum (a lane's own keys) and output.
template <int D, int T>
struct Wave {
  static constexpr int kChunks = D / 32, kV = D / 16;
  u32x4v q[T][kChunks];
  int token[T];
  f32x4 o[T][kV];
  float m[T], l[T];

  __device__ __forceinline__ void start(const TreeArgs& p, const Part& w, int c0) {
    const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int c = c0 + 16 * t + r;     // past the last column: the last token, not stored
      token[t] = min(c / p.G, w.at.rows - 1);
      const uint16_t* qp = p.q + (w.at.first + token[t]) * p.ld_q + (w.h * p.G + c % p.G) * D + 8 * g;
#pragma unroll
      for (int k = 0; k < kChunks; ++k) q[t][k] = *reinterpret_cast<const u32x4v*>(qp + 32 * k) ^ p.flip;
      m[t] = kNone;
      l[t] = 0.f;
#pragma unroll
      for (int v = 0; v < kV; ++v) o[t][v] = {0.f, 0.f, 0.f, 0.f};
    }
  }

  // The 16 kBlocks keys from k0 on; block b of them on page page[b] of the pool (-1: none).
  // kPlain: every row sees all of them.
  // `src`: where the operands are, k(b, ..) block b's keys, v(b, ..) those of blocks b and
  // b + 1.
  template <bool kPlain, int kBlocks, typename Source>
  __device__ __forceinline__ void step(const TreeArgs& p, const Part& w, const Source& src, int k0,
                                       const int (&page)[kBlocks]) {
    constexpr int kOwn = 4 * kBlocks;    // keys of a lane: e is 16 (e / 4) + 4 g + e % 4
    const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
    float s[T][kOwn];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      u32x4v k[kChunks];
      src.k(b, k);
#pragma unroll
      for (int t = 0; t < T; ++t) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kChunks; ++c) x = dev::mfma_bf16(k[c], q[t][c], x);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][4 * b + i] = x[i];
      }
    }
    uint32_t seen[T];
    if constexpr (!kPlain) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const uint8_t* see = p.mask ? p.mask + (w.at.first + token[t]) * p.ld_mask : nullptr;
        seen[t] = 0;
#pragma unroll
        for (int e = 0; e < kOwn; ++e) {
          const int j = k0 + 16 * (e >> 2) + 4 * g + (e & 3) - w.cached;
          const int own = see && j >= 0 && j < p.mask_wide ? see[j] : 0;
          const bool ok = j < w.hi - w.cached && page[e >> 2] >= 0 && (j < 0 || (see ? own != 0 : j <= token[t]));
          seen[t] |= static_cast<uint32_t>(ok) << e;
        }
#pragma unroll
        for (int e = 0; e < kOwn; ++e)
          if (!(seen[t] >> e & 1)) s[t][e] = kNone;
      }
    }

    // A lane whose scores pass the running maximum by more than the slack renews it.
    bool past = false;
    float top[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      top[t] = max_of(s[t][0], s[t][1]);
#pragma unroll
      for (int e = 2; e < kOwn; e += 2) top[t] = max_of(top[t], s[t][e], s[t][e + 1]);
      past |= top[t] > m[t] + p.slack;
    }
    if (__any(past)) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        float x = max_of(m[t], top[t]);
        x = max_of(x, __shfl_xor(x, 16));
        x = max_of(x, __shfl_xor(x, 32));
        const float a = exp2_from(m[t], x, p.scale);
        m[t] = x;
        l[t] *= a;
#pragma unroll
        for (int v = 0; v < kV; ++v) o[t][v] *= a;
      }
    }
    u32x4v pw[T][kBlocks / 2];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const float from = m[t] == kNone ? 0.f : m[t] * p.scale;
#pragma unroll
      for (int b = 0; b < kBlocks; b += 2) {
        float* x = s[t] + 4 * b;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = exp2_fast(__builtin_fmaf(x[e], p.scale, -from));
        l[t] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
        for (int e = 0; e < 4; ++e) pw[t][b / 2][e] = dev::pack_bf16(x[2 * e], x[2 * e + 1]);
      }
    }
    bool odd_v = false;                  // some key's V holds an infinity or a NaN
#pragma unroll
    for (int b = 0; b < kBlocks / 2; ++b) {
      if (b) __builtin_amdgcn_sched_barrier(0);              // one pair's V in registers at a time
      uint32_t y[8][D / 32];
      src.v(2 * b, y);
      // What no row may see must not reach the product either (0 x NaN): V past the
      // keys becomes 0, and infinities and NaN are taken out and added below for the
      // rows that do see them.
      if constexpr (!kPlain) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool ok = k0 + 32 * b + 16 * (e >> 2) + 4 * g + (e & 3) < w.hi && page[2 * b + (e >> 2)] >= 0;
#pragma unroll
          for (int x = 0; x < D / 32; ++x) {
            if (!ok) y[e][x] = 0;
            if (!word_finite(y[e][x])) {
              y[e][x] = 0;
              odd_v = true;
            }
          }
        }
      }
      // V^T: register pairs of neighbouring keys -> the low and the high halves' columns.
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        u32x4v even, odd;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          even[e] = __builtin_amdgcn_perm(y[2 * e + 1][x], y[2 * e][x], 0x05040100u);
          odd[e] = __builtin_amdgcn_perm(y[2 * e + 1][x], y[2 * e][x], 0x07060302u);
        }
#pragma unroll
        for (int t = 0; t < T; ++t) {
          o[t][2 * x] = dev::mfma_bf16(even, pw[t][b], o[t][2 * x]);
          o[t][2 * x + 1] = dev::mfma_bf16(odd, pw[t][b], o[t][2 * x + 1]);
        }
      }
    }
    if (!kPlain && __any(odd_v)) {            // rare: the words taken out above, row by row
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const int64_t base = block_base<D>(p, w.h, page[b], k0 + 16 * b);
        for (int kk = 0; kk < 16; ++kk) {
          if (k0 + 16 * b + kk >= w.hi || page[b] < 0) break;
          const uint16_t* vp = p.V + base + kk * D;
          const int from = 16 * (kk >> 2) + r;
#pragma unroll
          for (int t = 0; t < T; ++t) {
            float mine = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) mine = x == (kk & 3) ? s[t][4 * b + x] : mine;
            const float pk = __shfl(mine, from);
            const bool sees = (__shfl(static_cast<int>(seen[t]), from) >> (4 * b + (kk & 3))) & 1;
#pragma unroll
            for (int v = 0; v < kV; ++v)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int d = kV * (4 * g + i) + v;
                const uint32_t word = vp[d & ~1] | static_cast<uint32_t>(vp[d | 1]) << 16;
                if (sees && !word_finite(word)) o[t][v][i] += pk * dev::bf16_float(vp[d]);
              }
          }
        }
      }
    }
  }
};

// The page of the block at `key`, -1 where there is none.
__device__ __forceinline__ int page_entry(const TreeArgs& p, const Part& w, int key) {
  const int page = key < w.hi ? p.pages[w.at.segment * p.ld_pages + (key >> p.page_shift)] : -1;
  return page < p.num_pages ? page : -1;
}

// Up to 16 query columns: the waves take every fourth 32 keys each, straight into
// registers, the next ones under way, and join through LDS at the end.
template <int D>
__global__ __launch_bounds__(kThreads, D <= 128 ? 2 : 1) void tree_attention_kernel(const TreeArgs p) {
  constexpr int kV = D / 16, kPitch = D + 4;
  __shared__ __align__(16) float sh_o[kWaves][16][kPitch];
  __shared__ float sh_m[kWaves][16], sh_l[kWaves][16];
  Part w;
  if (!find_part(p, 16, &w)) return;
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int first = w.lo + 32 * wave;
  const int steps = w.hi > first ? (w.hi - first + kStep - 1) / kStep : 0;
  // lane 2 s + b: page of block b of step s (of 32 steps)
  int entries = page_entry(p, w, first + kStep * (lane >> 1) + 16 * (lane & 1));
  int page[2];
  auto load = [&](int step, Tile<D>* tile) {
    int64_t base[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      page[b] = __builtin_amdgcn_readlane(entries, 2 * (step & 31) + b);
      base[b] = block_base<D>(p, w.h, page[b], first + kStep * step + 16 * b);
    }
    load_tile<D>(p, base, tile);
  };
  Wave<D, 1> q;
  q.start(p, w, w.c0);
  Tile<D> now, next;
  if (steps > 0) load(0, &now);
  auto one = [&](int step, auto plain) {
    const int page_now[2] = {page[0], page[1]};
    if (step + 1 < steps) {
      if (((step + 1) & 31) == 0)
        entries = page_entry(p, w, first + kStep * (step + 1 + (lane >> 1)) + 16 * (lane & 1));
      load(step + 1, &next);
    }
    q.template step<decltype(plain)::value, 2>(p, w, now, first + kStep * step, page_now);
    if (step + 1 < steps) now = next;
  };
  // every row sees the whole step: of cached tokens alone, on pages of the pool
  int step = 0;
  for (; step < steps && first + kStep * step + 32 <= min(w.cached, w.hi) && (page[0] | page[1]) >= 0; ++step)
    one(step, std::true_type{});
  for (; step < steps; ++step) one(step, std::false_type{});

  // Join the waves.
  float l = q.l[0];
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) {
    sh_m[wave][r] = q.m[0];
    sh_l[wave][r] = l;
  }
  __syncthreads();
  const float a = exp2_from(q.m[0], fmaxf(fmaxf(sh_m[0][r], sh_m[1][r]), fmaxf(sh_m[2][r], sh_m[3][r])), p.scale);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int v = 0; v < kV; v += 4)
      *reinterpret_cast<f32x4*>(&sh_o[wave][r][kV * (4 * g + i) + v]) =
          f32x4{q.o[0][v][i], q.o[0][v + 1][i], q.o[0][v + 2][i], q.o[0][v + 3][i]} * a;
  __syncthreads();
  constexpr int kPer = D / 8;            // threads a column
  for (int x = static_cast<int>(threadIdx.x); x < w.cols * kPer; x += kThreads) {
    const int c = x / kPer, d = 8 * (x % kPer);
    const float top = fmaxf(fmaxf(sh_m[0][c], sh_m[1][c]), fmaxf(sh_m[2][c], sh_m[3][c]));
    float sum = 0.f;
    f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll
    for (int y = 0; y < kWaves; ++y) {
      sum += sh_l[y][c] * exp2_from(sh_m[y][c], top, p.scale);
      lo += *reinterpret_cast<const f32x4*>(&sh_o[y][c][d]);
      hi += *reinterpret_cast<const f32x4*>(&sh_o[y][c][d + 4]);
    }
    const int64_t head = (w.at.first + (w.c0 + c) / p.G) * static_cast<int64_t>(p.Hq) + w.h * p.G + (w.c0 + c) % p.G;
    if (p.splits == 1) {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      const u32x4v y = {dev::pack_bf16(lo[0] * inv, lo[1] * inv), dev::pack_bf16(lo[2] * inv, lo[3] * inv),
                        dev::pack_bf16(hi[0] * inv, hi[1] * inv), dev::pack_bf16(hi[2] * inv, hi[3] * inv)};
      *reinterpret_cast<u32x4v*>(p.out + head * D + d) = y;
      if (p.lse && d == 0) p.lse[head] = sum == 0.f ? kNone : (top * p.scale + log2f(sum)) * 0.69314718055994531f;
    } else {
      const int64_t part = w.split * static_cast<int64_t>(p.M) * p.Hq + head;
      *reinterpret_cast<f32x4*>(p.part_o + part * D + d) = lo;
      *reinterpret_cast<f32x4*>(p.part_o + part * D + d + 4) = hi;
      if (d == 0) p.part_ml[part] = {top * p.scale, sum};
    }
  }
}

// Copies 16 bytes a lane straight to LDS, lane l's at lds + 16 l (LDS address, the same for
// the wave).
__device__ __forceinline__ void lds_copy16(const uint16_t* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(src), "s"(lds)
               : "memory", "m0");
}

// K and V of a stage in LDS, and a lane's places in it (elements): rows r of a 16-key block
// of K, 4 g + i of V.
template <int D>
struct Staged {
  const uint16_t *ks, *vs;
  const int (&k_at)[D / 32];
  const int (&v_at)[4];

  __device__ __forceinline__ void k(int b, u32x4v (&out)[D / 32]) const {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) out[c] = *reinterpret_cast<const u32x4v*>(ks + k_at[c] + 16 * b * D);
  }
  __device__ __forceinline__ void v(int b, uint32_t (&out)[8][D / 32]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint16_t* const at = vs + 16 * (b + (e >> 2)) * D;
      if constexpr (D <= 128) {
        load_v<D>(at + v_at[e & 3], out[e]);
      } else {                           // the row's second unit lies at the first one's neighbour
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const u32x4v x = *reinterpret_cast<const u32x4v*>(at + (v_at[e & 3] ^ (8 * c)));
#pragma unroll
          for (int i = 0; i < 4; ++i) out[e][4 * c + i] = x[i];
        }
      }
    }
  }
};

// More columns: each wave its own T tiles of them, all waves the same keys, K and V staged
// in LDS (two stages of kKeys keys; a row's 16-byte units permuted by its number, so
// that neither the K reads, a column of rows, nor the V reads, a whole row, conflict).
template <int D, int T>
__global__ __launch_bounds__(kThreads, D <= 128 ? 2 : 1) void tree_attention_wide_kernel(const TreeArgs p) {
  constexpr int kV = D / 16, kKeys = D <= 128 ? 64 : 32;
  constexpr int kUnits = D / 8, kRows = 64 / kUnits, kCopies = kKeys / kRows / kWaves;
  __shared__ __align__(16) uint16_t sh[2][2][kKeys * D];     // stage, K or V
  Part w;
  if (!find_part(p, 16 * T * kWaves, &w)) return;
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const uint32_t sh_at = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)(&sh[0][0][0])));
  // Unit u of row k lies at unit u ^ turn(k).
  auto turn = [](int k) { return D == 64 ? (k >> 1) & 7 : k & 15; };

  int entries = page_entry(p, w, w.lo + 16 * lane);          // lane b: page of block b (of 64)
  Wave<D, T> q;
  q.start(p, w, w.c0 + 16 * T * wave);
  const bool works = 16 * T * wave < w.cols;                 // else the wave only helps to load

  // A stage's rows are copied kRows to a wave copy (a kilobyte), lane i to unit i of it.
  auto load = [&](int stage) {
    const uint32_t to = sh_at + (stage & 1) * 2 * kKeys * D * 2;
#pragma unroll
    for (int x = 0; x < kCopies; ++x) {
      const int c = wave + kWaves * x;                       // rows kRows c .. of the stage
      const int k = kRows * c + lane / kUnits;
      const int page = __builtin_amdgcn_readlane(entries, (stage * (kKeys / 16) + kRows * c / 16) & 63);
      const int64_t at = block_base<D>(p, w.h, page, w.lo + kKeys * stage + (kRows * c / 16) * 16) + (k & 15) * D +
                         8 * (lane % kUnits ^ turn(k));
      lds_copy16(p.K + at, to + c * 1024);
      lds_copy16(p.V + at, to + kKeys * D * 2 + c * 1024);
    }
  };
  const int stages = (w.hi - w.lo + kKeys - 1) / kKeys;
  // Stages that every row sees whole: of cached tokens alone, on pages of the pool (as far
  // as the entries at hand say).
  int plain = max(min(w.cached, w.hi) - w.lo, 0) / kKeys;
  auto check = [&](int stage) {
    if (__any(w.lo + kKeys * stage + 16 * lane < w.hi && entries < 0)) plain = min(plain, stage);
  };
  check(0);
  if (stages > 0) load(0);
  // the blocks are 16 rows apart, and turn(k) has k's low bits alone
  int k_at[D / 32], v_at[4];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) k_at[c] = r * D + 8 * ((4 * c + g) ^ turn(r));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = 4 * g + i;
    v_at[i] = k * D + (D == 64 ? 8 * ((r >> 1) ^ turn(k)) + 4 * (r & 1) : 8 * ((D / 128 * r) ^ turn(k)));
  }
  auto one = [&](int stage, auto all) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");         // this wave's copies of the stage
    __syncthreads();
    const int entries_now = entries;
    if (stage + 1 < stages) {
      if (((stage + 1) * (kKeys / 16) & 63) == 0) {
        entries = page_entry(p, w, w.lo + kKeys * (stage + 1) + 16 * lane);
        check(stage + 1);
      }
      load(stage + 1);
    }
    if (works) {
      constexpr int kBlocks = kKeys / 16;
      const Staged<D> src{sh[stage & 1][0], sh[stage & 1][1], k_at, v_at};
      int page[kBlocks];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
        page[b] = decltype(all)::value ? 0 : __builtin_amdgcn_readlane(entries_now, (stage * kBlocks + b) & 63);
      q.template step<decltype(all)::value, kBlocks>(p, w, src, w.lo + kKeys * stage, page);
    }
  };
  int stage = 0;
  for (; stage < plain; ++stage) one(stage, std::true_type{});
  for (; stage < stages; ++stage) one(stage, std::false_type{});

#pragma unroll
  for (int t = 0; t < T; ++t) {
    float sum = q.l[t];
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const int c = 16 * (T * wave + t) + r;
    if (c >= w.cols) continue;
    const int64_t head = (w.at.first + (w.c0 + c) / p.G) * static_cast<int64_t>(p.Hq) + w.h * p.G + (w.c0 + c) % p.G;
    const float top = q.m[t] * p.scale;
    if (p.splits == 1) {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < kV; v += 4) {
          const dev::u32x2 y = {dev::pack_bf16(q.o[t][v][i] * inv, q.o[t][v + 1][i] * inv),
                                dev::pack_bf16(q.o[t][v + 2][i] * inv, q.o[t][v + 3][i] * inv)};
          *reinterpret_cast<dev::u32x2*>(p.out + head * D + kV * (4 * g + i) + v) = y;
        }
      if (p.lse && g == 0) p.lse[head] = sum == 0.f ? kNone : (top + log2f(sum)) * 0.69314718055994531f;
    } else {
      const int64_t part = w.split * static_cast<int64_t>(p.M) * p.Hq + head;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int v = 0; v < kV; v += 4)
          *reinterpret_cast<f32x4*>(p.part_o + part * D + kV * (4 * g + i) + v) =
              f32x4{q.o[t][v][i], q.o[t][v + 1][i], q.o[t][v + 2][i], q.o[t][v + 3][i]};
      if (g == 0) p.part_ml[part] = {top, sum};
    }
  }
}

// The splits' (m, l, O) of one row and head, a wave each.
template <int D>
__global__ __launch_bounds__(kThreads) void tree_join_kernel(const float* __restrict__ part_o,
                                                             const float2* __restrict__ part_ml, int64_t heads,
                                                             int splits, uint16_t* __restrict__ out,
                                                             float* __restrict__ lse) {
  constexpr int kPer = D / 4, kAtOnce = 64 / kPer;     // lanes a split, splits a load
  constexpr int kBatch = 8;                            // loads under way
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int64_t head = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (head >= heads) return;
  float2 ml = {kNone, 0.f};
  if (lane < splits) ml = part_ml[lane * heads + head];
  f32x4 in[kBatch];
  auto load = [&](int s0) {
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      const int s = min(s0 + x * kAtOnce + lane / kPer, splits - 1);
      in[x] = *reinterpret_cast<const f32x4*>(part_o + (s * heads + head) * D + 4 * (lane % kPer));
    }
  };
  load(0);
  float top = ml.x;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float a = exp2_from(ml.x, top, 1.0f);
  float sum = a * ml.y;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += kBatch * kAtOnce) {
    if (s0 > 0) load(s0);
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      const int s = s0 + x * kAtOnce + lane / kPer;
      const float w = __shfl(a, s & 63);
      if (s < splits && w != 0.f) o += w * in[x];      // a split with nothing for this row wrote no O
    }
  }
#pragma unroll
  for (int d = kPer; d < 64; d <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], d);
  if (lane < kPer) {
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    const dev::u32x2 w = {dev::pack_bf16(o[0] * inv, o[1] * inv), dev::pack_bf16(o[2] * inv, o[3] * inv)};
    *reinterpret_cast<dev::u32x2*>(out + head * D + 4 * lane) = w;
    if (lse && lane == 0) lse[head] = sum == 0.f ? kNone : (top + log2f(sum)) * 0.69314718055994531f;
  }
}

template <int D>
void launch(const TreeArgs& p, int tile_cols, int64_t blocks, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(blocks));
  if (tile_cols == 16)
    tree_attention_kernel<D><<<grid, kThreads, 0, stream>>>(p);
  else if (tile_cols == 64)
    tree_attention_wide_kernel<D, 1><<<grid, kThreads, 0, stream>>>(p);
  else if constexpr (D <= 128)
    tree_attention_wide_kernel<D, 2><<<grid, kThreads, 0, stream>>>(p);
  if (p.splits > 1) {
    const int64_t heads = static_cast<int64_t>(p.M) * p.Hq;
    tree_join_kernel<D><<<dim3(static_cast<unsigned>((heads + kWaves - 1) / kWaves)), kThreads, 0, stream>>>(
        p.part_o, p.part_ml, heads, p.splits, p.out, p.lse);
  }
}

}  // namespace

TreePlan plan_tree_attention(int M, int B, int Hq, int Hk, int D, int max_kv_len, int num_cus) {
  TreePlan c;
  const int64_t G = Hq / Hk;
  const int64_t used = std::max(1, std::min(M, B));
  const int64_t per = (M * G + used - 1) / used;        // query columns of a mean request
  c.tile_cols = per <= 16 ? 16 : per <= 64 || D > 128 ? 64 : 128;
  c.tiles = most_tiles(M, B, G, c.tile_cols);
  const int64_t groups = c.tiles * Hk;
  const int64_t want = (4 * static_cast<int64_t>(num_cus) + groups - 1) / groups;
  const int64_t keys = std::max(max_kv_len, 1);
  const int64_t most = std::min<int64_t>(kMaxSplits, (keys + kStep - 1) / kStep);
  c.splits = static_cast<int>(std::max<int64_t>(1, std::min(want, most)));
  c.blocks = groups * c.splits;
  return c;
}

size_t tree_workspace_bytes(const TreePlan& c, int M, int Hq, int D) {
  return c.splits > 1 ? static_cast<size_t>(c.splits) * M * Hq * (D + 2) * 4 : 0;
}

hipError_t launch_tree_attention(const TreePlan& c, const uint16_t* q, int64_t ld_q, int M, int Hq, int Hk, int D,
                                 const PagedCache& cache, const int32_t* pages, int64_t ld_pages, int max_keys,
                                 const int32_t* cached, const int32_t* offsets, int B, float scale,
                                 const uint8_t* mask, int64_t ld_mask, int mask_wide, uint16_t* out, float* lse,
                                 void* workspace, hipStream_t stream) {
  const int64_t heads = static_cast<int64_t>(M) * Hq;
  float* const part_o = static_cast<float*>(workspace);
  float2* const part_ml = c.splits > 1 ? reinterpret_cast<float2*>(part_o + c.splits * heads * D) : nullptr;
  // A negative scale turns the queries' signs; 0 is as good as the smallest used here
  // (q . k times it vanishes beside 1) and keeps an unseen -inf from becoming 0 x inf.
  const float size = std::max(std::fabs(scale) * 1.44269504088896341f, 0x1p-100f);
  const TreeArgs p{q, ld_q, cache.K, cache.V, cache.page_stride, cache.page_shift, cache.num_pages, pages, ld_pages,
                   max_keys, cached, offsets, mask, ld_mask, mask_wide, size, kSlack / size,
                   std::signbit(scale) ? 0x80008000u : 0u, out, lse, part_o, part_ml, M, B, Hq, Hk, Hq / Hk, static_cast<int>(c.tiles), c.splits};
  if (D == 64) launch<64>(p, c.tile_cols, c.blocks, stream);
  else if (D == 128) launch<128>(p, c.tile_cols, c.blocks, stream);
  else launch<256>(p, c.tile_cols, c.blocks, stream);
  return hipGetLastError();
}

}  // namespace prq
