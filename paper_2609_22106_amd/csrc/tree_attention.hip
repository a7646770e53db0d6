// Attention of each request's tokens -- one, a tree of drafted ones, or a chunk of a
// prompt -- over that request's pages of the cache.
//
// Request b has `cached` tokens that all its rows see, then its n rows' own tokens
// (in the cache too), seen as the tree mask says (no mask: a row and those before
// it).  Row i, query head h, kv head h / G:
//   s_j = scale q . k_j,  p = softmax of the visible s,  o = sum_j p_j v_j,
// o = 0 and lse = -inf for a row that sees nothing.
//
// One pass over K and V with the running maximum and sum.  Scores are computed transposed,
// keys x queries (A = K rows, B = Q rows), so that a lane ends with 8 of 32 keys of one
// query: rounded to bf16 they are its operand of the second product, O^T = V^T P^T, as they
// stand.  The 16 queries of a product's column side are the G query heads of the kv head for
// 16 / G tokens.
//
// Up to 16 columns a request (narrow): K and V are read once for few products, so memory
// bounds it.  The waves of a workgroup take 32 keys each at a time, straight into registers,
// the next ones under way, and join through LDS.  V's operand needs 8 keys of one column: a
// lane group loads whole rows of its 8 keys, 16 lanes a row, and pairs up halves of registers
// (32 v_perm per 32 x 128 tile).  32 sequences of up to 2176 tokens, 8 kv heads of 128:
// 45 us, 206 MB of K and V at 4.6 TB/s; one token over 4097: 13.3 us, the latency of the
// loads, the arrival and the join one after another.
//
// More columns (wide): they are dealt to the waves, one or two tiles of 16 each, and 32 keys
// at a time go through LDS once for all of them, copied there without a register; V is read
// back transposed.  Trees of up to 64 nodes over 8 x 32 k tokens (377 rows, 204 k keys): straight
// from memory 714 us, through LDS with v_perm 272, transposed reads 258; a stage's scores
// beside the exponentials of the one before and LDS read ahead, 8 waves for more than 128
// columns, those dealt evenly to the SIMDs, a barrier every two stages, 230 (224 to 232 from card
// to card): 690 TFLOP/s, the matrix units 41% of the time, 9 us of it the join's.  What is left:
// the parts, unequal by 17%, and a SIMD's two waves, in step more often than in turn.
//
// The maximum is kept per lane group and only joined across the groups when a score
// passes it by 8 (powers of two): until then the stale maximum serves, P up to 2^8.
// Scores, statistics and O are float32; P is rounded to bf16 for its product (relative
// error 2^-9 each, as large as the rounding of the output; the sum that divides takes
// the unrounded P).
//
// Few rows leave most CUs idle, so a request's keys are split over workgroups: as many
// parts as the chip holds at once, dealt to the requests by their lengths, and the partial
// (m, l, O) joined in a fixed order: by the last part of a tile to arrive where there are few
// columns, by a second kernel where they are many (trees of up to 13 nodes over 6 x 8 k tokens
// 50 us the first way, 24.5 the second, 22.5 by now: one workgroup is then slow to read all parts
// of a tile).
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
  uint32_t* arrived;                     // narrow: parts done, of every tile that has several (0 between calls)
  int4* joins;                           // wide, of every row: its request's first row, first slot, tiles, and
                                         // parts (8 bits) beside its number
  int M, B, Hq, Hk, G, slots, step;      // a part of the keys is a multiple of `step`
  bool split, spread;                    // keys may be split; there are enough tiles as it is
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

__device__ __forceinline__ bool finite_bf16(uint32_t b) { return (b & 0x7F80u) != 0x7F80u; }

// The sign bits of the halves that are infinite or NaN.
__device__ __forceinline__ uint32_t odd_halves(uint32_t two) {
  return ((two & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
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
  // V^T's operand of the product's dims dim(x, 0 .. 15): register pairs of neighbouring keys
  // -> the low or the high halves.
  __device__ __forceinline__ u32x4v v(int x) const {
    u32x4v out;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      out[e] = __builtin_amdgcn_perm(values[2 * e + 1][x >> 1], values[2 * e][x >> 1],
                                     x & 1 ? 0x07060302u : 0x05040100u);
    return out;
  }
  // Whether a V among the keys `ok` is infinite or NaN.
  __device__ __forceinline__ uint32_t odd(uint32_t ok, const u32x4v&) const {
    uint32_t out = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t row = 0;
#pragma unroll
      for (int x = 0; x < kWords; ++x) row |= odd_halves(values[e][x]);
      out |= ok >> e & 1 ? row : 0u;
    }
    return out;
  }
  static __device__ __forceinline__ int dim(int x, int m) { return D / 16 * m + x; }
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
// c / G, head h G + c % G), and a part of its keys.
struct Part {
  int segment, first, rows;              // the request, its first row and their number
  int h, c0, cols, cached, lo, hi;       // kv head, first column and their number, keys
  int splits, first_slot, tiles;         // parts of this request's keys; the tile's slots are
};                                       // first_slot + tiles s

// One request as a lane holds it; offsets and lengths that no table should hold are
// clamped, so that nothing outside the buffers is reached.
struct Request {
  int first = 0, rows = 0, cached = 0, tiles = 0, keys = 0, units = 0;
};

__device__ __forceinline__ Request load_request(const TreeArgs& p, int s, int per_tile) {
  Request r;
  if (s < p.B) {
    r.first = p.offsets[s];
    r.rows = p.offsets[s + 1];
    r.cached = p.cached[s];
    r.first = min(max(r.first, 0), p.M);
    r.rows = max(min(max(r.rows, 0), p.M) - r.first, 0);
    r.cached = min(max(r.cached, 0), p.max_keys);
    r.tiles = (r.rows * p.G + per_tile - 1) / per_tile;
    r.keys = min(r.rows, p.max_keys - r.cached) + r.cached;
    r.units = (r.keys + p.step - 1) / p.step;
  }
  return r;
}

// Parts of `units` of at most about 1 / per units each: a plan, any number is right.
__device__ __forceinline__ int parts_of(int units, float per) {
  return min(max(static_cast<int>(ceilf(static_cast<float>(units) * per)), 1), kMaxSplits);
}

// Slot x of the launch (the same for the kv heads).  A request's keys are cut into equal
// parts, and the most units (of p.step keys) that a part may have is the least for which
// the slots suffice: every workgroup then has as much to do, and all of them are on the
// chip at once.  false: nothing to do.
__device__ __forceinline__ bool find_part(const TreeArgs& p, int per_tile, Part* w) {
  const int lane = static_cast<int>(threadIdx.x) & 63;
  w->h = static_cast<int>(blockIdx.x) % p.Hk;
  const int x = static_cast<int>(blockIdx.x) / p.Hk;
  Request r = load_request(p, lane, per_tile);
  float per = 0.f;                       // parts a unit
  if (p.split && !p.spread && p.B == 1) {
    per = static_cast<float>(p.slots / max(r.tiles, 1)) / static_cast<float>(max(r.units, 1));
    per = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(per))) * 0.999f;
    // (rounded up by parts_of, and never past the slots)
  } else if (p.split) {
    int tiles = 0;
    float total = 0.f, longest = 1.f;
    for (int base = 0; base < p.B; base += 64) {
      const Request y = base ? load_request(p, base + lane, per_tile) : r;
      const float units = static_cast<float>(y.units);
      tiles += __builtin_amdgcn_readlane(dev::prefix_sum(y.tiles), 63);
      total += dev::wave_sum(static_cast<float>(y.tiles) * units);
      longest = fmaxf(longest, dev::wave_max(units));
    }
    // total / most + tiles parts at most: `high` suffices, nothing below `low` does.  Where
    // there are tiles enough to fill the chip only what is half as long again as the mean
    // is cut (and no more than there are slots for: offsets that rise and fall count rows twice).
    float low = max(total / p.slots, 1.f);
    float high = p.slots > tiles ? max(min(total / (p.slots - tiles), longest), low) : longest;
    if (p.spread)
      high = max(1.5f * max(total, 1.f) / max(tiles, 1), total / max(p.slots - tiles, 1));
    else if (p.B <= 64)
      for (int i = 0; i < 4; ++i) {
        const float mid = 0.5f * (low + high);
        const bool fits =
            __builtin_amdgcn_readlane(dev::prefix_sum(r.tiles * parts_of(r.units, 1.f / mid)), 63) <= p.slots;
        low = fits ? low : mid;
        high = fits ? mid : high;
      }
    per = p.slots > tiles ? 1.f / (1.0001f * high) : 0.f;
  }
  int before = 0, base = 0, at = -1, splits = 1, sum = 0;
  for (; base < p.B; base += 64) {
    if (base) r = load_request(p, base + lane, per_tile);
    splits = p.split ? parts_of(r.units, per) : 1;
    sum = dev::prefix_sum(r.tiles * splits);
    if (p.B <= 64 && __builtin_amdgcn_readlane(sum, 63) > p.slots) {   // (not by the bounds above)
      splits = 1;
      sum = dev::prefix_sum(r.tiles);
    }
    const uint64_t past = __ballot(before + sum > x);
    if (past) {
      at = __builtin_ctzll(past);
      break;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  if (at < 0) return false;
  const int tiles = __builtin_amdgcn_readlane(r.tiles, at);
  const int keys = __builtin_amdgcn_readlane(r.keys, at);
  w->segment = base + at;
  w->first = __builtin_amdgcn_readlane(r.first, at);
  w->rows = __builtin_amdgcn_readlane(r.rows, at);
  w->cached = __builtin_amdgcn_readlane(r.cached, at);
  w->splits = __builtin_amdgcn_readlane(splits, at);
  const int slot = before + __builtin_amdgcn_readlane(sum, at) - tiles * w->splits;    // the request's first
  const int split = (x - slot) / tiles, tile = (x - slot) - split * tiles;
  w->tiles = tiles;
  w->first_slot = slot + tile;
  w->c0 = tile * per_tile;
  w->cols = min(w->rows * p.G - w->c0, per_tile);
  const int part = ((keys + w->splits - 1) / w->splits + p.step - 1) / p.step * p.step;
  w->lo = min(split * part, keys);
  w->hi = min(w->lo + part, keys);
  if (!p.mask)                           // a chain: nothing past the tile's last token is seen
    w->hi = max(min(w->hi, w->cached + (w->c0 + w->cols - 1) / p.G + 1), w->lo);
  return true;
}

// Output (row, query head) of a column.
__device__ __forceinline__ int64_t head_of(const TreeArgs& p, const Part& w, int c) {
  return (w.first + (w.c0 + c) / p.G) * static_cast<int64_t>(p.Hq) + w.h * p.G + (w.c0 + c) % p.G;
}

// Element offset of the 16-key block with key `key` on page `page` of the pool.  A block
// past the keys, or on a page outside the pool (-1), reads the pool's first page, and its
// keys are not seen.
template <int D>
__device__ __forceinline__ int64_t block_base(const TreeArgs& p, int h, int page, int key) {
  return max(page, 0) * p.page_stride +
         ((static_cast<int64_t>(h) << p.page_shift) + (key & ((1 << p.page_shift) - 1))) * D;
}

// The page of the block at `key`, -1 where there is none.
__device__ __forceinline__ int page_entry(const TreeArgs& p, const Part& w, int key) {
  const int page = key < w.hi ? p.pages[w.segment * p.ld_pages + (key >> p.page_shift)] : -1;
  return page < p.num_pages ? page : -1;
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

  // Tile t holds columns c0 + 16 t .. + 15.
  __device__ __forceinline__ void start(const TreeArgs& p, const Part& w, int c0) {
    const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const int c = c0 + 16 * t + r;     // past the last column: the last token, not stored
      token[t] = min(c / p.G, w.rows - 1);
      const uint16_t* qp = p.q + (w.first + token[t]) * p.ld_q + (w.h * p.G + c % p.G) * D + 8 * g;
#pragma unroll
      for (int k = 0; k < kChunks; ++k) q[t][k] = *reinterpret_cast<const u32x4v*>(qp + 32 * k) ^ p.flip;
      m[t] = kNone;
      l[t] = 0.f;
#pragma unroll
      for (int v = 0; v < kV; ++v) o[t][v] = {0.f, 0.f, 0.f, 0.f};
    }
  }

  // A step: 32 keys from k0 on, blocks 0 and 1 of them on pages of the pool (page[]; -1: on none).
  // kPlain: every row sees all of them.
  // `src`: where the operands are, k(b, ..) block b's keys, v(x) V^T's for both blocks and the
  // dims dim(x, 0 .. 15), odd(ok, keep) whether V holds an infinity or a NaN in the keys that
  // `ok` names (`keep`: the same as masks of v's words).  A lane's keys: e is 16 (e / 4) + 4 g + e % 4.
  struct Scores {
    float s[T][8];
    uint32_t seen[T];                    // (not plain) bit e
  };

  template <bool kPlain>
  __device__ __forceinline__ void scores(const TreeArgs& p, const Part& w, const u32x4v (&k)[2][kChunks], int k0,
                                         const int (&page)[2], Scores* out) const {
    const int lane = static_cast<int>(threadIdx.x) & 63, g = lane >> 4;
    f32x4 x[T][2];
    // blocks and tiles in turn: a product does not wait for the one before it
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int t = 0; t < T; ++t)
          x[t][y] = dev::mfma_bf16(k[y][c], q[t][c], c ? x[t][y] : f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int e = 0; e < 8; ++e) out->s[t][e] = x[t][e >> 2][e & 3];
    if constexpr (!kPlain) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        // own token of the lane's first key, and which of the request's the row sees: the mask's
        // bytes are all loaded, from its last column on past it, so that none waits for another
        const int j0 = k0 + 4 * g - w.cached, have = w.hi - w.cached;
        uint32_t seen = 0;
        if (p.mask_wide > 0) {
          const uint8_t* see = p.mask + (w.first + token[t]) * p.ld_mask;
          uint8_t own[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) own[e] = see[min(max(j0 + 16 * (e >> 2) + (e & 3), 0), p.mask_wide - 1)];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int j = j0 + 16 * (e >> 2) + (e & 3);
            seen |= static_cast<uint32_t>(j < 0 || (j < p.mask_wide && own[e] != 0)) << e;
          }
        } else {
          const int last = p.mask ? -1 : token[t];           // a mask without a column: no own tokens
#pragma unroll
          for (int e = 0; e < 8; ++e) seen |= static_cast<uint32_t>(j0 + 16 * (e >> 2) + (e & 3) <= last) << e;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (j0 + 16 * (e >> 2) + (e & 3) >= have || page[e >> 2] < 0) seen &= ~(1u << e);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!(seen >> e & 1)) out->s[t][e] = kNone;
        out->seen[t] = seen;
      }
    }
  }

  // A lane whose scores pass the running maximum by more than the slack renews it.
  __device__ __forceinline__ void renew(const TreeArgs& p, const Scores& in) {
    bool past = false;
    float top[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      top[t] = max_of(in.s[t][0], in.s[t][1]);
#pragma unroll
      for (int e = 2; e < 8; e += 2) top[t] = max_of(top[t], in.s[t][e], in.s[t][e + 1]);
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
  }

  // Probabilities (left in `in`, too) and their sum.
  __device__ __forceinline__ void weights(const TreeArgs& p, Scores* in, u32x4v (&pw)[T]) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const float from = m[t] == kNone ? 0.f : m[t] * p.scale;
      float* x = in->s[t];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = exp2_fast(__builtin_fmaf(x[e], p.scale, -from));
      l[t] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
      for (int e = 0; e < 4; ++e) pw[t][e] = dev::pack_bf16(x[2 * e], x[2 * e + 1]);
    }
  }

  template <bool kPlain, typename Source>
  __device__ __forceinline__ void absorb(const TreeArgs& p, const Part& w, const Source& src, int k0,
                                         const int (&page)[2], const Scores* in, const u32x4v (&pw)[T]) {
    const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
    // What no row may see must not reach the product either (0 x NaN): V past the keys becomes
    // 0, and if there are infinities and NaN, those are taken out and added below for the rows
    // that do see them.
    u32x4v keep;
    bool odd_v = false;
    if constexpr (!kPlain) {
      uint32_t ok = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        ok |= static_cast<uint32_t>(k0 + 16 * (e >> 2) + 4 * g + (e & 3) < w.hi && page[e >> 2] >= 0) << e;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        keep[e] = (ok >> 2 * e & 1 ? 0xFFFFu : 0u) | (ok >> (2 * e + 1) & 1 ? 0xFFFF0000u : 0u);
      odd_v = __any(src.odd(ok, keep) != 0);
    }
#pragma unroll
    for (int x = 0; x < kV; ++x) {
      u32x4v a = src.v(x);
      if constexpr (!kPlain) {
        a &= keep;
        if (odd_v)
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] &= ~((odd_halves(a[e]) >> 15) * 0xFFFFu);
      }
#pragma unroll
      for (int t = 0; t < T; ++t) o[t][x] = dev::mfma_bf16(a, pw[t], o[t][x]);
    }
    if (!kPlain && odd_v) {                   // rare: the values taken out above, row by row
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int at = page_entry(p, w, k0 + 16 * b);
        const int64_t base = block_base<D>(p, w.h, at, k0 + 16 * b);
        for (int kk = 0; kk < 16; ++kk) {
          if (k0 + 16 * b + kk >= w.hi || at < 0) break;
          const uint16_t* vp = p.V + base + kk * D;
          const int from = 16 * (kk >> 2) + r;
#pragma unroll
          for (int t = 0; t < T; ++t) {
            float mine = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) mine = x == (kk & 3) ? in->s[t][4 * b + x] : mine;
            const float pk = __shfl(mine, from);
            const bool sees = (__shfl(static_cast<int>(in->seen[t]), from) >> (4 * b + (kk & 3))) & 1;
#pragma unroll
            for (int v = 0; v < kV; ++v)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint16_t x = vp[Source::dim(v, 4 * g + i)];
                if (sees && !finite_bf16(x)) o[t][v][i] += pk * dev::bf16_float(x);
              }
          }
        }
      }
    }
  }

  template <bool kPlain, typename Source>
  __device__ __forceinline__ void step(const TreeArgs& p, const Part& w, const Source& src, int k0,
                                       const int (&page)[2]) {
    Scores s;
    u32x4v k[2][kChunks], pw[T];
#pragma unroll
    for (int b = 0; b < 2; ++b) src.k(b, k[b]);
    scores<kPlain>(p, w, k, k0, page, &s);
    renew(p, s);
    weights(p, &s, pw);
    absorb<kPlain>(p, w, src, k0, page, &s, pw);
  }
};

// Values that another workgroup reads in this launch, perhaps on another XCD with an L2 of its
// own: device-scope accesses, 8 bytes each.
__device__ __forceinline__ void put(void* at, float a, float b) {
  const uint64_t x = static_cast<uint64_t>(__float_as_uint(b)) << 32 | __float_as_uint(a);
  __hip_atomic_store(static_cast<uint64_t*>(at), x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put(float* at, f32x4 v) {
  put(at, v[0], v[1]);
  put(at + 2, v[2], v[3]);
}
__device__ __forceinline__ float2 get(const void* at) {
  const uint64_t x =
      __hip_atomic_load(static_cast<const uint64_t*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return {__uint_as_float(static_cast<uint32_t>(x)), __uint_as_float(static_cast<uint32_t>(x >> 32))};
}

// The end of a narrow workgroup with one of several parts of a tile: the last of them to
// arrive joins the parts' (m, l, O), in an order that does not depend on who that is.  sh:
// LDS of kJoinFloats, no longer used for anything else.
template <int D>
constexpr int kJoinCols = D <= 128 ? 4 : 1;                  // columns at a time
constexpr int kJoinWeights = 16 * (2 * kMaxSplits + 1);
template <int D, int kN>
constexpr int kJoinFloats = kJoinWeights + 2 * kJoinCols<D> * 64 * kN;

template <int D, int kN>
__device__ __forceinline__ void join_parts(const TreeArgs& p, const Part& w, float* sh) {
  constexpr int kThreads = 64 * kN, kCols = kJoinCols<D>;
  __shared__ int sh_last;
  const int tid = static_cast<int>(threadIdx.x);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // what this wave has put is there
  __syncthreads();
  uint32_t* const arrived = p.arrived + w.first_slot * p.Hk + w.h;
  if (tid == 0)
    sh_last = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
              static_cast<uint32_t>(w.splits - 1);
  __syncthreads();
  if (!sh_last) return;
  if (tid == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  auto part = [&](int s) { return (static_cast<int64_t>(w.first_slot + w.tiles * s) * p.Hk + w.h) * 16; };
  // A thread's two elements of every kGroups-th part, kCols columns at a time; the
  // first ones under way before their weights are known.
  constexpr int kPairs = D / 2, kGroups = kThreads / kPairs, kEach = kMaxSplits / kGroups;
  const int pair = tid % kPairs, group = tid / kPairs;
  float2 in[kCols][kEach];
  auto load = [&](int c0) {
#pragma unroll
    for (int c = 0; c < kCols; ++c)
#pragma unroll
      for (int y = 0; y < kEach; ++y)
        if (c0 + c < w.cols && group + kGroups * y < w.splits)
          in[c][y] = get(p.part_o + (part(group + kGroups * y) + c0 + c) * D + 2 * pair);
  };
  load(0);
  // Each part's maximum, then its weight, in each column; its sum; 1 / the column's sum.
  float* const weight = sh;                                  // [column][part]
  float* const l = weight + 16 * kMaxSplits;                 // [column][part]
  float* const inv = l + 16 * kMaxSplits;
  float* const red = sh + kJoinWeights;                      // [group][column][D]
  for (int e = tid; e < w.cols * w.splits; e += kThreads) {
    const int c = e / w.splits, s = e - c * w.splits;
    const float2 ml = get(p.part_ml + part(s) + c);
    weight[c * kMaxSplits + s] = ml.x;
    l[c * kMaxSplits + s] = ml.y;
  }
  __syncthreads();
  for (int c = tid >> 6; c < w.cols; c += kN) {         // a wave a column
    const int s = tid & 63;
    const float m = s < w.splits ? weight[c * kMaxSplits + s] : kNone;
    const float top = dev::wave_max(m), a = exp2_from(m, top, 1.0f);
    const float sum = dev::wave_sum(s < w.splits ? a * l[c * kMaxSplits + s] : 0.f);
    weight[c * kMaxSplits + s] = a;
    if (s == 0) {
      inv[c] = sum == 0.f ? 0.f : 1.0f / sum;
      if (p.lse) p.lse[head_of(p, w, c)] = sum == 0.f ? kNone : (top + log2f(sum)) * 0.69314718055994531f;
    }
  }
  __syncthreads();
  for (int c0 = 0; c0 < w.cols; c0 += kCols) {
    if (c0) load(c0);
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      float2 o = {0.f, 0.f};
#pragma unroll
      for (int y = 0; y < kEach; ++y)
        if (c0 + c < w.cols && group + kGroups * y < w.splits) {
          const float a = weight[(c0 + c) * kMaxSplits + group + kGroups * y];
          if (a != 0.f) {                                    // a part that a row saw nothing of adds nothing
            o.x += a * in[c][y].x;
            o.y += a * in[c][y].y;
          }
        }
      *reinterpret_cast<float2*>(red + (group * kCols + c) * D + 2 * pair) = o;
    }
    __syncthreads();
    for (int x = tid; x < kCols * kPairs; x += kThreads) {
      const int c = x / kPairs, d = 2 * (x % kPairs);
      if (c0 + c < w.cols) {
        float2 o = {0.f, 0.f};
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          const float2 y = *reinterpret_cast<const float2*>(red + (g * kCols + c) * D + d);
          o.x += y.x;
          o.y += y.y;
        }
        *reinterpret_cast<uint32_t*>(p.out + head_of(p, w, c0 + c) * D + d) =
            dev::pack_bf16(o.x * inv[c0 + c], o.y * inv[c0 + c]);
      }
    }
    __syncthreads();
  }
}

// Up to 16 query columns: the waves take every kN-th 32 keys each, straight into
// registers, the next ones under way, and join through LDS at the end.
template <int D, int kN>
__global__ __launch_bounds__(64 * kN, D <= 128 ? 2 : 1) void tree_attention_kernel(const TreeArgs p) {
  constexpr int kV = D / 16, kPitch = D + 4, kThreads = 64 * kN, kStride = 32 * kN;
  __shared__ __align__(16) float sh_o[kN][16][kPitch];
  static_assert(kN * 16 * kPitch >= (kJoinFloats<D, kN>), "the join's LDS");
  __shared__ float sh_m[kN][16], sh_l[kN][16];
  Part w;
  if (!find_part(p, 16, &w)) return;
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int first = w.lo + 32 * wave;
  const int steps = w.hi > first ? (w.hi - first + kStride - 1) / kStride : 0;
  // lane 2 s + b: page of block b of step s (of 32 steps)
  int entries = page_entry(p, w, first + kStride * (lane >> 1) + 16 * (lane & 1));
  int page[2];
  auto load = [&](int step, Tile<D>* tile) {
    int64_t base[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      page[b] = __builtin_amdgcn_readlane(entries, 2 * (step & 31) + b);
      base[b] = block_base<D>(p, w.h, page[b], first + kStride * step + 16 * b);
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
        entries = page_entry(p, w, first + kStride * (step + 1 + (lane >> 1)) + 16 * (lane & 1));
      load(step + 1, &next);
    }
    q.template step<decltype(plain)::value>(p, w, now, first + kStride * step, page_now);
    if (step + 1 < steps) now = next;
  };
  // every row sees the whole step: of cached tokens alone, on pages of the pool
  int step = 0;
  for (; step < steps && first + kStride * step + 32 <= min(w.cached, w.hi) && (page[0] | page[1]) >= 0; ++step)
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
  auto top_of = [&](int c) {
    float top = sh_m[0][c];
#pragma unroll
    for (int y = 1; y < kN; ++y) top = max_of(top, sh_m[y][c]);
    return top;
  };
  const float a = exp2_from(q.m[0], top_of(r), p.scale);
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
    const float top = top_of(c);
    float sum = 0.f;
    f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll
    for (int y = 0; y < kN; ++y) {
      sum += sh_l[y][c] * exp2_from(sh_m[y][c], top, p.scale);
      lo += *reinterpret_cast<const f32x4*>(&sh_o[y][c][d]);
      hi += *reinterpret_cast<const f32x4*>(&sh_o[y][c][d + 4]);
    }
    const int64_t head = head_of(p, w, c);
    if (w.splits == 1) {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      const u32x4v y = {dev::pack_bf16(lo[0] * inv, lo[1] * inv), dev::pack_bf16(lo[2] * inv, lo[3] * inv),
                        dev::pack_bf16(hi[0] * inv, hi[1] * inv), dev::pack_bf16(hi[2] * inv, hi[3] * inv)};
      *reinterpret_cast<u32x4v*>(p.out + head * D + d) = y;
      if (p.lse && d == 0) p.lse[head] = sum == 0.f ? kNone : (top * p.scale + log2f(sum)) * 0.69314718055994531f;
    } else {
      const int64_t part = static_cast<int64_t>(blockIdx.x) * 16 + c;
      put(p.part_o + part * D + d, lo);
      put(p.part_o + part * D + d + 4, hi);
      if (d == 0) put(p.part_ml + part, top * p.scale, sum);
    }
  }
  if (w.splits > 1) join_parts<D, kN>(p, w, &sh_o[0][0][0]);
}

// Copies 16 bytes a lane straight to LDS: from src (the same for the wave) + the lane's
// offset, lane l's to lds + 16 l (LDS address, the same for the wave).
__device__ __forceinline__ void lds_copy16(const void* src, uint32_t bytes, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(bytes), "s"(src), "s"(lds)
               : "memory", "m0");
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
template <typename T>
using InLds = const __attribute__((address_space(3))) T*;

// K and V of a stage in LDS.  Unit u (16 bytes) of row k lies at unit u ^ turn(k), so that
// neither a K read (a unit of 16 rows) nor a V read (32 bytes of 8 rows at a time) conflicts.
template <int D>
struct Staged {
  static __device__ __forceinline__ int turn_k(int k) { return D == 64 ? (k >> 1) & 7 : k & 15; }
  static __device__ __forceinline__ int turn_v(int k) { return D == 64 ? k & 6 : 2 * (k & 7); }
  // A lane's own places in a stage (bytes): unit g of row r; dims 4 (r % 4) .. of row 4 g + r / 4.
  static __device__ __forceinline__ uint32_t k_lane(int r, int g) { return 2 * r * D + 16 * (g ^ turn_k(r)); }
  static __device__ __forceinline__ uint32_t v_lane(int r, int g) {
    const int k = 4 * g + (r >> 2);
    return 2 * k * D + 16 * turn_v(k) + 8 * (r & 3);
  }

  uint32_t k_at, v_at;                   // LDS addresses: those in the stage

  // (the blocks are 16 rows apart, and the turns have a row's low bits alone)
  __device__ __forceinline__ void k(int b, u32x4v (&out)[D / 32]) const {
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      out[c] = *reinterpret_cast<InLds<u32x4v>>(static_cast<uintptr_t>((k_at ^ 64 * c) + 32 * b * D));
  }
  // Transposed as they are read: of 16 lanes, four to a row's 16 dims, lane i gets dim i of
  // the four rows.
  __device__ __forceinline__ u32x4v v(int x) const {
    u32x4v out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto at = static_cast<uintptr_t>((v_at ^ 32 * x) + 32 * h * D);
      const dev::u32x2 y = __builtin_bit_cast(
          dev::u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at)));
      out[2 * h] = y.x;
      out[2 * h + 1] = y.y;
    }
    return out;
  }
  __device__ __forceinline__ uint32_t odd(uint32_t, const u32x4v& keep) const {
    uint32_t out = 0;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
      const u32x4v a = v(x) & keep;
#pragma unroll
      for (int e = 0; e < 4; ++e) out |= odd_halves(a[e]);
    }
    return out;
  }
  static __device__ __forceinline__ int dim(int x, int m) { return 16 * x + m; }
};

// V^T's operands of a stage, read from LDS.
template <int D>
struct Taken {
  u32x4v values[D / 16];
  __device__ __forceinline__ void take(const Staged<D>& src, int from, int to) {
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
      if (x >= from && x < to) values[x] = src.v(x);
  }
  __device__ __forceinline__ u32x4v v(int x) const { return values[x]; }
  static __device__ __forceinline__ int dim(int x, int m) { return Staged<D>::dim(x, m); }
};

// More columns: each of kN waves its own 1 .. T tiles of them, all waves the same keys, K and
// V copied to LDS 32 keys (a stage) at a time, kAhead stages ahead.  Within a wave a stage's
// scores are formed beside the exponentials of the one before it, and its keys are read from
// LDS beside the second product of the one before that, so that neither unit waits for the
// other or for LDS.  A wave in the first of these phases goes first: the second one, products
// alone, leaves room for it (236 -> 228 us).
template <int D, int T, int kN>
__global__ __launch_bounds__(64 * kN, D <= 128 ? 2 : 1) void tree_attention_wide_kernel(const TreeArgs p) {
  constexpr int kV = D / 16, kKeys = 32, kThreads = 64 * kN;
  constexpr int kAhead = kN == 8 ? 6 : 2;                    // even
  // Stages in LDS: under way, and the two whose keys are read; for V also the two behind them.
  constexpr int kKeyBuffers = kAhead + 2, kValueBuffers = kAhead + 4;
  constexpr int kUnits = D / 8, kRows = 64 / kUnits;         // 16 bytes of a row; rows a copy
  constexpr int kEach = kKeys / kRows, kCopies = 2 * kEach / kN;         // copies of K; a wave's
  constexpr int kStage = kKeys * D;                          // of K or of V
  __shared__ __align__(1024) uint16_t sh[(kKeyBuffers + kValueBuffers) * kStage];
  Part w;
  if (!find_part(p, 16 * T * kN, &w)) return;
  if (p.split && w.h == 0 && static_cast<int>(blockIdx.x) / p.Hk == w.first_slot)      // for the join
    for (int row = w.c0 / p.G + static_cast<int>(threadIdx.x); row * p.G < w.c0 + w.cols; row += kThreads)
      p.joins[w.first + row] = {w.first, w.first_slot - w.c0 / (16 * T * kN), w.tiles, w.segment << 8 | w.splits};
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const uint32_t sh_at = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)(sh)));
  // The columns in tiles of 16, as many to each SIMD (a wave or two of the workgroup): a
  // SIMD's second wave has one the less, or as many.
  const int tiles = (w.cols + 15) / 16, simd = wave % 4;
  const int simd_tiles = tiles / 4 + (simd < tiles % 4), second = kN == 8 ? simd_tiles / 2 : 0;
  const int mine = wave < 4 ? simd_tiles - second : second;
  const int tile0 = simd * (tiles / 4) + min(simd, tiles % 4) + (wave < 4 ? 0 : simd_tiles - second);
  const int stages = (w.hi - w.lo + kKeys - 1) / kKeys;
  // Stages that every row sees whole: of cached tokens alone, on pages of the pool (as far
  // as the entries at hand say).
  int plain = max(min(w.cached, w.hi) - w.lo, 0) / kKeys;
  // A stage's place in LDS (bytes) follows the one before it, around a ring.
  auto keys_after = [&](uint32_t at) { return at == (kKeyBuffers - 1) * 2 * kStage ? 0 : at + 2 * kStage; };
  auto values_after = [&](uint32_t at) {
    return at == (kKeyBuffers + kValueBuffers - 1) * 2 * kStage ? kKeyBuffers * 2 * kStage : at + 2 * kStage;
  };

  // A stage's rows are copied kRows to a wave copy (a kilobyte), lane i to unit i of it.
  // (Stages past the last are copied from the pool's first page, so that as many are always
  // under way.)
  int64_t entry = 0;                     // lane b: byte offset of block b (of 64)
  uint64_t there = 0, before = 0;        // which of them are on a page, and of the 64 before them
  int looked_up = 0;                     // the stage of the first
  uint32_t load_k = 0, load_v = kKeyBuffers * 2 * kStage;    // of the next stage to load
  auto look_up = [&](int stage) {        // before the load of a stage that starts 64 blocks
    if (stage % 32) return;
    const int key = w.lo + kKeys * stage + 16 * lane, page = page_entry(p, w, key);
    entry = 2 * block_base<D>(p, w.h, page, key);
    before = there;
    there = __ballot(page >= 0);
    looked_up = stage;
    if (__any(key < w.hi && page < 0)) plain = min(plain, stage);
  };
  uint32_t of[kCopies];                  // a lane's place in its block
#pragma unroll
  for (int x = 0; x < kCopies; ++x) {
    const int c = wave + kN * x, k = kRows * (c % kEach) % 16 + lane / kUnits, unit = lane % kUnits;
    of[x] = 2 * k * D + 16 * (unit ^ (c < kEach ? Staged<D>::turn_k(k) : Staged<D>::turn_v(k)));
  }
  auto load = [&](int stage) {
#pragma unroll
    for (int x = 0; x < kCopies; ++x) {
      const int c = wave + kN * x, rows = c % kEach;         // rows kRows rows .. of the stage
      const int b = (2 * stage + kRows * rows / 16) & 63;
      const uint64_t at = static_cast<uint64_t>(static_cast<uint32_t>(
                              __builtin_amdgcn_readlane(static_cast<int>(entry >> 32), b))) << 32 |
                          static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(entry), b));
      lds_copy16(reinterpret_cast<const char*>(c < kEach ? p.K : p.V) + at, of[x],
                 sh_at + (c < kEach ? load_k : load_v) + rows * 1024);
    }
    load_k = keys_after(load_k);
    load_v = values_after(load_v);
  };
  // A stage's copies are there (a wave's end in order, and the later stages' are under way):
  // the next load takes buffers whose last readers are behind this barrier.
  auto arrive = [&] {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kAhead - 2) * kCopies) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto enter = [&](int stage) {
    look_up(stage + kAhead);
    arrive();
    load(stage + kAhead);
  };
  if (stages > 0) {
    look_up(0);
    for (int stage = 0; stage < kAhead; ++stage) load(stage);
  }
  uint32_t read_k = 0, read_v = kKeyBuffers * 2 * kStage;    // of the next stage to read
  const uint32_t k_lane = sh_at + Staged<D>::k_lane(r, g), v_lane = sh_at + Staged<D>::v_lane(r, g);
  auto work = [&](auto count) {
    constexpr int kT = decltype(count)::value;
    Wave<D, kT> q;
    q.start(p, w, w.c0 + 16 * tile0);
    using Scores = typename Wave<D, kT>::Scores;
    constexpr int kNoPage[2] = {0, 0};
    Scores now, after;
    u32x4v k[2][D / 32], pw[kT];
    auto read_keys = [&] {
      const Staged<D> src{read_k + k_lane, 0};
      src.k(0, k[0]);
      src.k(1, k[1]);
      read_k = keys_after(read_k);
    };
    if (plain > 0) {
      enter(0);
      read_keys();
      q.template scores<true>(p, w, k, 0, kNoPage, &now);
      q.renew(p, now);
      enter(1);
      read_keys();
      for (int stage = 0; stage + 1 < plain; ++stage) {
        if (!(stage & 1)) look_up(stage + 2 + kAhead);
        Taken<D> values;
        const Staged<D> src{0, read_v + v_lane};
        read_v = values_after(read_v);
        values.take(src, 0, kV / 2);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        q.template scores<true>(p, w, k, 0, kNoPage, &after);
        q.weights(p, &now, pw);
#pragma unroll
        for (int t = 0; t < kT; ++t) asm volatile("" : "+v"(pw[t]));     // here, not after the barrier
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        values.take(src, kV / 2, kV);
        if (!(stage & 1)) {              // two stages, if only to wait: they may not be plain, or none
          arrive();
          load(stage + 2 + kAhead);
          load(stage + 3 + kAhead);
        }
        read_keys();
        __builtin_amdgcn_sched_barrier(0);
        q.template absorb<true>(p, w, values, 0, kNoPage, &now, pw);
        now = after;
        q.renew(p, now);
      }
      q.weights(p, &now, pw);
      q.template absorb<true>(p, w, Staged<D>{0, read_v + v_lane}, 0, kNoPage, &now, pw);
    }
    // plain > 0: stage `plain` has been entered, and one more if it is even
    read_k = plain % kKeyBuffers * 2 * kStage;
    read_v = (kKeyBuffers + plain % kValueBuffers) * 2 * kStage;
    for (int stage = plain; stage < stages; ++stage) {
      if (stage > plain + 1 - (plain & 1) || plain == 0) enter(stage);
      const int k0 = w.lo + kKeys * stage;
      const uint64_t on = (stage >= looked_up ? there : before) >> (2 * stage & 63);
      const int page[2] = {on & 1 ? 0 : -1, on & 2 ? 0 : -1};
      q.template step<false>(p, w, Staged<D>{read_k + k_lane, read_v + v_lane}, k0, page);
      read_k = keys_after(read_k);
      read_v = values_after(read_v);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // no copy outlives the workgroup

#pragma unroll
    for (int t = 0; t < kT; ++t) {
      float sum = q.l[t];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      const int c = 16 * (tile0 + t) + r;
      if (c >= w.cols) continue;
      const int64_t head = head_of(p, w, c);
      const float top = q.m[t] * p.scale;
      if (w.splits == 1) {
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
        for (int x = 0; x < kV; ++x) {
          const dev::u32x2 y = {dev::pack_bf16(q.o[t][x][0] * inv, q.o[t][x][1] * inv),
                                dev::pack_bf16(q.o[t][x][2] * inv, q.o[t][x][3] * inv)};
          *reinterpret_cast<dev::u32x2*>(p.out + head * D + 16 * x + 4 * g) = y;
        }
        if (p.lse && g == 0) p.lse[head] = sum == 0.f ? kNone : (top + log2f(sum)) * 0.69314718055994531f;
      } else {
        const int64_t part = static_cast<int64_t>(blockIdx.x) * (16 * T * kN) + c;
#pragma unroll
        for (int x = 0; x < kV; ++x) *reinterpret_cast<f32x4*>(p.part_o + part * D + 16 * x + 4 * g) = q.o[t][x];
        if (g == 0) p.part_ml[part] = {top, sum};
      }
    }
  };
  if constexpr (T == 2) {
    if (mine == 2) return work(std::integral_constant<int, 2>{});
  }
  if (mine == 1) return work(std::integral_constant<int, 1>{});
  // a wave without columns only helps to load
  if (plain > 0) {
    enter(0);
    enter(1);
    for (int stage = 0; stage + 1 < plain; stage += 2) {
      look_up(stage + 2 + kAhead);
      arrive();
      load(stage + 2 + kAhead);
      load(stage + 3 + kAhead);
    }
  }
  for (int stage = plain > 0 ? plain + 2 - (plain & 1) : 0; stage < stages; ++stage) enter(stage);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// After the wide kernel: the parts' (m, l, O) of one row and head, a wave each; nothing
// where a workgroup had all of the row's keys.  What `joins` holds for a row of no request is
// an earlier call's, or anything: an entry counts if the request that it names has the row
// (of such a row it is this call's); the parts' places are clamped to the workspace, so
// that their loads need not wait to know.
constexpr int kJoinWaves = 4;
template <int D>
__global__ __launch_bounds__(64 * kJoinWaves) void tree_join_kernel(const float* __restrict__ part_o,
                                                             const float2* __restrict__ part_ml,
                                                             const int4* __restrict__ joins,
                                                             const int32_t* __restrict__ offsets, int B,
                                                             int64_t heads, int Hq, int Hk, int tile_cols, int slots,
                                                             uint16_t* __restrict__ out, float* __restrict__ lse) {
  constexpr int kPer = D / 4, kAtOnce = 64 / kPer;     // lanes a part, parts a load
  constexpr int kBatch = 8;                            // loads under way
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int64_t head = static_cast<int64_t>(blockIdx.x) * kJoinWaves + (threadIdx.x >> 6);
  if (head >= heads) return;
  const int64_t row = head / Hq;
  const int4 j = joins[row];
  const int splits = __builtin_amdgcn_readfirstlane(j.w & 255), segment = __builtin_amdgcn_readfirstlane(j.w >> 8);
  if (splits <= 1 || splits > kMaxSplits || segment < 0 || segment >= B) return;
  const int first = offsets[segment], end = offsets[segment + 1];
  const int G = Hq / Hk, q = static_cast<int>(head - row * Hq);
  const uint32_t c = static_cast<uint32_t>((row - j.x) * G + q % G);
  const int col = static_cast<int>(c % tile_cols), tile = static_cast<int>(c / tile_cols);
  auto at = [&](int s) {
    const int64_t slot = j.y + static_cast<int64_t>(s) * j.z + tile;
    return (min(max(slot, int64_t{0}), static_cast<int64_t>(slots - 1)) * Hk + q / G) * tile_cols + col;
  };
  float2 ml = {kNone, 0.f};
  if (lane < splits) ml = part_ml[at(lane)];
  f32x4 in[kBatch];
  auto load = [&](int s0) {
#pragma unroll
    for (int x = 0; x < kBatch; ++x)
      if (s0 + x * kAtOnce < splits)
        in[x] = *reinterpret_cast<const f32x4*>(
            part_o + at(min(s0 + x * kAtOnce + lane / kPer, splits - 1)) * D + 4 * (lane % kPer));
  };
  load(0);
  if (row < first || row >= end) return;
  const float top = dev::wave_max(ml.x), a = exp2_from(ml.x, top, 1.0f), sum = dev::wave_sum(a * ml.y);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += kBatch * kAtOnce) {
    if (s0 > 0) load(s0);
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      if (s0 + x * kAtOnce >= splits) break;
      const int s = s0 + x * kAtOnce + lane / kPer;
      const float w = __shfl(a, s & 63);
      if (s < splits && w != 0.f) o += w * in[x];      // a part that a row saw nothing of adds nothing
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
void launch(const TreeArgs& p, int tile_cols, int waves, int64_t blocks, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(blocks));
  if (tile_cols == 16 && waves == 4)
    tree_attention_kernel<D, 4><<<grid, 256, 0, stream>>>(p);
  else if (tile_cols == 16) {
    if constexpr (D <= 128) tree_attention_kernel<D, 8><<<grid, 512, 0, stream>>>(p);
  }
  else if (tile_cols == 64)
    tree_attention_wide_kernel<D, 1, 4><<<grid, 256, 0, stream>>>(p);
  else if constexpr (D <= 128) {
    if (tile_cols == 128)
      tree_attention_wide_kernel<D, 2, 4><<<grid, 256, 0, stream>>>(p);
    else
      tree_attention_wide_kernel<D, 2, 8><<<grid, 512, 0, stream>>>(p);
  }
  if (p.split && tile_cols > 16) {
    const int64_t heads = static_cast<int64_t>(p.M) * p.Hq;
    tree_join_kernel<D><<<dim3(static_cast<unsigned>((heads + kJoinWaves - 1) / kJoinWaves)), 64 * kJoinWaves, 0,
                          stream>>>(p.part_o, p.part_ml, p.joins, p.offsets, p.B, heads, p.Hq, p.Hk, tile_cols,
                                    p.slots, p.out, p.lse);
  }
}

}  // namespace

TreePlan plan_tree_attention(int M, int B, int Hq, int Hk, int D, int max_kv_len, int num_cus) {
  TreePlan c;
  const int64_t G = Hq / Hk;
  const int64_t used = std::max(1, std::min(M, B));
  const int64_t per = (M * G + used - 1) / used;        // query columns of a mean request
  // (188 columns a request over 32 k tokens, heads of 128: 256 / 128 columns a workgroup 247 / 258 us)
  c.tile_cols = per <= 16 ? 16 : per <= 64 || D > 128 ? 64 : per <= 128 ? 128 : 256;
  const int64_t tiles = most_tiles(M, B, G, c.tile_cols);
  // Slots a kv head: as many as the chip holds workgroups at once (by their registers and
  // LDS), but no more than there are parts; where the tiles alone are that many, some for
  // requests that are longer than the others.
  // (heads of 64, 64 columns, of which four would fit: 1 / 2 / 3 / 4 a CU 29.2 / 24.1 / 25.7 / 25.8 us,
  // trees of up to 13 nodes over 6 x 8 k tokens)
  const int per_cu = c.tile_cols == 16 || c.tile_cols == 256 || D > 128 ? 1 : 2;
  const int64_t at_once = std::max<int64_t>(static_cast<int64_t>(per_cu) * num_cus / Hk, 1);
  c.spread = tiles >= at_once;
  // Waves of a narrow workgroup: eight while a request has several of them, or is long; four,
  // two workgroups a CU, where short requests alone fill the chip and one's start and end hide
  // behind another's loads.  us, eight / four, 8 kv heads of 128, requests of up to as many tokens:
  // 1 x 4097 13.6 / 15.7, 16 x 1000 18.5 / 19.7, 32 x 300 19.7 / 12.1, 128 x 500 56.7 / 45.8,
  // 64 x 2000 83 / 80, 40 x 4000 112 / 121; 12 heads of 64: 50 x 1000 30.7 / 26.3, 50 x 2000
  // 55 / 54, 50 x 3000 74 / 77.  (Heads of 256 leave registers for four.)
  c.waves = D > 128 || (c.spread && max_kv_len <= 2048) ? 4 : 8;
  c.step = c.tile_cols == 16 ? 32 * c.waves : 128;
  const int64_t steps = (static_cast<int64_t>(max_kv_len) + c.step - 1) / c.step;
  const int64_t parts = tiles * std::min<int64_t>(kMaxSplits, std::max<int64_t>(steps, 1));
  c.slots = c.spread ? tiles + (2 * tiles + 2) / 3 : std::max(tiles, std::min(at_once, parts));
  c.split = c.slots > tiles && tiles < 4 * at_once &&
            c.slots * Hk * static_cast<int64_t>(sizeof(uint32_t)) <= static_cast<int64_t>(kWorkspaceStateBytes);
  if (!c.split) c.slots = tiles;
  c.blocks = c.slots * Hk;
  return c;
}

size_t tree_workspace_bytes(const TreePlan& c, int M, int D) {
  if (!c.split) return 0;
  return kWorkspaceStateBytes + static_cast<size_t>(c.blocks) * c.tile_cols * (D + 2) * 4 +
         static_cast<size_t>(M) * sizeof(int4);
}

hipError_t launch_tree_attention(const TreePlan& c, const uint16_t* q, int64_t ld_q, int M, int Hq, int Hk, int D,
                                 const PagedCache& cache, const int32_t* pages, int64_t ld_pages, int max_keys,
                                 const int32_t* cached, const int32_t* offsets, int B, float scale,
                                 const uint8_t* mask, int64_t ld_mask, int mask_wide, uint16_t* out, float* lse,
                                 void* workspace, hipStream_t stream) {
  const int64_t cols = c.blocks * c.tile_cols;
  uint32_t* const arrived = static_cast<uint32_t*>(workspace);         // the state head
  char* const parts = static_cast<char*>(workspace) + kWorkspaceStateBytes;
  float* const part_o = c.split ? reinterpret_cast<float*>(parts) : nullptr;
  float2* const part_ml = c.split ? reinterpret_cast<float2*>(part_o + cols * D) : nullptr;
  int4* const joins = c.split ? reinterpret_cast<int4*>(part_ml + cols) : nullptr;
  // A negative scale turns the queries' signs; 0 is as good as the smallest used here
  // (q . k times it vanishes beside 1) and keeps an unseen -inf from becoming 0 x inf.
  const float size = std::max(std::fabs(scale) * 1.44269504088896341f, 0x1p-100f);
  const TreeArgs p{q, ld_q, cache.K, cache.V, cache.page_stride, cache.page_shift, cache.num_pages, pages, ld_pages,
                   max_keys, cached, offsets, mask, ld_mask, mask ? mask_wide : 0, size, kSlack / size,
                   std::signbit(scale) ? 0x80008000u : 0u, out, lse, part_o, part_ml, arrived, joins, M, B, Hq, Hk,
                   Hq / Hk, static_cast<int>(c.slots), c.step, c.split, c.spread};
  if (D == 64) launch<64>(p, c.tile_cols, c.waves, c.blocks, stream);
  else if (D == 128) launch<128>(p, c.tile_cols, c.waves, c.blocks, stream);
  else launch<256>(p, c.tile_cols, c.waves, c.blocks, stream);
  return hipGetLastError();
}

}  // namespace prq
