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
// (32 v_perm per 32 x 128 tile); nothing goes through LDS until the waves' results
// are joined.  The 16 queries of a product's column side are the G query heads of
// the kv head for 16 / G tokens, 1, 2 or 4 such tiles a wave.
//
// The maximum is kept per lane group and only joined across the groups when a score
// passes it by 8 (powers of two): until then the stale maximum serves, P up to 2^8.
// Scores, statistics and O are float32; P is rounded to bf16 for its product (relative
// error 2^-9 each, as large as the rounding of the output; the sum that divides takes
// the unrounded P).
//
// Few rows leave most CUs idle, so the keys are split over workgroups and the partial
// (m, l, O) joined by a second kernel in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;
using dev::u32x4v;

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kStep = 32 * kWaves;       // keys a workgroup takes at a time
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
  float scale;                           // times log2 e
  uint16_t* out;
  float *lse, *part_o;
  float2* part_ml;
  int M, B, Hq, Hk, G, tiles, splits, split_len;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// exp2(a - b), 0 where a is -inf (b may be, too).
__device__ __forceinline__ float exp2_from(float a, float b) { return a == kNone ? 0.f : exp2_fast(a - b); }

template <int D>
struct Tile {                            // K and V of 32 keys, as a lane holds them
  static constexpr int kChunks = D / 32, kWords = D / 32;
  u32x4v k[2][kChunks];                  // keys l % 16 of two 16-key blocks, dims 32 c + 8 g ..
  uint32_t v[8][kWords];                 // keys 4 g .. + 3 of both blocks, dims (D / 16) (l % 16) ..
};

template <int D>
__device__ __forceinline__ void load_tile(const TreeArgs& p, const int64_t (&base)[2], Tile<D>* t) {
  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint16_t* kp = p.K + base[b] + r * D + 8 * g;
#pragma unroll
    for (int c = 0; c < Tile<D>::kChunks; ++c) t->k[b][c] = *reinterpret_cast<const u32x4v*>(kp + 32 * c);
  }
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint16_t* vp = p.V + base[b] + 4 * g * D + r * (D / 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (D == 64) {
        const dev::u32x2 w = *reinterpret_cast<const dev::u32x2*>(vp + i * D);
        t->v[4 * b + i][0] = w.x;
        t->v[4 * b + i][1] = w.y;
      } else {
#pragma unroll
        for (int c = 0; c < D / 128; ++c) {
          const u32x4v w = *reinterpret_cast<const u32x4v*>(vp + i * D + 8 * c);
#pragma unroll
          for (int e = 0; e < 4; ++e) t->v[4 * b + i][4 * c + e] = w[e];
        }
      }
    }
  }
}

__device__ __forceinline__ bool word_finite(uint32_t w) {
  return (w & 0x7F80u) != 0x7F80u && (w & 0x7F800000u) != 0x7F800000u;
}

template <int D, int T>
__global__ __launch_bounds__(kThreads, T == 1 && D <= 128 ? 2 : 1) void tree_attention_kernel(const TreeArgs p) {
  constexpr int kCols = 16 * T, kChunks = D / 32, kV = D / 16, kPitch = D + 4;
  __shared__ __align__(16) float sh_o[kWaves][kCols][kPitch];
  __shared__ float sh_m[kWaves][kCols], sh_l[kWaves][kCols];

  const int lane = static_cast<int>(threadIdx.x) & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
  const int h = static_cast<int>(blockIdx.x) % p.Hk;
  const int rest = static_cast<int>(blockIdx.x) / p.Hk;
  const int split = rest / p.tiles;
  const dev::TileAt at = dev::find_tile(p.offsets, p.B, p.M, rest % p.tiles, p.G, kCols);
  if (at.segment < 0) return;
  const int c0 = at.tile * kCols;
  const int cols = min(at.rows * p.G - c0, kCols);
  const int cached = min(max(p.cached[at.segment], 0), p.max_keys);
  const int keys = min(at.rows, p.max_keys - cached) + cached;
  const int lo = split * p.split_len;
  const int hi = split == p.splits - 1 ? keys : min(keys, lo + p.split_len);
  if (p.splits > 1 && hi <= lo) {        // nothing here for this request: say so to the join
    if (static_cast<int>(threadIdx.x) < cols) {
      const int c = c0 + static_cast<int>(threadIdx.x);
      const int64_t row = at.first + c / p.G;
      p.part_ml[(split * static_cast<int64_t>(p.M) + row) * p.Hq + h * p.G + c % p.G] = {kNone, 0.f};
    }
    return;
  }

  // Queries: column r of tile t is token c / G, head h G + c % G.
  u32x4v q[T][kChunks];
  int token[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int c = c0 + 16 * t + r;
    token[t] = min(c / p.G, at.rows - 1);
    const uint16_t* qp = p.q + (at.first + token[t]) * p.ld_q + (h * p.G + c % p.G) * D + 8 * g;
#pragma unroll
    for (int k = 0; k < kChunks; ++k) q[t][k] = *reinterpret_cast<const u32x4v*>(qp + 32 * k);
  }

  f32x4 o[T][kV];
  float m[T], l[T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    m[t] = kNone;
    l[t] = 0.f;
#pragma unroll
    for (int v = 0; v < kV; ++v) o[t][v] = {0.f, 0.f, 0.f, 0.f};
  }

  const int in_page = (1 << p.page_shift) - 1;
  const int32_t* table = p.pages + at.segment * p.ld_pages;
  const int first = lo + 32 * wave;
  const int steps = hi > first ? (hi - first + kStep - 1) / kStep : 0;
  int entries = -1;                      // lane 2 s + b: page of block b of step s (of 32 steps)
  auto load_entries = [&](int step) {
    const int key = first + kStep * (step + (lane >> 1)) + 16 * (lane & 1);
    entries = key < hi ? table[key >> p.page_shift] : -1;
    if (entries >= p.num_pages) entries = -1;
  };
  // Element offsets of a step's two blocks; a block past the keys, or on a page
  // outside the pool, reads the pool's first page, and its keys are not seen.
  int64_t base[2];
  bool held[2];
  auto find = [&](int step) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int page = __builtin_amdgcn_readlane(entries, 2 * (step & 31) + b);
      const int key = first + kStep * step + 16 * b;
      held[b] = page >= 0;
      base[b] = held[b] ? page * p.page_stride +
                              ((static_cast<int64_t>(h) << p.page_shift) + (key & in_page)) * D
                        : 0;
    }
  };

  Tile<D> now, next;
  bool held_now[2] = {false, false};
  int64_t base_now[2] = {0, 0};
  if (steps > 0) {
    load_entries(0);
    find(0);
    load_tile<D>(p, base, &now);
  }
  for (int step = 0; step < steps; ++step) {
    held_now[0] = held[0];
    held_now[1] = held[1];
    base_now[0] = base[0];
    base_now[1] = base[1];
    if (step + 1 < steps) {
      if (((step + 1) & 31) == 0) load_entries(step + 1);
      find(step + 1);
      load_tile<D>(p, base, &next);
    }
    const int k0 = first + kStep * step;
    float s[T][8];
#pragma unroll
    for (int t = 0; t < T; ++t) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < kChunks; ++c) x = dev::mfma_bf16(now.k[b][c], q[t][c], x);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][4 * b + i] = x[i] * p.scale;
      }
    }
    const bool plain = k0 + 32 <= cached && held_now[0] && held_now[1];
    uint32_t seen[T];
    bool odd_v = false;                  // some drafted key's V holds an infinity or a NaN
    if (!plain) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const uint8_t* see = p.mask ? p.mask + (at.first + token[t]) * p.ld_mask : nullptr;
        seen[t] = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int key = k0 + 16 * (e >> 2) + 4 * g + (e & 3);
          const int j = key - cached;
          bool ok = key < hi && held_now[e >> 2];
          if (ok && j >= 0) ok = see ? j < p.mask_wide && see[j] != 0 : j <= token[t];
          if (ok)
            seen[t] |= 1u << e;
          else
            s[t][e] = kNone;
        }
      }
      // What no row may see must not reach the product either (0 x NaN): V past the
      // keys becomes 0, and infinities and NaN are taken out and added below for the
      // rows that do see them.
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = k0 + 16 * (e >> 2) + 4 * g + (e & 3);
        const bool ok = key < hi && held_now[e >> 2];
#pragma unroll
        for (int w = 0; w < Tile<D>::kWords; ++w) {
          if (!ok) now.v[e][w] = 0;
          if (!word_finite(now.v[e][w])) {
            now.v[e][w] = 0;
            odd_v = true;
          }
        }
      }
      odd_v = __any(odd_v);
    }

    // A lane group whose scores pass the running maximum renews it.
    bool past = false;
    float top[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      top[t] = fmaxf(fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])),
                     fmaxf(fmaxf(s[t][4], s[t][5]), fmaxf(s[t][6], s[t][7])));
      past |= top[t] > m[t] + kSlack;
    }
    if (__any(past)) {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        float x = fmaxf(m[t], top[t]);
        x = fmaxf(x, __shfl_xor(x, 16));
        x = fmaxf(x, __shfl_xor(x, 32));
        const float a = exp2_from(m[t], x);
        m[t] = x;
        l[t] *= a;
#pragma unroll
        for (int v = 0; v < kV; ++v) o[t][v] *= a;
      }
    }
    u32x4v pw[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
      const float from = m[t] == kNone ? 0.f : m[t];
#pragma unroll
      for (int e = 0; e < 8; ++e) s[t][e] = exp2_fast(s[t][e] - from);
      l[t] += ((s[t][0] + s[t][1]) + (s[t][2] + s[t][3])) + ((s[t][4] + s[t][5]) + (s[t][6] + s[t][7]));
#pragma unroll
      for (int e = 0; e < 4; ++e) pw[t][e] = dev::pack_bf16(s[t][2 * e], s[t][2 * e + 1]);
    }
    // V^T: register pairs of neighbouring keys -> the low and the high halves' columns.
#pragma unroll
    for (int w = 0; w < Tile<D>::kWords; ++w) {
      u32x4v even, odd;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        even[e] = __builtin_amdgcn_perm(now.v[2 * e + 1][w], now.v[2 * e][w], 0x05040100u);
        odd[e] = __builtin_amdgcn_perm(now.v[2 * e + 1][w], now.v[2 * e][w], 0x07060302u);
      }
#pragma unroll
      for (int t = 0; t < T; ++t) {
        o[t][2 * w] = dev::mfma_bf16(even, pw[t], o[t][2 * w]);
        o[t][2 * w + 1] = dev::mfma_bf16(odd, pw[t], o[t][2 * w + 1]);
      }
    }
    if (!plain && odd_v) {               // rare: the words taken out above, row by row
      for (int kk = 0; kk < 32; ++kk) {
        if (k0 + kk >= hi || !(kk < 16 ? held_now[0] : held_now[1])) continue;
        const uint16_t* vp = p.V + (kk < 16 ? base_now[0] : base_now[1]) + (kk & 15) * D;
        const int from = 16 * ((kk & 15) >> 2) + r, e = 4 * (kk >> 4) + (kk & 3);
#pragma unroll
        for (int t = 0; t < T; ++t) {
          float mine = 0.f;
#pragma unroll
          for (int x = 0; x < 8; ++x) mine = x == e ? s[t][x] : mine;
          const float pk = __shfl(mine, from);
          const bool sees = (__shfl(static_cast<int>(seen[t]), from) >> e) & 1;
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
    if (step + 1 < steps) now = next;
  }

  // Join the waves.
#pragma unroll
  for (int t = 0; t < T; ++t) {
    l[t] += __shfl_xor(l[t], 16);
    l[t] += __shfl_xor(l[t], 32);
    if (g == 0) {
      sh_m[wave][16 * t + r] = m[t];
      sh_l[wave][16 * t + r] = l[t];
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const int c = 16 * t + r;
    const float top = fmaxf(fmaxf(sh_m[0][c], sh_m[1][c]), fmaxf(sh_m[2][c], sh_m[3][c]));
    const float a = exp2_from(m[t], top);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int v = 0; v < kV; v += 4)
        *reinterpret_cast<f32x4*>(&sh_o[wave][c][kV * (4 * g + i) + v]) =
            f32x4{o[t][v][i], o[t][v + 1][i], o[t][v + 2][i], o[t][v + 3][i]} * a;
  }
  __syncthreads();
  constexpr int kPer = D / 8;            // threads a column
  for (int x = static_cast<int>(threadIdx.x); x < cols * kPer; x += kThreads) {
    const int c = x / kPer, d = 8 * (x % kPer);
    const float top = fmaxf(fmaxf(sh_m[0][c], sh_m[1][c]), fmaxf(sh_m[2][c], sh_m[3][c]));
    float sum = 0.f;
    f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      sum += sh_l[w][c] * exp2_from(sh_m[w][c], top);
      a += *reinterpret_cast<const f32x4*>(&sh_o[w][c][d]);
      b += *reinterpret_cast<const f32x4*>(&sh_o[w][c][d + 4]);
    }
    const int64_t row = at.first + (c0 + c) / p.G;
    const int64_t head = row * p.Hq + h * p.G + (c0 + c) % p.G;
    if (p.splits == 1) {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      const u32x4v w = {dev::pack_bf16(a[0] * inv, a[1] * inv), dev::pack_bf16(a[2] * inv, a[3] * inv),
                        dev::pack_bf16(b[0] * inv, b[1] * inv), dev::pack_bf16(b[2] * inv, b[3] * inv)};
      *reinterpret_cast<u32x4v*>(p.out + head * D + d) = w;
      if (p.lse && d == 0) p.lse[head] = sum == 0.f ? kNone : (top + log2f(sum)) * 0.69314718055994531f;
    } else {
      const int64_t part = split * static_cast<int64_t>(p.M) * p.Hq + head;
      *reinterpret_cast<f32x4*>(p.part_o + part * D + d) = a;
      *reinterpret_cast<f32x4*>(p.part_o + part * D + d + 4) = b;
      if (d == 0) p.part_ml[part] = {top, sum};
    }
  }
}

// The splits' (m, l, O) of one row and head, a wave each.
template <int D>
__global__ __launch_bounds__(kThreads) void tree_join_kernel(const float* __restrict__ part_o,
                                                             const float2* __restrict__ part_ml, int64_t heads,
                                                             int splits, uint16_t* __restrict__ out,
                                                             float* __restrict__ lse) {
  constexpr int kPer = D / 4, kAtOnce = 64 / kPer;     // lanes a split, splits at a time
  const int lane = static_cast<int>(threadIdx.x) & 63;
  const int64_t head = static_cast<int64_t>(blockIdx.x) * kWaves + (threadIdx.x >> 6);
  if (head >= heads) return;
  float2 ml = {kNone, 0.f};
  if (lane < splits) ml = part_ml[lane * heads + head];
  float top = ml.x;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float a = exp2_from(ml.x, top);
  float sum = a * ml.y;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += kAtOnce) {
    const int s = s0 + lane / kPer;
    const float w = __shfl(a, s & 63);
    if (s < splits && w != 0.f)          // a split with nothing for this row wrote no O
      o += w * *reinterpret_cast<const f32x4*>(part_o + (s * heads + head) * D + 4 * (lane % kPer));
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
    tree_attention_kernel<D, 1><<<grid, kThreads, 0, stream>>>(p);
  else if constexpr (D <= 128)
    tile_cols == 32 ? tree_attention_kernel<D, 2><<<grid, kThreads, 0, stream>>>(p)
                    : tree_attention_kernel<D, 4><<<grid, kThreads, 0, stream>>>(p);
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
  c.tile_cols = per <= 16 || D > 128 ? 16 : per <= 32 ? 32 : 64;
  c.tiles = most_tiles(M, B, G, c.tile_cols);
  const int64_t groups = c.tiles * Hk;
  const int64_t want = (4 * static_cast<int64_t>(num_cus) + groups - 1) / groups;
  const int64_t keys = std::max(max_kv_len, 1);
  const int64_t splits = std::max<int64_t>(1, std::min({want, static_cast<int64_t>(kMaxSplits), (keys + kStep - 1) / kStep}));
  c.split_len = static_cast<int>(((keys + splits - 1) / splits + kStep - 1) / kStep * kStep);
  c.splits = static_cast<int>((keys + c.split_len - 1) / c.split_len);
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
  const TreeArgs p{q, ld_q, cache.K, cache.V, cache.page_stride, cache.page_shift, cache.num_pages, pages, ld_pages,
                   max_keys, cached, offsets, mask, ld_mask, mask_wide, scale * 1.44269504088896341f, out, lse,
                   part_o, part_ml, M, B, Hq, Hk, Hq / Hk, static_cast<int>(c.tiles), c.splits, c.split_len};
  if (D == 64) launch<64>(p, c.tile_cols, c.blocks, stream);
  else if (D == 128) launch<128>(p, c.tile_cols, c.blocks, stream);
  else launch<256>(p, c.tile_cols, c.blocks, stream);
  return hipGetLastError();
}

}  // namespace prq
