// All experts of a few tokens (up to 64), in two launches: MXFP4 weights, bf16 activations.
//
// Token t with experts e_j and weights w_j, expert e's gate, up and down weights G, U (I x H) and
// D (N x (I + k_tail)):
//   h_e = SiLU(G_e x) * (U_e x),  SiLU(z) = z / (1 + exp(-z))
//   y   = sum_j w_j D_{e_j} [h; the last k_tail of h again]
// Sums are float32.  Between the launches w h is held in two bf16, its upper bits and the rest (the
// operands of the second product's matrix instructions), which is off by less than 2^-15 of it; y is
// rounded to bf16, by up to 2^-8, at the end.  A token that names an expert twice gets it with both
// weights; an id outside [0, E) names none.
//
// The weights of the experts that are reached are most of the bytes, and what bounds both launches
// where they are many: 64 tokens of 128 experts, eight a token, of 2048 -> 768 + 64 -> 2048, 292 MB in
// 67 us, 38.5 and 29; 19 tokens of 64, six a token, of 2560 -> 1408, 282 MB in 54.5, 34 and 20.5 (a copy
// reaches 5.4 TB/s, the first launch 5.0 and 5.5).  The second loses 5 us to its start and 2.5 to the join of
// workgroups; twice the waves or workgroups changed nothing there.  A CU has 80 cycles of matrix work
// free for every kilobyte of weights, so the activations are not quantized and the weights are brought
// to bf16 in registers (a 4-bit value times a power of two is exact there below 2^128, where float32 ends
// too; scale codes 253 and 254 reach beyond).  A wave has two units of weights under way; enough waves a
// CU keep the memory busy meanwhile.  One token (21 MB, 3.8 us of them) takes 14.0 us, since its trips to
// memory follow each other: in the first launch (7.4) the launch itself 1.5, routing 2.2, x 0.4, weights
// 1.9, the rest of them and the sums 1.5; in the second the table, weights, and the join.
//
// A slot is an expert (its number), or where there are fewer pairs of a token and an expert than
// experts a pair (its first occurrence), so that a launch of `slots` workgroups in y reaches every
// expert that is named.  An expert's tokens are gathered into columns in ascending order, 16 to a
// block of the first launch and 8 or 16 to an item of the second.  The first launch finds them with a
// lane a token, and leaves the second a table.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

using dev::f32x4;
using dev::u32x4v;

constexpr int kMaxSplits = 8;                       // workgroups that share output tiles
constexpr int kSteps = 2;                            // K steps of 128 in a wave's unit

// What the first launch leaves.  `hidden`: w h of the pairs, an expert's behind those of the lower
// ones, its tokens an item (8 or 16) at a time: of n of them [K steps][2][16][n][8] elements, the upper
// bits of a K step's octets and then what is left (low_part), the octets in the order in which a lane
// group's operands are loaded (octet_at), so that one load's lanes read one or two stretches.  The
// table: the second launch's items, experts in ascending order; of each the expert, its tokens in
// `hidden` (first 2^5 n), and the token of column i, -1 past the last.  An expert that a token names twice
// may have an empty item.
struct Table {
  int32_t* total;                                    // the number of items
  int32_t* experts;
  int32_t* rows;
  int32_t* columns;                                  // [items][tokens of an item]
  int shift;                                         // an item's tokens: 2^shift
};

// Elements of a pair's row of `hidden`: whole K steps, twice.
__host__ __device__ constexpr int64_t hidden_pitch(int I) { return 2 * ((I + 127) & ~127); }
// What is left of x without its lower 16 bits: 16 bits, of which bf16 keeps 8.  (A finite x has a finite upper
// part; nothing is left of an infinity, where inf - inf would make it a NaN.)
__device__ __forceinline__ float low_part(float x) {
  return __builtin_isinf(x) ? 0.f : x - dev::bf16_hi(__float_as_uint(x));
}
// Where octet o of a row's upper bits stands: lane group q's j-th of a K step, which is octet 4 q + j of it, at
// 4 j + q; the rest of it 16 further.
__device__ __forceinline__ int octet_at(int o) { return (o & ~15) << 1 | (o & 3) << 2 | (o >> 2 & 3); }

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

// A buffer of `bytes` from p on, both the same for the wave: a load from outside it reads zeros and goes
// nowhere, so that loops may ask for what is past their end.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000);
}
constexpr uint32_t kOutside = 0x80000000u;
constexpr int kStreamed = 2;                         // non-temporal

// Consecutive tiles of 16 rows of a packed weight.
struct Tiles {
  __amdgpu_buffer_rsrc_t codes, scales;
  int groups, steps;
  __device__ __forceinline__ Tiles() = default;
  __device__ __forceinline__ Tiles(const uint8_t* Wp, const uint8_t* Wps, int64_t first, int count, int steps)
      : codes(buffer(Wp + first * steps * 1024, count * steps * 1024)),
        scales(buffer(Wps + first * ((steps + 3) >> 2) * 256, count * ((steps + 3) >> 2) * 256)),
        groups((steps + 3) >> 2), steps(steps) {}
  // A lane's 16 code bytes of step s of tile t, and the dword that has its scale. The whole offset is the
  // lane's, as only that is held against the buffer's size.
  __device__ __forceinline__ u32x4v code(int t, int s, uint32_t past = 0) const {
    const uint32_t at = (threadIdx.x & 63) * 16 + static_cast<uint32_t>(t * steps + s) * 1024 | past;
    return __builtin_bit_cast(u32x4v, __builtin_amdgcn_raw_buffer_load_b128(codes, at, 0, kStreamed));
  }
  __device__ __forceinline__ uint32_t scale(int t, int s, uint32_t past = 0) const {
    const uint32_t at = (threadIdx.x & 63) * 4 + static_cast<uint32_t>(t * groups + (s >> 2)) * 256 | past;
    return __builtin_amdgcn_raw_buffer_load_b32(scales, at, 0, 0);
  }
};

// kSteps steps of a tile, from a multiple of kSteps on (zeros past its end), and their scales.
struct Unit {
  u32x4v codes[kSteps];
  uint32_t scales;
  __device__ __forceinline__ void load(const Tiles& w, int unit) {
    scales = w.scale(0, kSteps * unit) >> (8 * (kSteps * unit & 3));
#pragma unroll
    for (int i = 0; i < kSteps; ++i) codes[i] = w.code(0, kSteps * unit + i);
  }
};

// The tokens' experts and weights in LDS, a token's k entries apart by an odd number, at which 64 tokens'
// j-th ones lie in different banks.
struct Routing {
  int* ids;
  float* weights;
  int pitch;
  __device__ __forceinline__ Routing(const MoeArgs& p, unsigned char* lds) {
    pitch = p.k | 1;
    ids = reinterpret_cast<int*>(lds);
    weights = reinterpret_cast<float*>(lds) + p.M * pitch;
    for (int i = static_cast<int>(threadIdx.x); i < p.M * p.k; i += static_cast<int>(blockDim.x)) {
      const int t = token(p, i), at = t * pitch + i - t * p.k;
      ids[at] = p.ids[i];
      weights[at] = p.weights[i];
    }
    __syncthreads();
  }
  // Pair i's: i + 1/2 is at least 1 / 64 of a token from a whole one, the product off by 2^-22 of it.
  __device__ __forceinline__ int token(const MoeArgs& p, int i) const {
    return static_cast<int>((static_cast<float>(i) + 0.5f) * (1.0f / static_cast<float>(p.k)));
  }
};
__host__ __device__ constexpr int routing_bytes(int M, int k) { return 8 * M * (k | 1); }

// A lane's token's share of expert e (>= 0): whether it has one, the first of its k ids that names it,
// and the sum of the weights that do.
struct Share {
  bool has = false;
  int first = 0;
  float weight = 0.f;
  __device__ __forceinline__ Share(const MoeArgs& p, const Routing& r, int e) {
    const int lane = static_cast<int>(threadIdx.x) & 63;
    if (lane >= p.M) return;
    for (int j = p.k - 1; j >= 0; --j)
      if (r.ids[lane * r.pitch + j] == e) {
        weight += r.weights[lane * r.pitch + j];
        first = j;
        has = true;
      }
  }
};

// The table's entries of expert e's n tokens (lane i: the i-th), whose pairs are behind `pairs` others, and
// with the first slot the number of all.  The whole workgroup; bins: LDS for an int an expert.
template <int kN>
__device__ __forceinline__ void write_items(const MoeArgs& p, int slot, int e, int n, int token, int pairs,
                                            const Table& table, int* bins) {
  __shared__ int sums[2][kN];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int whole = (1 << table.shift) - 1;
  __syncthreads();                                   // the routing has been read
  for (int i = tid; i < p.E; i += 64 * kN) bins[i] = 0;
  __syncthreads();
  for (int i = tid; i < p.M * p.k; i += 64 * kN) {
    const int id = p.ids[i];
    if (id >= 0 && id < p.E) atomicAdd(&bins[id], 1);
  }
  __syncthreads();
  int before = 0, all = 0;
  for (int i = tid; i < p.E; i += 64 * kN) {
    const int items = (bins[i] + whole) >> table.shift;
    all += items;
    if (i < e) before += items;
  }
  before = __builtin_amdgcn_readlane(dev::prefix_sum(before), 63);
  all = __builtin_amdgcn_readlane(dev::prefix_sum(all), 63);
  if (lane == 0) {
    sums[0][wave] = before;
    sums[1][wave] = all;
  }
  __syncthreads();
  before = all = 0;
  for (int w = 0; w < kN; ++w) {
    before += sums[0][w];
    all += sums[1][w];
  }
  if (slot == 0 && tid == 0) *table.total = all;
  if (wave || n == 0) return;
  const int items = (bins[e] + whole) >> table.shift;
  for (int i = lane; i < items << table.shift; i += 64) {
    if ((i & whole) == 0) {
      table.experts[before + (i >> table.shift)] = e;
      table.rows[before + (i >> table.shift)] = (pairs + i) << 5 | max(0, min(n - i, whole + 1));
    }
    table.columns[(before << table.shift) + i] = i < 64 ? token : -1;
  }
}

// Rows of x in LDS: piece_of() / kG elements of 16 kG tokens at a time, rows 32 bytes past a multiple of
// 128, at which the lanes of an operand's read meet different banks.  Pieces of 1024 where a wave has more
// than a piece's two turns anyway: a CU then holds four workgroups, not two (19 tokens of 64 experts
// 66.4 -> 62.4 us with workgroups of four waves, which in turn leave fewer CUs idle at the end than eight);
// 512 is no faster (63.1).
__host__ __device__ constexpr int piece_of(int parts, int blocks) {       // elements, of one block's rows
  return parts == 1 || parts * blocks == 2 ? 1024 : 2048;
}
__host__ __device__ constexpr int pitch_of(int parts, int blocks) {       // bytes
  return piece_of(parts, blocks) / blocks * 2 + 32;
}

// First launch: a wave has 16 intermediate features of one expert (a gate tile and an up tile) for
// all of its tokens, and of the steps of H every kS-th unit.  The workgroup's waves share the
// expert's rows of x in LDS.  The last workgroup of a slot writes the table.
template <int kN, int kS>
__global__ __launch_bounds__(64 * kN, 4) void moe_up_kernel(const MoeArgs p, bool by_expert, int rows_bytes,
                                                              uint16_t* __restrict__ hidden, const Table table) {
  constexpr int kTiles = kN / kS;
  extern __shared__ __align__(16) unsigned char smem[];
  f32x4* const sums = reinterpret_cast<f32x4*>(smem + rows_bytes);       // [kN][2][64]
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int slot = static_cast<int>(blockIdx.y);
  const int tile = static_cast<int>(blockIdx.x) * kTiles + wave / kS, part = wave % kS;
  const int steps = (p.H + 127) >> 7, tiles = p.I >> 4, units = (steps + kSteps - 1) / kSteps;

  const Routing routing(p, smem);
  int e = slot;
  if (!by_expert) {
    e = __builtin_amdgcn_readfirstlane(routing.ids[slot / p.k * routing.pitch + slot % p.k]);
    if (e >= p.E) e = -1;
  }
  const Share share(p, routing, e);
  const uint64_t mine = e < 0 ? 0 : __ballot(share.has);
  int n = __popcll(mine);
  if (!by_expert) {                                  // an earlier pair of the same expert has it
    const int token = slot / p.k;
    if (__ballot(e >= 0 && share.has && (lane < token || (lane == token && lane * p.k + share.first < slot)))) n = 0;
  }
  // Column i: the i-th token.  Lanes without a share go behind the others.
  const uint64_t below = (uint64_t{1} << lane) - 1;
  const bool has = mine >> lane & 1;
  const int at = has ? __popcll(mine & below) : __popcll(mine) + __popcll(~mine & below);
  const int column = __builtin_amdgcn_ds_permute(4 * at, has ? lane : -1);
  int pairs = 0;                                     // of lower experts
  for (int i = lane; i < ((p.M * p.k + 63) & ~63); i += 64) {
    const int t = routing.token(p, i), id = i < p.M * p.k ? routing.ids[t * routing.pitch + i - t * p.k] : -1;
    pairs += __popcll(__ballot(id >= 0 && id < e));
  }
  if (blockIdx.x + 1 == gridDim.x) return write_items<kN>(p, slot, e, n, column, pairs, table, reinterpret_cast<int*>(smem));
  if (n == 0) return;                                // the whole workgroup
  const float weight = __int_as_float(__builtin_amdgcn_ds_permute(4 * at, __float_as_int(share.weight)));

  const int64_t first = static_cast<int64_t>(e) * 2 * tiles + min(tile, tiles - 1);
  const Tiles gate(p.up_codes, p.up_scales, first, 1, steps), up(p.up_codes, p.up_scales, first + tiles, 1, steps);
  // Tokens 16 block0 .. 16 (block0 + kG) - 1 of the expert.
  auto pass = [&](int block0, auto blocks) {
    constexpr int kG = decltype(blocks)::value, kPiece = piece_of(kS, kG), kUnits = kPiece / (128 * kSteps) / kG, kPitch = pitch_of(kS, kG);
    const int rows = min(n - 16 * block0, 16 * kG);
    // A piece's units of a wave, of which there is an even number (zeros past the end), so that the two that
    // are under way have registers of their own.
    auto turns = [&](int u0) { return max(((min(units - u0, kUnits) + kS - 1) / kS + 1) & ~1, 2); };
    struct Both {
      Unit gate, up;
    } ring[2];
    int next_u0 = 0, next_turn = 0;                  // what is asked for next
    auto ask = [&](Both& w) {
      const int turn = next_turn * kS + part, u = turn < kUnits ? next_u0 + turn : units;
      w.gate.load(gate, u);
      w.up.load(up, u);
      if (++next_turn == turns(next_u0)) {
        next_turn = 0;
        next_u0 += kUnits;
      }
    };
    f32x4 acc[kG][2] = {};
    auto compute = [&](const Both& w, int u0, int turn) {
      const int u = turn * kS + part;                // of the piece
      if (u >= min(units - u0, kUnits)) return;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        u32x4v a[4], a2[4], b[4];
        to_bf16(w.gate.codes[i], w.gate.scales >> (8 * i) & 255u, a);
        to_bf16(w.up.codes[i], w.up.scales >> (8 * i) & 255u, a2);
#pragma unroll
        for (int g = 0; g < kG; ++g) {
          // columns without a token read the first one's row: their sums are nobody's
          const unsigned char* from = smem + (16 * g + c < rows ? 16 * g + c : 0) * kPitch + (u * kSteps + i) * 256 + q * 64;
#pragma unroll
          for (int j = 0; j < 4; ++j) b[j] = *reinterpret_cast<const u32x4v*>(from + 16 * j);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            acc[g][0] = dev::mfma_bf16(a[j], b[j], acc[g][0]);
            acc[g][1] = dev::mfma_bf16(a2[j], b[j], acc[g][1]);
          }
        }
      }
    };
    ask(ring[0]);
    for (int u0 = 0; u0 < units; u0 += kUnits) {
      __syncthreads();                               // what is there has been read
      constexpr int kRow = kPiece / kG / 8;          // 16-byte parts of a row
      for (int i = tid; i < rows * kRow; i += 64 * kN) {
        const int r = i / kRow, k = u0 * 128 * kSteps + i % kRow * 8;
        const int token = __builtin_amdgcn_readfirstlane(__shfl(column, 16 * block0 + r, 64)) & 63;
        u32x4v v = 0u;
        if (k < p.H) v = *reinterpret_cast<const u32x4v*>(p.x + token * p.ld_x + k);
        *reinterpret_cast<u32x4v*>(smem + r * kPitch + i % kRow * 16) = v;
      }
      __syncthreads();
#pragma unroll 1
      for (int turn = 0; turn < turns(u0); turn += 2) {
        ask(ring[1]);
        compute(ring[0], u0, turn);
        ask(ring[0]);
        compute(ring[1], u0, turn + 1);
      }
    }
#pragma unroll
    for (int g = 0; g < kG; ++g) {
      f32x4 z = acc[g][0], y = acc[g][1];
      if constexpr (kS > 1) {
        if (g || block0) __syncthreads();
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
      const float w = __shfl(weight, 16 * (block0 + g) + c, 64);
      const int row = 16 * (block0 + g) + c;
      if (row < n && tile < tiles) {
        float h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = z[i] / (1.f + expf(-z[i])) * y[i] * w;
        auto upper = [](float x, float y) { return __float_as_uint(x) >> 16 | (__float_as_uint(y) & 0xFFFF0000u); };
        auto rest = [](float x, float y) { return dev::pack_bf16(low_part(x), low_part(y)); };
        const int first = row >> table.shift << table.shift, columns = min(n - first, 1 << table.shift);
        uint16_t* to = hidden + (pairs + first) * hidden_pitch(p.I) +
                       (octet_at(2 * tile + (q >> 1)) * columns + row - first) * 8 + 4 * (q & 1);
        *reinterpret_cast<dev::u32x2*>(to) = dev::u32x2{upper(h[0], h[1]), upper(h[2], h[3])};
        *reinterpret_cast<dev::u32x2*>(to + 16 * 8 * columns) = dev::u32x2{rest(h[0], h[1]), rest(h[2], h[3])};
      }
    }
  };
  if (n <= 16) {
    pass(0, std::integral_constant<int, 1>{});
  } else {                                           // past 32 tokens the weights come from L2 again
    for (int block = 0; 16 * block < n; block += 2) pass(block, std::integral_constant<int, 2>{});
  }
}

// Floats between two tokens' sums of kT tiles in LDS: the 16 columns of a store meet different banks.
constexpr int sums_pitch(int tiles) { return 16 * tiles + 4; }

// Second launch: kT tiles of 16 output features of all tokens.  The items are dealt in turn to the
// tiles' workgroups, and the K steps of up to kWindow of a workgroup's evenly, in order, to its waves.
// An item's sums are added to its tokens' in LDS, of which each wave has its own.  The waves' sums are
// added in their order, the workgroups' in theirs, by the one that arrives last.
//
// kBoth: an item has 8 tokens, whose upper bits are columns 0 to 7 of the operand and the rest columns 8
// to 15, so that one load and one product serve both.  (16 tokens take two of each, and a load's time in
// the address unit goes by its lanes, also those that get nothing.)
//
// A wave asks for the weights and activations of a step kAhead steps ahead.  The loop has loads
// without conditions only (past the end, and of columns without a token, outside their buffers), so
// that every wait counts exactly the loads behind it.
constexpr int kWindow = 64;

template <int kT, int kN, int kAhead, bool kBoth>
__global__ __launch_bounds__(64 * kN, kBoth ? 4 : 2) void moe_down_kernel(const MoeArgs p,
                                                                          const uint16_t* __restrict__ hidden,
                                                                          const Table table, int most, float* parts,
                                                                          uint32_t* arrived) {
  constexpr int kPitch = sums_pitch(kT), kRing = kAhead + 1;
  constexpr int kItem = kBoth ? 8 : 16, kOperands = kBoth ? 1 : 2;
  extern __shared__ __align__(16) float own[];       // [kN][M][kPitch]
  __shared__ int sh_experts[kWindow], sh_rows[kWindow];
  __shared__ int sh_columns[kWindow][kItem];
  __shared__ int sh_last;
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, q = lane >> 4, token = c % kItem;           // of the item
  const int tile = static_cast<int>(blockIdx.x) * kT, splits = static_cast<int>(gridDim.y), part = static_cast<int>(blockIdx.y);
  const int K = p.I + p.k_tail, steps = (K + 127) >> 7, tiles = p.N >> 4;
  const auto rsrc = buffer(hidden, static_cast<int>(p.M * p.k * hidden_pitch(p.I) * 2));
  float* const mine = own + wave * p.M * kPitch;

  // Item i of this workgroup is item part + splits i of all; the first window's are loaded before their
  // number is known.
  for (int item0 = 0;; item0 += kWindow) {
    int expert = 0, rows = 0, column[kWindow * kItem / (64 * kN)];
    const int at = part + splits * item0;
    if (tid < kWindow) {
      expert = table.experts[min(at + splits * tid, most - 1)];
      rows = table.rows[min(at + splits * tid, most - 1)];
    }
#pragma unroll
    for (int i = 0; i < kWindow * kItem / (64 * kN); ++i) {
      const int entry = tid + i * 64 * kN;
      column[i] = table.columns[min(at + splits * (entry / kItem), most - 1) * kItem + entry % kItem];
    }
    const int total = *table.total;
    if (item0 == 0) {
      for (int i = lane; i < p.M * kPitch / 4; i += 64) reinterpret_cast<f32x4*>(mine)[i] = 0.f;
    } else {
      __syncthreads();                               // the window before has been read
    }
    const int items = min((total - at + splits - 1) / splits, kWindow);
    if (at >= total) break;                          // the whole workgroup
    if (tid < kWindow) {
      sh_experts[tid] = expert;
      sh_rows[tid] = rows;
    }
#pragma unroll
    for (int i = 0; i < kWindow * kItem / (64 * kN); ++i) {
      const int entry = tid + i * 64 * kN;
      sh_columns[entry / kItem][entry % kItem] = column[i];
    }
    __syncthreads();

    const int begin = items * steps * wave / kN, n = items * steps * (wave + 1) / kN - begin;
    if (n > 0) {
      // The step that is asked for next: its item, the expert's tiles, and where the item's tokens are
      // in `hidden`, in bytes, and how many.
      int item = begin / steps, step = begin % steps, u = 0, columns;
      Tiles down;
      uint32_t base;
      auto enter = [&] {
        const int64_t first = static_cast<int64_t>(__builtin_amdgcn_readfirstlane(sh_experts[item])) * tiles + tile;
        down = Tiles(p.down_codes, p.down_scales, first, kT, steps);
        const int rows = __builtin_amdgcn_readfirstlane(sh_rows[item]);
        base = static_cast<uint32_t>((rows >> 5) * hidden_pitch(p.I) * 2);
        columns = rows & 31;
      };
      enter();
      struct Step {
        u32x4v codes[kT];
        uint32_t scales[kT];
        u32x4v b[kOperands][4];
      } ring[kRing];
      auto ask = [&](Step& s) {
        int k = 128 * step + 32 * q;                 // the tail meets the last values again, zeros behind it
        const uint32_t past = u < n ? 0 : kOutside;
        const bool in = k < K && token < columns && u < n;
        if (k >= p.I) k -= p.k_tail;
        const int slot = (k >> 7) * 32 + (k >> 5 & 3) + (kBoth && c >= kItem ? 16 : 0);
        const uint32_t at = in ? base + static_cast<uint32_t>((slot * columns + token) * 16) : kOutside;
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          s.codes[t] = down.code(t, step, past);
          s.scales[t] = down.scale(t, step, past);
        }
#pragma unroll
        for (int h = 0; h < kOperands; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            s.b[h][j] = __builtin_bit_cast(
                u32x4v, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, (256 * h + 64 * j) * columns, 0));
        if (++u < n && ++step == steps) {
          step = 0;
          ++item;
          enter();
        }
      };
      f32x4 acc[kT] = {};
      int now = step, now_item = item, now_column = sh_columns[item][token];    // of the step that is computed
      auto compute = [&](const Step& s, bool last) {
#pragma unroll
        for (int t = 0; t < kT; ++t) {
          u32x4v a[4];
          to_bf16(s.codes[t], s.scales[t] >> (8 * (now & 3)) & 255u, a);
#pragma unroll
          for (int h = 0; h < kOperands; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[t] = dev::mfma_bf16(a[j], s.b[h][j], acc[t]);
        }
        if (++now == steps || last) {                // the item's sums are complete here
          now = 0;
#pragma unroll
          for (int t = 0; t < kT; ++t) {
            if constexpr (kBoth)                     // the upper bits' sums and the rest's
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[t][i] += dev::moved<0x128, 0xF>(0.f, acc[t][i]);        // row_ror 8
            if (now_column >= 0 && c < kItem)
              *reinterpret_cast<f32x4*>(mine + now_column * kPitch + 16 * t + 4 * q) += acc[t];
            acc[t] = 0.f;
          }
          dev::wave_lds_barrier();
          if (!last) now_column = sh_columns[++now_item][token];
        }
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ask(ring[i]);
      for (int i0 = 0; i0 < n; i0 += kRing) {
#pragma unroll
        for (int r = 0; r < kRing; ++r) {
          ask(ring[(r + kAhead) % kRing]);
          if (i0 + r < n) compute(ring[r], i0 + r + 1 == n);
        }
      }
    }
  }
  __syncthreads();
  // Thread (t, i): features 4 i .. 4 i + 3 of tokens t, t + kTogether, ...
  constexpr int kTogether = 16 * kN / kT, kPasses = (kMaxLayerTokens + kTogether - 1) / kTogether;
  const int t0 = tid / (4 * kT), i = tid % (4 * kT);
  f32x4 y[kPasses];
  auto here = [&](int s) { return t0 + s * kTogether < p.M; };
  auto place = [&](int s) { return static_cast<int64_t>(t0 + s * kTogether) * p.N + 16 * tile + 4 * i; };
#pragma unroll
  for (int s = 0; s < kPasses; ++s) {
    y[s] = 0.f;
    if (here(s)) {
#pragma unroll
      for (int w = 0; w < kN; ++w)
        y[s] += *reinterpret_cast<const f32x4*>(own + (w * p.M + t0 + s * kTogether) * kPitch + 4 * i);
    }
  }
  if (splits > 1) {
    const int64_t stride = static_cast<int64_t>(p.M) * p.N;
#pragma unroll
    for (int s = 0; s < kPasses; ++s)
      if (here(s)) {
        // device scope: the last workgroup may be on another XCD with an L2 of its own
#pragma unroll
        for (int j = 0; j < 4; j += 2)
          __hip_atomic_store(reinterpret_cast<uint64_t*>(parts + part * stride + place(s) + j),
                             static_cast<uint64_t>(__float_as_uint(y[s][j + 1])) << 32 | __float_as_uint(y[s][j]),
                             __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // what this wave has stored is there
    __syncthreads();
    if (tid == 0)
      sh_last = __hip_atomic_fetch_add(arrived + blockIdx.x, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
                static_cast<uint32_t>(splits - 1);
    __syncthreads();
    if (!sh_last) return;
    if (tid == 0) __hip_atomic_store(arrived + blockIdx.x, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    uint64_t v[kPasses][kMaxSplits][2];              // all loads under way together
#pragma unroll
    for (int s = 0; s < kPasses; ++s)
#pragma unroll
      for (int w = 0; w < kMaxSplits; ++w)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          v[s][w][j] = w < splits && here(s)
                           ? __hip_atomic_load(reinterpret_cast<const uint64_t*>(parts + w * stride + place(s)) + j,
                                               __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)
                           : 0;
#pragma unroll
    for (int s = 0; s < kPasses; ++s) {
      y[s] = 0.f;
#pragma unroll
      for (int w = 0; w < kMaxSplits; ++w)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          y[s][2 * j] += __uint_as_float(static_cast<uint32_t>(v[s][w][j]));
          y[s][2 * j + 1] += __uint_as_float(static_cast<uint32_t>(v[s][w][j] >> 32));
        }
    }
  }
#pragma unroll
  for (int s = 0; s < kPasses; ++s)
    if (here(s)) {
      const dev::u32x2 v = {dev::pack_bf16(y[s][0], y[s][1]), dev::pack_bf16(y[s][2], y[s][3])};
      *reinterpret_cast<dev::u32x2*>(p.out + (t0 + s * kTogether) * p.ld_out + 16 * tile + 4 * i) = v;
    }
}

size_t up16(size_t n) { return (n + 15) & ~size_t{15}; }
size_t hidden_bytes(const MoeArgs& p) { return up16(static_cast<size_t>(p.M) * p.k * hidden_pitch(p.I) * 2); }
// An expert has as many items as their size goes into the pairs that name it, rounded up.
int most_items(const MoePlan& c, const MoeArgs& p) { return std::min(p.M * p.k, c.slots + p.M * p.k / c.item); }
size_t table_bytes(const MoePlan& c, const MoeArgs& p) {
  return up16(4 * (4 + static_cast<size_t>(most_items(c, p)) * (2 + c.item)));
}

}  // namespace

MoePlan plan_moe_layer(const MoeArgs& p, int num_cus) {
  MoePlan c;
  c.slots = std::min(p.E, p.M * p.k);
  c.by_expert = c.slots == p.E;
  // The first launch: a wave a tile, or two or four where those would be few, fewer where a wave has
  // more to compute.  us of the whole call, four / two / one (128 experts, eight a token, of 2048 -> 768):
  // one token 14.6 / 15.3 / 16.6, 3 22.5 / 22.0 / 23.1, 8 40.6 / 37.6 / 37.4, 16 64.2 / 49.2 / 45.5, 64 104 / 84 / 70;
  // 64 experts, six a token, of 2560 -> 1408: 2 24.0 / 24.1 / 26.4, 5 38.3 / 35.9 / 36.9, 19 85.1 / 70.2 / 62.4;
  // 64 tokens of 2048 -> 1408: two of 8 experts 33.0 / 30.6 / 33.5, four of 16 51.0 / 42.9 / 39.0.
  const int64_t waves = static_cast<int64_t>(p.I / 16) * c.slots * (p.M <= 16 ? 1 : 3);
  c.parts = waves <= 4 * num_cus ? 4 : waves <= 12 * num_cus ? 2 : 1;
  // The second: two tiles a workgroup where their number is even, so that the activations are loaded for
  // two, and a workgroup a CU, of which a wave has three steps at least.  us, two tiles and four
  // workgroups along the experts / two / one, then one tile and two workgroups (128 experts of 768 + 64,
  // N = 2048): one token 7.5 / 8.0 / 8.3 / 7.4, 4 tokens 10.1 / 13.0 / 18.7 / 11.7, 8 tokens
  // 13.3 / 18.8 / 29.0 / 16.3.
  const int64_t steps = static_cast<int64_t>(c.slots) * ((p.I + p.k_tail + 127) / 128);
  c.tiles = p.N % 32 == 0 ? 2 : 1;
  c.splits = static_cast<int>(std::min<int64_t>(num_cus / (p.N / 16 / c.tiles), steps / 12));
  c.splits = std::max(1, std::min(c.splits, kMaxSplits));
  // Its items: 8 tokens, whose w h fill an operand's columns with both parts, while an expert has no more than
  // four on average; else 16, which need twice the loads and products but the weights less often.  us of the
  // whole call, 8 / 16: one token of 128 experts 14.0 / 14.3, 16 45.9 / 49.7, 64 74.0 / 75.3; 24 of 64 experts 68.6 / 73.1;
  // 16 of 8 experts of 2816, two a token 25.4 / 26.4, 32 30.5 / 29.7, 64 42.0 / 40.9, four a token 60.4 / 55.9.
  c.item = p.M <= 8 || p.M * p.k <= 4 * p.E ? 8 : 16;
  return c;
}

size_t moe_workspace_bytes(const MoePlan& c, const MoeArgs& p) {
  return kWorkspaceStateBytes + hidden_bytes(p) + table_bytes(c, p) +
         (c.splits > 1 ? static_cast<size_t>(c.splits) * p.M * p.N * 4 : 0);
}

hipError_t launch_moe_layer(const MoePlan& c, const MoeArgs& p, void* workspace, hipStream_t stream) {
  char* at = static_cast<char*>(workspace);
  uint32_t* arrived = reinterpret_cast<uint32_t*>(at);
  uint16_t* hidden = reinterpret_cast<uint16_t*>(at += kWorkspaceStateBytes);
  int32_t* const ints = reinterpret_cast<int32_t*>(at += hidden_bytes(p));
  const int most = most_items(c, p);
  int32_t* const experts = ints + 4 + c.item * most;
  const Table table{ints, experts, experts + most, ints + 4, c.item == 8 ? 3 : 4};
  float* parts = reinterpret_cast<float*>(at += table_bytes(c, p));
  auto up = [&](auto kernel, int kN, int kS) {
    const int rows = p.M <= 16 ? p.M * pitch_of(kS, 1) : std::max(16 * pitch_of(kS, 1), 32 * pitch_of(kS, 2));
    const int lds = std::max(rows + (kS > 1 ? kN * 2 * 64 * 16 : 0), std::max(routing_bytes(p.M, p.k), 4 * p.E));
    const int tiles = kN / kS;
    kernel<<<dim3((p.I / 16 + tiles - 1) / tiles + 1, c.slots), 64 * kN, lds, stream>>>(p, c.by_expert, rows, hidden, table);
    return hipGetLastError();
  };
  const hipError_t e = c.parts == 1   ? up(LargeLds<&moe_up_kernel<4, 1>>::kernel(), 4, 1)
                       : c.parts == 2 ? up(LargeLds<&moe_up_kernel<4, 2>>::kernel(), 4, 2)
                                      : up(LargeLds<&moe_up_kernel<4, 4>>::kernel(), 4, 4);
  if (e != hipSuccess) return e;
  auto down = [&](auto kernel, int kT, int kN) {
    kernel<<<dim3(p.N / 16 / kT, c.splits), 64 * kN, kN * p.M * sums_pitch(kT) * 4, stream>>>(p, hidden, table, most, parts,
                                                                                             arrived);
    return hipGetLastError();
  };
  if (c.item == 8)
    return c.tiles == 2 ? down(&moe_down_kernel<2, 4, 2, true>, 2, 4) : down(&moe_down_kernel<1, 4, 3, true>, 1, 4);
  return c.tiles == 2 ? down(&moe_down_kernel<2, 4, 1, false>, 2, 4) : down(&moe_down_kernel<1, 4, 2, false>, 1, 4);
}

}  // namespace prq
