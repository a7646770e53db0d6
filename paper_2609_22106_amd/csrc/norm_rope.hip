// Queries, keys and values from the projections to the attention: every query and
// key head normed over its D elements (optional), its first `rot` dims rotated by
// the row's position, queries written as bf16 and keys and values into their slots
// of the paged cache, all in one pass.
//
// x one head's vector, w the norm's weight, (c, s) the table's entry of the row's
// position and the pair:
//   y = x / sqrt(mean(x^2) + eps) * w
//   (y_a, y_b) -> (y_a c - y_b s, y_b c + y_a s)     pairs (i, i + rot / 2), or (2i, 2i + 1)
// in float32, rounded once, to bf16, as it is stored.
//
// Bytes: 4 (or 2) in and 2 out per element and 4 rot for each row's table entry: HBM
// bounds long prompts, the launch a decoding step.  A head is D / 8 lanes; a lane
// holds the two elements' quadruples that rotate with each other (4i.. and
// rot / 2 + 4i.., or 8 consecutive elements of interleaved pairs), so that the
// rotation needs no other lane and loads and stores stay 16 and 8 bytes wide.  A
// workgroup takes heads of one row, the loads of all of its kHeads heads a lane
// group in flight at once.  8192 rows of 32 + 8 + 8 float32 heads of 128: 59 us, 306 MB at
// 5.2 TB/s (a plain copy here 5.5); one row: 2.9 us, a launch and two dependent loads.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_device.hpp"
#include "prq_internal.h"

namespace prq {
namespace {

constexpr int kThreads = 256;

struct RopeArgs {
  const void *q, *k, *v;
  int64_t ld_q, ld_k, ld_v;
  const void *wq, *wk;
  const int32_t* positions;
  const float* table;
  const int64_t* slots;
  uint16_t *q_out, *K, *V;
  int64_t page_stride, num_slots;
  int Hq, Hk, rot, table_rows, page_shift;
  float eps;
  bool w_bf16, interleaved;
};

template <bool kBf16>
__device__ __forceinline__ dev::f32x4 load4(const void* p, int64_t at) {
  if constexpr (kBf16) {
    const dev::u32x2 w = *reinterpret_cast<const dev::u32x2*>(static_cast<const uint16_t*>(p) + at);
    return {dev::bf16_lo(w.x), dev::bf16_hi(w.x), dev::bf16_lo(w.y), dev::bf16_hi(w.y)};
  } else {
    return *reinterpret_cast<const dev::f32x4*>(static_cast<const float*>(p) + at);
  }
}

__device__ __forceinline__ void store4(uint16_t* p, dev::f32x4 x) {
  const dev::u32x2 w = {dev::pack_bf16(x[0], x[1]), dev::pack_bf16(x[2], x[3])};
  *reinterpret_cast<dev::u32x2*>(p) = w;
}

template <int D, bool kBf16, int kHeads>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(const RopeArgs p) {
  constexpr int kLanes = D / 8, kGroups = kThreads / kLanes;
  const int64_t row = blockIdx.x;
  const int i = static_cast<int>(threadIdx.x) % kLanes;
  const int first = static_cast<int>(blockIdx.y) * kGroups * kHeads + static_cast<int>(threadIdx.x) / kLanes;
  const int heads = p.Hq + 2 * p.Hk;
  // the lane's two quadruples
  const bool turned = p.interleaved ? 8 * i < p.rot : i < (p.rot >> 3);
  const bool halves = turned && !p.interleaved;
  const int a = halves ? 4 * i : p.interleaved ? 8 * i : p.rot + 8 * (i - (p.rot >> 3));
  const int b = halves ? (p.rot >> 1) + 4 * i : a + 4;

  dev::f32x4 x[kHeads], y[kHeads];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int h = first + u * kGroups;
    if (h < heads) {
      const bool is_q = h < p.Hq, is_k = h < p.Hq + p.Hk;
      const void* src = is_q ? p.q : is_k ? p.k : p.v;
      const int64_t ld = is_q ? p.ld_q : is_k ? p.ld_k : p.ld_v;
      const int64_t at = row * ld + (is_q ? h : is_k ? h - p.Hq : h - p.Hq - p.Hk) * D;
      x[u] = load4<kBf16>(src, at + a);
      y[u] = load4<kBf16>(src, at + b);
    }
  }
  // The row's cosines and sines of pairs 4i .. 4i + 3.  A position outside the table
  // has none: its rotated elements become NaN.
  dev::f32x4 cs[2] = {{1.f, 0.f, 1.f, 0.f}, {1.f, 0.f, 1.f, 0.f}};
  if (turned) {
    const int pos = p.positions[row];
    if (pos >= 0 && pos < p.table_rows) {
      const dev::f32x4* t = reinterpret_cast<const dev::f32x4*>(p.table + static_cast<int64_t>(pos) * p.rot + 8 * i);
      cs[0] = t[0];
      cs[1] = t[1];
    } else {
      cs[0] = cs[1] = __builtin_nanf("");
    }
  }
  const int64_t slot = p.slots[row];
  const bool kept = slot >= 0 && slot < p.num_slots;   // others' keys and values are not written
  const int64_t page = slot >> p.page_shift;
  const int64_t in_page = slot & ((int64_t{1} << p.page_shift) - 1);

#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int h = first + u * kGroups;
    const bool is_q = h < p.Hq, is_k = !is_q && h < p.Hq + p.Hk;
    const void* w = is_q ? p.wq : is_k ? p.wk : nullptr;
    if (w && h < heads) {                       // the same for the lanes of a head
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += x[u][j] * x[u][j] + y[u][j] * y[u][j];
#pragma unroll
      for (int d = kLanes / 2; d > 0; d >>= 1) sum += __shfl_xor(sum, d, kLanes);
      const float inv = 1.0f / sqrtf(sum * (1.0f / D) + p.eps);
      x[u] *= inv * (p.w_bf16 ? load4<true>(w, a) : load4<false>(w, a));
      y[u] *= inv * (p.w_bf16 ? load4<true>(w, b) : load4<false>(w, b));
    }
    if (turned && (is_q || is_k)) {
      const dev::f32x4 s = x[u], t = y[u];
      if (p.interleaved) {
        x[u] = {s[0] * cs[0][0] - s[1] * cs[0][1], s[1] * cs[0][0] + s[0] * cs[0][1],
                s[2] * cs[0][2] - s[3] * cs[0][3], s[3] * cs[0][2] + s[2] * cs[0][3]};
        y[u] = {t[0] * cs[1][0] - t[1] * cs[1][1], t[1] * cs[1][0] + t[0] * cs[1][1],
                t[2] * cs[1][2] - t[3] * cs[1][3], t[3] * cs[1][2] + t[2] * cs[1][3]};
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float c = cs[j >> 1][2 * (j & 1)], sn = cs[j >> 1][2 * (j & 1) + 1];
          x[u][j] = s[j] * c - t[j] * sn;
          y[u][j] = t[j] * c + s[j] * sn;
        }
      }
    }
    if (h < heads && (is_q || kept)) {
      uint16_t* out;
      if (is_q) {
        out = p.q_out + (row * p.Hq + h) * D;
      } else {
        const int kv = is_k ? h - p.Hq : h - p.Hq - p.Hk;
        out = (is_k ? p.K : p.V) + page * p.page_stride +
              (((static_cast<int64_t>(kv) << p.page_shift) + in_page) * D);
      }
      store4(out + a, x[u]);
      store4(out + b, y[u]);
    }
  }
}

template <int D, bool kBf16>
void launch(const RopeArgs& p, int M, int num_cus, hipStream_t stream) {
  constexpr int kGroups = kThreads / (D / 8);
  const int heads = p.Hq + 2 * p.Hk;
  const int most = (heads + kGroups - 1) / kGroups;   // heads a lane group would take in one workgroup a row
  // Few rows: a head a lane group, so that more workgroups share the latency; many: two, whose
  // loads are under way together.  us, 1 / 2 / 3 heads: 48 heads of 128 in float32, 61 rows
  // 3.1 / 3.9 / 4.9, 512 rows 6.2 / 6.6 / 7.6, 1024 rows 9.7 / 9.7 / 10.8, 8192 rows
  // 62.4 / 61.4 / 62.9; 48 heads of 64 in bf16, 1537 rows 7.7 / 7.2 / 7.2.
  const int per = static_cast<int64_t>(M) * most <= 8 * num_cus ? 1 : std::min(most, 2);
  const dim3 grid(M, (heads + kGroups * per - 1) / (kGroups * per));
  if (per == 1) norm_rope_kernel<D, kBf16, 1><<<grid, kThreads, 0, stream>>>(p);
  else norm_rope_kernel<D, kBf16, 2><<<grid, kThreads, 0, stream>>>(p);
}

}  // namespace

hipError_t launch_qk_norm_rope(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                               bool in_bf16, int M, int Hq, int Hk, int D, const void* wq, const void* wk,
                               bool w_bf16, float eps, const int32_t* positions, const float* table, int table_rows,
                               int rot, bool interleaved, uint16_t* q_out, const PagedCache& cache,
                               const int64_t* slots, int num_cus, hipStream_t stream) {
  const RopeArgs p{q, k, v, ld_q, ld_k, ld_v, wq, wk, positions, table, slots, q_out,
                   cache.K, cache.V, cache.page_stride, static_cast<int64_t>(cache.num_pages) << cache.page_shift,
                   Hq, Hk, rot, table_rows, cache.page_shift, eps, w_bf16, interleaved};
  auto go = [&](auto d) {
    constexpr int kD = decltype(d)::value;
    in_bf16 ? launch<kD, true>(p, M, num_cus, stream) : launch<kD, false>(p, M, num_cus, stream);
  };
  if (D == 64) go(std::integral_constant<int, 64>{});
  else if (D == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 256>{});
  return hipGetLastError();
}

}  // namespace prq
