// C ABI of the attention block's calls (include/prq.h): argument checks, device
// check, plans and workspace sizes.
#include <cstdint>

#include <hip/hip_runtime_api.h>

#include "prq.h"
#include "prq_internal.h"

namespace {

constexpr int kMaxHeads = 1024;
constexpr int64_t kMaxBlocks = ((int64_t{1} << 32) - 1) / 256;   // of 256 threads, in a launch
constexpr int kMaxSegments = 4096;
constexpr int kMaxRank = 256;

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int launch_status(hipError_t e) { return e == hipSuccess ? PRQ_OK : PRQ_EDEVICE; }

int check_heads(int32_t Hq, int32_t Hk, int32_t D) {
  if (Hq < 1 || Hk < 1 || Hq % Hk) return PRQ_EINVAL;
  if (Hq > kMaxHeads || (D != 64 && D != 128 && D != 256)) return PRQ_EUNSUPPORTED;
  return PRQ_OK;
}

// The cache's pool as the kernels take it.
int check_cache(const void* K, const void* V, int64_t page_stride, int32_t num_pages, int32_t page_size, int32_t Hk,
                int32_t D, prq::PagedCache* c) {
  if (!K || !V || num_pages < 1) return PRQ_EINVAL;
  if (page_size < 16 || page_size > 4096 || (page_size & (page_size - 1))) return PRQ_EUNSUPPORTED;
  if (page_stride < static_cast<int64_t>(Hk) * page_size * D) return PRQ_EINVAL;
  if (!aligned(K, 16) || !aligned(V, 16) || page_stride % 8) return PRQ_EALIGN;
  c->K = static_cast<uint16_t*>(const_cast<void*>(K));
  c->V = static_cast<uint16_t*>(const_cast<void*>(V));
  c->page_stride = page_stride;
  c->num_pages = num_pages;
  c->page_shift = 0;
  while ((1 << c->page_shift) < page_size) ++c->page_shift;
  return PRQ_OK;
}

int device_cus() {
  int cus = 0;
  return prq::current_device_cus(&cus) == PRQ_OK ? cus : 256;
}

int check_tree_sizes(int32_t M, int32_t B, int32_t Hq, int32_t Hk, int32_t D, int32_t max_kv_len) {
  if (M < 0 || B < 0 || max_kv_len < 0) return PRQ_EINVAL;
  const int st = check_heads(Hq, Hk, D);
  if (st != PRQ_OK) return st;
  if (B > kMaxSegments || static_cast<int64_t>(M) * Hq > (1 << 25)) return PRQ_EUNSUPPORTED;
  return PRQ_OK;
}

int check_lora_sizes(int32_t M, int32_t segments, int32_t N, int32_t K, int32_t max_rank) {
  if (M < 0 || segments < 0 || N <= 0 || K <= 0 || max_rank < 0) return PRQ_EINVAL;
  if (N % 16 || K % 8 || max_rank % 8) return PRQ_EALIGN;
  if (segments > kMaxSegments || max_rank > kMaxRank || K > (1 << 24) || N > (1 << 24) || M > (1 << 19))
    return PRQ_EUNSUPPORTED;
  return PRQ_OK;
}

}  // namespace

extern "C" {

int prq_qk_norm_rope(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                     int32_t in_type, int32_t M, int32_t Hq, int32_t Hk, int32_t D, const void* q_weight,
                     const void* k_weight, int32_t weight_type, float eps, const int32_t* positions,
                     const float* table, int32_t table_rows, int32_t rotary_dim, int32_t interleaved, void* q_out,
                     void* K_cache, void* V_cache, int64_t page_stride, int32_t num_pages, int32_t page_size,
                     const int64_t* slots, hipStream_t stream) {
  if (M < 0 || rotary_dim < 0 || table_rows < 0 || !(eps >= 0.0f)) return PRQ_EINVAL;
  if ((in_type != PRQ_F32 && in_type != PRQ_BF16) || (weight_type != PRQ_F32 && weight_type != PRQ_BF16) ||
      (interleaved != 0 && interleaved != 1))
    return PRQ_EINVAL;
  int st = check_heads(Hq, Hk, D);
  if (st != PRQ_OK) return st;
  if (rotary_dim > D || rotary_dim % 8) return PRQ_EALIGN;
  prq::PagedCache cache;
  st = check_cache(K_cache, V_cache, page_stride, num_pages, page_size, Hk, D, &cache);
  if (st != PRQ_OK) return st;
  if (M == 0) return PRQ_OK;
  if (M > kMaxBlocks) return PRQ_EUNSUPPORTED;
  if (!q || !k || !v || !q_out || !slots || (rotary_dim && (!positions || !table))) return PRQ_EINVAL;
  if (M > 1 && (ld_q < static_cast<int64_t>(Hq) * D || ld_k < static_cast<int64_t>(Hk) * D ||
                ld_v < static_cast<int64_t>(Hk) * D))
    return PRQ_EINVAL;
  const int wide = in_type == PRQ_F32 ? 4 : 8;         // elements of 16 bytes
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(table, 16) ||
      !aligned(q_weight, 16) || !aligned(k_weight, 16) ||
      (M > 1 && (ld_q % wide || ld_k % wide || ld_v % wide)))
    return PRQ_EALIGN;
  int cus = 0;
  st = prq::current_device_cus(&cus);
  if (st != PRQ_OK) return st;
  return launch_status(prq::launch_qk_norm_rope(
      q, ld_q, k, ld_k, v, ld_v, in_type == PRQ_BF16, M, Hq, Hk, D, q_weight, k_weight, weight_type == PRQ_BF16, eps,
      positions, table, table_rows, rotary_dim, interleaved != 0, static_cast<uint16_t*>(q_out), cache, slots, cus,
      stream));
}

size_t prq_tree_attention_workspace_bytes(int32_t M, int32_t B, int32_t Hq, int32_t Hk, int32_t D,
                                          int32_t max_kv_len) {
  if (check_tree_sizes(M, B, Hq, Hk, D, max_kv_len) != PRQ_OK || M == 0 || B == 0) return 0;
  return prq::tree_workspace_bytes(prq::plan_tree_attention(M, B, Hq, Hk, D, max_kv_len, device_cus()), M, D);
}

int prq_tree_attention(const void* q, int64_t ld_q, int32_t M, int32_t Hq, int32_t Hk, int32_t D,
                       const void* K_cache, const void* V_cache, int64_t page_stride, int32_t num_pages,
                       int32_t page_size, const int32_t* page_table, int64_t ld_pages, int32_t pages_wide,
                       const int32_t* cached_lens, const int32_t* q_offsets, int32_t B, int32_t max_kv_len,
                       float scale, const uint8_t* tree_mask, int64_t ld_mask, int32_t mask_wide, void* out,
                       float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int st = check_tree_sizes(M, B, Hq, Hk, D, max_kv_len);
  if (st != PRQ_OK) return st;
  prq::PagedCache cache;
  st = check_cache(K_cache, V_cache, page_stride, num_pages, page_size, Hk, D, &cache);
  if (st != PRQ_OK) return st;
  if (pages_wide < 0 || ld_pages < pages_wide || mask_wide < 0 || (tree_mask && ld_mask < mask_wide) ||
      scale != scale)
    return PRQ_EINVAL;
  if (static_cast<int64_t>(pages_wide) * page_size > (1 << 30)) return PRQ_EUNSUPPORTED;
  if (M == 0 || B == 0) return PRQ_OK;
  if (!q || !out || !cached_lens || !q_offsets || (pages_wide && !page_table)) return PRQ_EINVAL;
  if (M > 1 && ld_q < static_cast<int64_t>(Hq) * D) return PRQ_EINVAL;
  if (!aligned(q, 16) || !aligned(out, 16) || (M > 1 && ld_q % 8)) return PRQ_EALIGN;
  int cus = 0;
  st = prq::current_device_cus(&cus);
  if (st != PRQ_OK) return st;
  const prq::TreePlan plan = prq::plan_tree_attention(M, B, Hq, Hk, D, max_kv_len, cus);
  if (plan.blocks > kMaxBlocks) return PRQ_EUNSUPPORTED;
  const size_t need = prq::tree_workspace_bytes(plan, M, D);
  if (need && (!workspace || workspace_bytes < need)) return PRQ_EWORKSPACE;
  if (need && !aligned(workspace, 16)) return PRQ_EALIGN;
  return launch_status(prq::launch_tree_attention(
      plan, static_cast<const uint16_t*>(q), ld_q, M, Hq, Hk, D, cache, page_table, ld_pages, pages_wide * page_size,
      cached_lens, q_offsets, B, scale, tree_mask, ld_mask, mask_wide, static_cast<uint16_t*>(out), lse, workspace,
      stream));
}

size_t prq_lora_workspace_bytes(int32_t M, int32_t segments, int32_t N, int32_t K, int32_t max_rank) {
  if (check_lora_sizes(M, segments, N, K, max_rank) != PRQ_OK || M == 0 || segments == 0) return 0;
  return prq::lora_workspace_bytes(prq::plan_lora(M, segments, M, N, K, max_rank, device_cus()), M, max_rank);
}

int prq_lora_ex(const void* x_bf16, int64_t ld_x, int32_t M, int32_t K, const void* A, const void* B,
                const int32_t* rank_offsets, const int32_t* ranks, const float* scales, int32_t adapters,
                int32_t rank_rows, int32_t max_rank, const int32_t* segment_offsets,
                const int32_t* segment_adapter, int32_t segments, int32_t N, const float* Y, int64_t ld_y,
                float* out, int64_t ld_out, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (adapters < 0 || rank_rows < 0) return PRQ_EINVAL;
  int st = check_lora_sizes(M, segments, N, K, max_rank);
  if (st != PRQ_OK) return st;
  if (M == 0 || segments == 0) return PRQ_OK;
  if (!x_bf16 || !segment_offsets || !segment_adapter || !Y || !out || (adapters && (!rank_offsets || !scales)) ||
      (rank_rows && (!A || !B)))
    return PRQ_EINVAL;
  if (M > 1 && (ld_x < K || ld_y < N || ld_out < N)) return PRQ_EINVAL;
  if (out == Y && M > 1 && ld_y != ld_out) return PRQ_EINVAL;
  if (!aligned(x_bf16, 16) || !aligned(A, 16) || !aligned(B, 16) || !aligned(Y, 16) || !aligned(out, 16) ||
      (M > 1 && (ld_x % 8 || ld_y % 4 || ld_out % 4)))
    return PRQ_EALIGN;
  int cus = 0;
  st = prq::current_device_cus(&cus);
  if (st != PRQ_OK) return st;
  const prq::LoraPlan plan = prq::plan_lora(M, segments, adapters, N, K, max_rank, cus);
  const size_t need = prq::lora_workspace_bytes(plan, M, max_rank);
  if (need && (!workspace || workspace_bytes < need)) return PRQ_EWORKSPACE;
  if (need && !aligned(workspace, 16)) return PRQ_EALIGN;
  return launch_status(prq::launch_lora(
      plan, static_cast<const uint16_t*>(x_bf16), ld_x, M, K, static_cast<const uint16_t*>(A),
      static_cast<const uint16_t*>(B), rank_offsets, ranks, scales, adapters, rank_rows, max_rank, segment_offsets,
      segment_adapter, segments, N, Y, ld_y, out, ld_out, workspace, stream));
}

int prq_lora(const void* x_bf16, int64_t ld_x, int32_t M, int32_t K, const void* A, const void* B,
             const int32_t* rank_offsets, const float* scales, int32_t adapters, int32_t rank_rows,
             int32_t max_rank, const int32_t* segment_offsets, const int32_t* segment_adapter, int32_t segments,
             int32_t N, const float* Y, int64_t ld_y, float* out, int64_t ld_out, void* workspace,
             size_t workspace_bytes, hipStream_t stream) {
  return prq_lora_ex(x_bf16, ld_x, M, K, A, B, rank_offsets, nullptr, scales, adapters, rank_rows, max_rank,
                     segment_offsets, segment_adapter, segments, N, Y, ld_y, out, ld_out, workspace,
                     workspace_bytes, stream);
}

}  // extern "C"
