// C ABI of the mixture-of-experts half of a layer (include/prq.h): argument checks, device
// check, plans and workspace sizes.
#include <cmath>
#include <cstdint>
#include <cstring>
#include <tuple>
#include <type_traits>
#include <utility>

#include <hip/hip_runtime_api.h>

#include "prq.h"
#include "prq_internal.h"

namespace {

constexpr int kMaxRows = (1 << 24) - 1;              // 256 threads each fit a launch
constexpr int kMaxWidth = 65536;
constexpr int kMaxIntermediate = 32768;
constexpr int kMaxExperts = 4096;

bool aligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int launch_status(hipError_t e) { return e == hipSuccess ? PRQ_OK : PRQ_EDEVICE; }

int device_cus() {
  int cus = 0;
  return prq::current_device_cus(&cus) == PRQ_OK ? cus : 256;
}

bool is_type(int32_t t) { return t == PRQ_F32 || t == PRQ_BF16; }

// A matrix of M rows of `wide` elements of `type`, ld apart, is there and its rows are aligned.
int check_rows(const void* p, int64_t ld, int64_t M, int64_t wide, int32_t type) {
  if (!p || (M > 1 && ld < wide)) return PRQ_EINVAL;
  if (!aligned(p, 16) || (M > 1 && ld % (type == PRQ_F32 ? 4 : 8))) return PRQ_EALIGN;
  return PRQ_OK;
}

int check_route_sizes(int32_t M, int32_t E, int32_t H) {
  if (M < 0 || E < 1 || H < 1) return PRQ_EINVAL;
  if (H % 8) return PRQ_EALIGN;
  if (M > kMaxRows || E > prq::kMaxRouteExperts || H > kMaxWidth) return PRQ_EUNSUPPORTED;
  return PRQ_OK;
}

int check_layer_sizes(int32_t M, int32_t k, int32_t E, int32_t H, int32_t I, int32_t k_tail, int32_t N) {
  if (M < 0 || k < 1 || E < 1 || H < 1 || I < 1 || k_tail < 0 || N < 1) return PRQ_EINVAL;
  if (H % 32 || I % 32 || k_tail % 32 || k_tail > I || N % 16) return PRQ_EALIGN;
  if (M > prq::kMaxLayerTokens || k > prq::kMaxLayerTop || E > kMaxExperts || H > kMaxWidth || N > kMaxWidth ||
      I > kMaxIntermediate)
    return PRQ_EUNSUPPORTED;
  return PRQ_OK;
}

prq::MoeArgs layer_sizes(int32_t M, int32_t k, int32_t E, int32_t H, int32_t I, int32_t k_tail, int32_t N) {
  prq::MoeArgs p{};
  p.M = M, p.k = k, p.E = E, p.H = H, p.I = I, p.k_tail = k_tail, p.N = N;
  return p;
}

// One argument of a record as its parameter's type; fits: an integer lies in that type's range.
template <typename T>
T argument(uint64_t raw, bool& fits) {
  if constexpr (std::is_pointer_v<T>) {
    return reinterpret_cast<T>(static_cast<uintptr_t>(raw));
  } else if constexpr (std::is_floating_point_v<T>) {
    double v;
    std::memcpy(&v, &raw, sizeof(v));
    return static_cast<T>(v);
  } else {
    if (sizeof(T) < 8 && static_cast<int64_t>(raw) != static_cast<int64_t>(static_cast<T>(raw))) fits = false;
    return static_cast<T>(raw);
  }
}
template <typename... T, size_t... kAt>
int call_record(int (*call)(T...), const void* record, std::index_sequence<kAt...>) {
  uint64_t raw[sizeof...(T)];
  if (!record) return PRQ_EINVAL;
  std::memcpy(raw, record, sizeof(raw));
  bool fits = true;
  const std::tuple<T...> arguments{argument<T>(raw[kAt], fits)...};
  return fits ? call(std::get<kAt>(arguments)...) : PRQ_EINVAL;
}
template <typename... T>
int call_record(int (*call)(T...), const void* record) {
  return call_record(call, record, std::index_sequence_for<T...>{});
}

}  // namespace

extern "C" {

int prq_block_norm(const void* y, int64_t ld_y, int32_t y_type, const void* residual, int64_t ld_r, int32_t r_type,
                   int32_t M, int32_t H, const void* post_weight, const void* pre_weight, int32_t weight_type,
                   float weight_offset, const void* gate, int64_t ld_gate, int32_t gate_type, int32_t gate_rows,
                   const int32_t* gate_index, float eps, float residual_scale, float block_scale,
                   void* residual_out, int64_t ld_ro, void* h_out, int64_t ld_h, hipStream_t stream) {
  if (M < 0 || H < 1 || !(eps >= 0.0f) || !std::isfinite(weight_offset) || !std::isfinite(residual_scale) ||
      !std::isfinite(block_scale))
    return PRQ_EINVAL;
  if (!is_type(y_type) || !is_type(r_type) || !is_type(weight_type) || !is_type(gate_type)) return PRQ_EINVAL;
  if (H % 8) return PRQ_EALIGN;
  if (H > prq::kMaxNormWidth || M > kMaxRows) return PRQ_EUNSUPPORTED;
  if (M == 0) return PRQ_OK;
  if ((!y && !residual) || (!residual_out && !h_out) || (h_out != nullptr) != (pre_weight != nullptr) ||
      (!y && (post_weight || gate)) || (gate_index && !gate))
    return PRQ_EINVAL;
  if (gate && (gate_rows < 1 || (!gate_index && gate_rows != 1 && gate_rows != M))) return PRQ_EINVAL;
  if (residual_out && residual_out == residual && M > 1 && ld_ro != ld_r) return PRQ_EINVAL;
  int st = y ? check_rows(y, ld_y, M, H, y_type) : PRQ_OK;
  if (st == PRQ_OK && residual) st = check_rows(residual, ld_r, M, H, r_type);
  if (st == PRQ_OK && gate) st = check_rows(gate, ld_gate, gate_rows, H, gate_type);
  if (st == PRQ_OK && residual_out) st = check_rows(residual_out, ld_ro, M, H, r_type);
  if (st == PRQ_OK && h_out) st = check_rows(h_out, ld_h, M, H, PRQ_BF16);
  if (st != PRQ_OK) return st;
  if (!aligned(post_weight, 16) || !aligned(pre_weight, 16) || !aligned(gate_index, 4)) return PRQ_EALIGN;
  int cus = 0;
  st = prq::current_device_cus(&cus);
  if (st != PRQ_OK) return st;
  const prq::BlockNormArgs p{y, residual, ld_y, ld_r, post_weight, pre_weight, gate, ld_gate, gate_index,
                             residual_out, ld_ro, static_cast<uint16_t*>(h_out), ld_h, M, H, gate_rows,
                             weight_type == PRQ_BF16, gate_type == PRQ_BF16, weight_offset, eps, residual_scale,
                             block_scale};
  return launch_status(prq::launch_block_norm(p, y_type == PRQ_BF16, r_type == PRQ_BF16, stream));
}

size_t prq_moe_route_workspace_bytes(int32_t M, int32_t E, int32_t H) {
  if (check_route_sizes(M, E, H) != PRQ_OK || M == 0) return 0;
  return prq::route_workspace_bytes(prq::plan_moe_route(M, E, H, device_cus()), M, E);
}

int prq_moe_route(const void* x_bf16, int64_t ld_x, int32_t M, int32_t H, const void* W_bf16, int64_t ld_w, int32_t E,
                  int32_t k, int32_t scoring, const float* bias, int32_t renormalize, float scale, int32_t* ids,
                  float* weights, float* logits, int64_t ld_logits, void* workspace, size_t workspace_bytes,
                  hipStream_t stream) {
  int st = check_route_sizes(M, E, H);
  if (st != PRQ_OK) return st;
  if (k < 1 || k > E || (scoring != PRQ_ROUTE_SOFTMAX && scoring != PRQ_ROUTE_SIGMOID) ||
      (renormalize != 0 && renormalize != 1) || !std::isfinite(scale) || (bias && scoring != PRQ_ROUTE_SIGMOID))
    return PRQ_EINVAL;
  if (k > prq::kMaxRouteTop) return PRQ_EUNSUPPORTED;
  if (M == 0) return PRQ_OK;
  if (!ids || !weights || (logits && M > 1 && ld_logits < E)) return PRQ_EINVAL;
  st = check_rows(x_bf16, ld_x, M, H, PRQ_BF16);
  if (st == PRQ_OK) st = check_rows(W_bf16, ld_w, E, H, PRQ_BF16);
  if (st != PRQ_OK) return st;
  if (!aligned(ids, 4) || !aligned(weights, 4) || !aligned(logits, 4) || !aligned(bias, 4)) return PRQ_EALIGN;
  int cus = 0;
  st = prq::current_device_cus(&cus);
  if (st != PRQ_OK) return st;
  const prq::RoutePlan plan = prq::plan_moe_route(M, E, H, cus);
  const size_t need = prq::route_workspace_bytes(plan, M, E);
  if (need && (!workspace || workspace_bytes < need)) return PRQ_EWORKSPACE;
  if (need && !aligned(workspace, 16)) return PRQ_EALIGN;
  const prq::RouteArgs p{static_cast<const uint16_t*>(x_bf16), static_cast<const uint16_t*>(W_bf16), ld_x, ld_w, bias,
                         ids, weights, logits, ld_logits, M, E, H, k, scoring == PRQ_ROUTE_SIGMOID, renormalize != 0,
                         scale};
  return launch_status(prq::launch_moe_route(plan, p, workspace, stream));
}

size_t prq_moe_layer_workspace_bytes(int32_t M, int32_t k, int32_t E, int32_t H, int32_t I, int32_t k_tail,
                                     int32_t N) {
  if (check_layer_sizes(M, k, E, H, I, k_tail, N) != PRQ_OK || M == 0) return 0;
  const prq::MoeArgs p = layer_sizes(M, k, E, H, I, k_tail, N);
  return prq::moe_workspace_bytes(prq::plan_moe_layer(p, device_cus()), p);
}

int prq_moe_layer(const void* x_bf16, int64_t ld_x, int32_t M, const int32_t* ids, const float* weights, int32_t k,
                  const uint8_t* up_Wp, const uint8_t* up_Wps, const uint8_t* down_Wp, const uint8_t* down_Wps,
                  int32_t E, int32_t H, int32_t I, int32_t k_tail, int32_t N, void* out, int64_t ld_out,
                  void* workspace, size_t workspace_bytes, hipStream_t stream) {
  int st = check_layer_sizes(M, k, E, H, I, k_tail, N);
  if (st != PRQ_OK) return st;
  if (M == 0) return PRQ_OK;
  if (!ids || !weights || !up_Wp || !up_Wps || !down_Wp || !down_Wps) return PRQ_EINVAL;
  st = check_rows(x_bf16, ld_x, M, H, PRQ_BF16);
  if (st == PRQ_OK) st = check_rows(out, ld_out, M, N, PRQ_BF16);
  if (st != PRQ_OK) return st;
  if (!aligned(ids, 4) || !aligned(weights, 4) || !aligned(up_Wp, 16) || !aligned(up_Wps, 16) ||
      !aligned(down_Wp, 16) || !aligned(down_Wps, 16))
    return PRQ_EALIGN;
  int cus = 0;
  st = prq::current_device_cus(&cus);
  if (st != PRQ_OK) return st;
  prq::MoeArgs p = layer_sizes(M, k, E, H, I, k_tail, N);
  const prq::MoePlan plan = prq::plan_moe_layer(p, cus);
  if (!workspace || workspace_bytes < prq::moe_workspace_bytes(plan, p)) return PRQ_EWORKSPACE;
  if (!aligned(workspace, 16)) return PRQ_EALIGN;
  p.x = static_cast<const uint16_t*>(x_bf16);
  p.ld_x = ld_x;
  p.ids = ids;
  p.weights = weights;
  p.up_codes = up_Wp, p.up_scales = up_Wps, p.down_codes = down_Wp, p.down_scales = down_Wps;
  p.out = static_cast<uint16_t*>(out);
  p.ld_out = ld_out;
  return launch_status(prq::launch_moe_layer(plan, p, workspace, stream));
}

int prq_block_norm_record(const void* record) { return call_record(prq_block_norm, record); }
int prq_moe_route_record(const void* record) { return call_record(prq_moe_route, record); }
int prq_moe_layer_record(const void* record) { return call_record(prq_moe_layer, record); }

}  // extern "C"
