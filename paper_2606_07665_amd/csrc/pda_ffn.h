// Internal interface of the routing, expert and block norm kernels (not part
// of the public ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace pda {

constexpr int kMaxExperts = 1024;
constexpr int kMaxTopK = 16;
constexpr int kMaxRouteTokens = 1 << 20;
constexpr int kMaxMoeTokens = 256;
constexpr int kMaxMoePairs = kMaxMoeTokens * kMaxTopK;

struct RouteArgs {
  const float* logits;       // fp32 [tokens, stride]
  const float* select_bias;  // fp32 [experts] or null
  int32_t* ids;              // [tokens, top_k]
  float* weights;            // fp32 [tokens, top_k]
  int64_t stride;
  int tokens, experts, top_k;
  int sigmoid, renormalise;
  float scale;
};
hipError_t launch_route(const RouteArgs& a, hipStream_t st);

// A token's choice of an expert is a pair, p = token * top_k + j.
struct ExpertsArgs {
  const uint16_t* x;         // bf16 [tokens, hidden]
  const int32_t* ids;        // [tokens, top_k]; outside [0, experts): no expert
  const float* weights;      // fp32 [tokens, top_k]
  const uint16_t* w_gate_up; // packed bf16 [experts][2 inter, hidden]
  const uint16_t* w_down;    // packed bf16 [experts][hidden, inter]
  const uint16_t* residual;  // bf16 [tokens, hidden] or null
  uint16_t* out;             // bf16 [tokens, hidden]
  uint16_t* h;               // bf16 [pairs, inter] scratch
  float* y;                  // fp32 [pairs, hidden] scratch
  int tokens, hidden, inter, experts, top_k, activation;
};
hipError_t launch_experts(const ExpertsArgs& a, int num_cus, hipStream_t st);

constexpr int kMaxNormRows = 1 << 24;
struct BlockNormArgs {
  const uint16_t* y;         // bf16 [rows, hidden]
  const uint16_t* residual;  // bf16 [rows, hidden] or null
  const uint16_t* post_w;    // bf16 [hidden] or null
  const uint16_t* pre_w;     // bf16 [hidden] or null
  const uint16_t* gate;      // bf16 [hidden] or [rows, hidden], or null
  uint16_t* z;               // bf16 [rows, hidden]
  uint16_t* h;               // bf16 [rows, hidden], null without pre_w
  int64_t gate_stride;       // 0 or hidden
  int rows, hidden;
  float scale, weight_offset, eps;
};
hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t st);

}  // namespace pda
