// Internal interface of the routing, expert and block norm kernels (not part
// of the public ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "pda_gemv.h"

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
  float* y;                  // fp32 [splits, pairs, hidden] scratch
  int tokens, hidden, inter, experts, top_k, activation;
  bool weighted_h;           // h carries the pair's weight
  int splits;                // parts of the down products' k range
};

// Segments of up to `cols` pairs of one expert: the most that the pairs make.
constexpr int kMoeCols = 128;
inline int moe_most_segments(int pairs, int experts, int cols) {
  const int most = experts < pairs ? experts : pairs;  // experts that any pair may ask for
  return (pairs + most * (cols - 1)) / cols;
}

// Whether the waves of a workgroup share each pair of row tiles (`tiles` of them
// an expert) instead of taking one each: where the pairs of tiles of all segments
// (of up to 32 pairs) are too few to keep the chip's waves busy one by one.  us,
// a pair of tiles a wave -> shared; gate and up: 1 token over 128 experts of 768
// 15.5 -> 11.7, 4 tokens 38.6 -> 35.6, 24 tokens of 5 pairs over 8 of 480 14.8 ->
// 9.2, 200 of 2 over 8 of 512 22.2 -> 10.9, 33 of 2 over 8 of 1024 (4096 features)
// 35.2 -> 27.6, 93 of 3 over 64 of 384 (1680 workgroups) 23.2 -> 23.6; down: the
// same 7.0 -> 6.5, 13.0 -> 6.9, 16.7 -> 15.0, 67 tokens of 8 over 32 (2538) 16.7 ->
// 21.7.  Up to twice as many stay ahead where an expert has few pairs and the
// products' k range is long (cold weights; gate and up of 2240 features: 33 tokens
// of 4 over 16 of 2272, 2698 workgroups, 59.2 -> 53.7; 33 of 3 over 64 of 512, 2080,
// 40.4 -> 32.6; 80 of 4 over 16 of 1056, 1650, 56.0 -> 54.0; 128 of 6 over 32 of 512,
// 24 pairs each, 1760, 37.3 -> 38.0; down: 33 of 4 over 16 of 2272, 1330, 36.5 ->
// 30.9; k 512: 33 of 6 over 32, 2368, 15.9 -> 18.7).
constexpr int kMoeFewCols = 32;
inline bool moe_shares_tiles(int tokens, int pairs, int experts, int tiles, int k, int num_cus) {
  const int a_cu = k >= 1536 && pairs <= 20 * experts ? 11 : tokens <= 8 ? 8 : 5;
  return static_cast<int64_t>(moe_most_segments(pairs, experts, kMoeFewCols)) * tiles <= static_cast<int64_t>(a_cu) * num_cus;
}

// Parts of the down products' k range: doubled while the workgroups (128 rows
// of a segment) are fewer than four a CU and a part keeps 20 steps of 64 k: 8
// experts of 14336, 200 tokens to 4096 rows, 264, 246 and 236 us in 1, 2 and 4
// parts; shorter ranges only lose (32 of 512, 256 tokens: 19, 26, 35).
constexpr int kMaxMoeSplits = 8;
inline int moe_splits(int pairs, int experts, int hidden, int inter, int num_cus) {
  const int64_t workgroups = static_cast<int64_t>(moe_most_segments(pairs, experts, kMoeCols)) * ((hidden + 127) / 128);
  const int steps = (inter + 63) / 64;
  int splits = 1;
  while (splits < kMaxMoeSplits && workgroups * splits < 4 * num_cus && steps / (2 * splits) >= 20) splits *= 2;
  return splits;
}
// Floats of y that moe_splits() asks for, never less for more pairs: several
// parts are fewer than 8 workgroups a CU, of 128 rows x 128 pairs.
inline int64_t moe_most_floats(int pairs, int hidden, int num_cus) {
  const int64_t one = static_cast<int64_t>(pairs) * hidden, bound = int64_t{8} * num_cus * 128 * kMoeCols;
  const int64_t most = kMaxMoeSplits * one < bound ? kMaxMoeSplits * one : bound;
  return one > most ? one : most;
}

// How a call runs: what it launches and what it writes of the workspace.
struct ExpertsPlan {
  bool shared_up, shared_down;  // waves share row tiles, of the gate and up or of the down products
  bool joined;                  // down products and combination in one kernel; h carries the pair's weight
  int splits;                   // parts of the down products' k range
  int64_t y_floats;             // of y
};
inline ExpertsPlan plan_experts(int tokens, int hidden, int inter, int experts, int top_k, int num_cus) {
  const int pairs = tokens * top_k;
  ExpertsPlan p{};
  p.shared_up = moe_shares_tiles(tokens, pairs, experts, inter / kTileRows, hidden, num_cus);
  p.joined = tokens <= 8 && pairs <= 64;
  p.shared_down = !p.joined && moe_shares_tiles(tokens, pairs, experts, hidden / (2 * kTileRows), inter, num_cus);
  p.splits = p.joined || p.shared_down ? 1 : moe_splits(pairs, experts, hidden, inter, num_cus);
  p.y_floats = p.joined ? 0 : static_cast<int64_t>(p.splits) * pairs * hidden;
  return p;
}
hipError_t launch_experts(const ExpertsArgs& a, const ExpertsPlan& p, hipStream_t st);

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
