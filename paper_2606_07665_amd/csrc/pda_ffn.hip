// Routing and block norms of a decode layer's feed-forward half for MI355X
// (gfx950, CDNA4, wave64).
#include "pda_ffn.h"

#include <type_traits>

#include "pda_device.h"

namespace pda {
namespace {

// ---------------------------------------------------------------- routing
// One wave per token; lane l holds the logits of experts l + 64 v.  top_k
// rounds pick the largest key that is left, ties to the lowest expert, then
// the lanes below top_k work out one weight each.
//
// Keys: the logits themselves where nothing is added to the scores (both
// scores grow with the logit, and the order of fp32 logits is exact); with a
// selection bias the scores plus the bias, in fp64, so that two experts next
// to each other are told apart by their scores and not by fp32's rounding.
//
// What bounds it is latency: 4 experts bytes a token in, then top_k dependent
// rounds.  A round's maximum goes through the wave by DPP moves (register to
// register); through LDS permutes a round would take several times as long.
constexpr int kRouteWaves = 4;

template <int kCtrl, int kRowMask>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  const uint32_t y = static_cast<uint32_t>(
      __builtin_amdgcn_update_dpp(0, static_cast<int>(x), kCtrl, kRowMask, 0xF, false));
  return y > x ? y : x;
}
// The wave's maximum, in every lane.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = dpp_max<0x111, 0xF>(x);  // row_shr:1
  x = dpp_max<0x112, 0xF>(x);  // row_shr:2
  x = dpp_max<0x114, 0xF>(x);  // row_shr:4
  x = dpp_max<0x118, 0xF>(x);  // row_shr:8
  x = dpp_max<0x142, 0xA>(x);  // row_bcast:15 into rows 1 and 3
  x = dpp_max<0x143, 0xC>(x);  // row_bcast:31 into rows 2 and 3
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), 63));
}

// Integers in the order of the numbers, above 0 (a NaN never comes here).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x == 0.f ? 0.f : x);  // -0 ties with 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x == 0.0 ? 0.0 : x);
  return b >> 63 ? ~b : b | (uint64_t{1} << 63);
}

template <int V, bool kBias>
__global__ __launch_bounds__(kRouteWaves * 64) void route_kernel(RouteArgs a) {
  using Key = typename std::conditional<kBias, uint64_t, uint32_t>::type;
  const int lane = threadIdx.x & 63;
  const int t = static_cast<int>(blockIdx.x) * kRouteWaves + uniform(threadIdx.x >> 6);
  if (t >= a.tokens) return;
  const float* row = a.logits + t * a.stride;
  const float kInf = __builtin_huge_valf(), kMost = 3.4028234663852886e38f;
  float x[V];
  float add[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = lane + 64 * v;
    x[v] = e < a.experts ? row[e] : -kInf;
    if constexpr (kBias) add[v] = e < a.experts ? a.select_bias[e] : 0.f;
  }
  float top = -kInf;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    x[v] = x[v] != x[v] ? -kInf : (x[v] > kMost ? kMost : x[v]);  // a NaN is never preferred, infinity a number
    top = fmaxf(top, x[v]);
  }
  {  // the row's largest logit
    const uint32_t m = wave_max(ordered(top));
    top = __builtin_bit_cast(float, m & 0x80000000u ? m & 0x7FFFFFFFu : ~m);
  }
  // the sum of exp(x - top), where a softmax's weights (or its keys) need it
  const bool masked = top == -kInf;  // no expert may be chosen: all weights are 0
  double total = 1.0;
  if (!a.sigmoid && (kBias || !a.renormalise)) {
    double s = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) s += masked ? 0.0 : exp(static_cast<double>(x[v]) - static_cast<double>(top));
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
    total = masked ? 1.0 : s;
  }
  auto score = [&](float l) -> double {
    if (l == -kInf) return 0.0;
    return a.sigmoid ? 1.0 / (1.0 + exp(-static_cast<double>(l)))
                     : exp(static_cast<double>(l) - static_cast<double>(top)) / total;
  };
  Key key[V];  // 0: not a candidate
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if constexpr (kBias)
      key[v] = lane + 64 * v >= a.experts ? 0
               : x[v] == -kInf            ? 1  // below every number that a score and a bias add up to
                                          : ordered(score(x[v]) + static_cast<double>(add[v]));
    else
      key[v] = lane + 64 * v >= a.experts ? 0 : ordered(x[v]);
  }
  int my_id = 0;
  float my_x = -kInf;
  for (int j = 0; j < a.top_k; ++j) {
    Key best = key[0];
    int at = 0;
#pragma unroll
    for (int v = 1; v < V; ++v) {
      const bool more = key[v] > best;
      best = more ? key[v] : best;
      at = more ? v : at;
    }
    bool mine;
    if constexpr (kBias) {
      const uint32_t hi = wave_max(static_cast<uint32_t>(best >> 32));
      mine = static_cast<uint32_t>(best >> 32) == hi;
      if (__popcll(__ballot(mine)) > 1) {
        const uint32_t lo = wave_max(mine ? static_cast<uint32_t>(best) : 0u);
        mine = mine && static_cast<uint32_t>(best) == lo;
      }
    } else {
      mine = best == wave_max(best);
    }
    // of equal keys the lowest expert, the largest of its complements
    uint64_t m = __ballot(mine);
    if (__popcll(m) > 1) {
      const uint32_t low = wave_max(mine ? ~static_cast<uint32_t>(lane + 64 * at) : 0u);
      mine = mine && ~static_cast<uint32_t>(lane + 64 * at) == low;
      m = __ballot(mine);
    }
    const int from = __builtin_ctzll(m);
    const int id = __builtin_amdgcn_readlane(lane + 64 * at, from);
    float xs = x[0];
#pragma unroll
    for (int v = 1; v < V; ++v) xs = at == v ? x[v] : xs;
    const int xb = __builtin_amdgcn_readlane(__builtin_bit_cast(int, xs), from);
    if (lane == j) {
      my_id = id;
      my_x = __builtin_bit_cast(float, xb);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane + 64 * v == id) key[v] = 0;
  }
  // weights in fp64: one value a lane
  double w = lane < a.top_k ? score(my_x) : 0.0;
  if (a.renormalise) {
    double s = w;
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) s += __shfl_xor(s, off);  // top_k is at most 16
    w = s > 0.0 ? w / s : 0.0;
  }
  if (lane < a.top_k) {
    const int64_t o = static_cast<int64_t>(t) * a.top_k + lane;
    a.ids[o] = my_id;
    a.weights[o] = static_cast<float>(w * static_cast<double>(a.scale));
  }
}

// ---------------------------------------------------------------- block norms
// One workgroup per row, 8 consecutive features a thread and pass:
//   u = post_w ? y / rms(y) * (post_w + offset) : y
//   z = residual + scale * gate * u,   h = z / rms(z) * (pre_w + offset)
// The row stays in registers between the sums; h is taken from the unrounded z.
template <int kThreads, int kPasses>
__global__ __launch_bounds__(kThreads) void block_norm_kernel(BlockNormArgs a) {
  constexpr int kWaves = kThreads / 64;
  __shared__ float part[2][kWaves];
  const int64_t base = static_cast<int64_t>(blockIdx.x) * a.hidden;
  auto row_sum = [&](float s, int which) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off);
    if ((threadIdx.x & 63) == 0) part[which][threadIdx.x >> 6] = s;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) t += part[which][i];
    return t;
  };
  uint32_t ry[kPasses][4], rr[kPasses][4], rg[kPasses][4], rp[kPasses][4], rn[kPasses][4];
  float z[kPasses][8];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int n = 8 * (static_cast<int>(threadIdx.x) + i * kThreads);
#pragma unroll
    for (int j = 0; j < 4; ++j) ry[i][j] = rr[i][j] = rp[i][j] = rn[i][j] = 0u, rg[i][j] = 0x3F803F80u;  // gate 1
    if (n < a.hidden) {
      load_bf16<8>(a.y + base + n, ry[i]);
      if (a.residual) load_bf16<8>(a.residual + base + n, rr[i]);
      if (a.gate) load_bf16<8>(a.gate + blockIdx.x * a.gate_stride + n, rg[i]);
      if (a.post_w) load_bf16<8>(a.post_w + n, rp[i]);
      if (a.pre_w) load_bf16<8>(a.pre_w + n, rn[i]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z[i][j] = unpack_bf16(ry[i], j);
      ss += z[i][j] * z[i][j];
    }
  }
  if (a.post_w) {
    const float inv = rsqrtf(row_sum(ss, 0) / a.hidden + a.eps);
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) z[i][j] = z[i][j] * inv * (unpack_bf16(rp[i], j) + a.weight_offset);
  }
  ss = 0.f;
#pragma unroll
  for (int i = 0; i < kPasses; ++i)
    if (8 * (static_cast<int>(threadIdx.x) + i * kThreads) < a.hidden) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (a.gate) z[i][j] *= unpack_bf16(rg[i], j);
        z[i][j] = unpack_bf16(rr[i], j) + a.scale * z[i][j];
        ss += z[i][j] * z[i][j];
      }
      store_bf16<8>(a.z + base + 8 * (static_cast<int>(threadIdx.x) + i * kThreads), z[i]);
    }
  if (!a.pre_w) return;
  const float inv = rsqrtf(row_sum(ss, 1) / a.hidden + a.eps);
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int n = 8 * (static_cast<int>(threadIdx.x) + i * kThreads);
    if (n >= a.hidden) continue;
    float h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = z[i][j] * inv * (unpack_bf16(rn[i], j) + a.weight_offset);
    store_bf16<8>(a.h + base + n, h);
  }
}

template <int V>
hipError_t route_as(const RouteArgs& a, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>((a.tokens + kRouteWaves - 1) / kRouteWaves));
  if (a.select_bias)
    hipLaunchKernelGGL((route_kernel<V, true>), grid, dim3(kRouteWaves * 64), 0, st, a);
  else
    hipLaunchKernelGGL((route_kernel<V, false>), grid, dim3(kRouteWaves * 64), 0, st, a);
  return hipGetLastError();
}

// A launch takes fewer than 2^32 threads: more rows (of 8192 features 4194304, 68
// GB) go in several.
constexpr int64_t kNormThreadsALaunch = int64_t{1} << 31;
template <int kThreads, int kPasses>
hipError_t block_norm_as(BlockNormArgs a, hipStream_t st) {
  constexpr int kMost = static_cast<int>(kNormThreadsALaunch / kThreads);
  for (int left = a.rows; left > 0; left -= kMost) {
    a.rows = left < kMost ? left : kMost;
    hipLaunchKernelGGL((block_norm_kernel<kThreads, kPasses>), dim3(static_cast<unsigned>(a.rows)), dim3(kThreads), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t on = static_cast<int64_t>(a.rows) * a.hidden;
    a.y += on;
    a.z += on;
    if (a.residual) a.residual += on;
    if (a.gate) a.gate += a.rows * a.gate_stride;
    if (a.h) a.h += on;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t st) {
  if (a.experts <= 64) return route_as<1>(a, st);
  if (a.experts <= 128) return route_as<2>(a, st);
  if (a.experts <= 256) return route_as<4>(a, st);
  if (a.experts <= 512) return route_as<8>(a, st);
  return route_as<16>(a, st);
}

hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t st) {
  if (a.hidden <= 512) return block_norm_as<64, 1>(a, st);
  if (a.hidden <= 1024) return block_norm_as<128, 1>(a, st);
  if (a.hidden <= 2048) return block_norm_as<256, 1>(a, st);
  if (a.hidden <= 4096) return block_norm_as<512, 1>(a, st);
  if (a.hidden <= 8192) return block_norm_as<1024, 1>(a, st);
  if (a.hidden <= 16384) return block_norm_as<1024, 2>(a, st);
  return block_norm_as<1024, 4>(a, st);
}

}  // namespace pda
