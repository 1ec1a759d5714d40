// Device helpers that the projection, feed-forward and expert kernels share
// (not part of the public ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "pda.h"
#include "pda_gemv.h"

namespace pda {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBufferDword3 = 0x00020000;  // raw 32-bit buffer format
constexpr int kCachePolicyNT = 2;          // non-temporal: weights are read once

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32));
  void* ub = reinterpret_cast<void*>((static_cast<uint64_t>(hi) << 32) | lo);
  return __builtin_amdgcn_make_buffer_rsrc(ub, 0, static_cast<int>(__builtin_amdgcn_readfirstlane(bytes)),
                                           kBufferDword3);
}

__device__ __forceinline__ float bf16_to_f32(uint16_t h) {
  return __builtin_bit_cast(float, static_cast<uint32_t>(h) << 16);
}

__device__ __forceinline__ uint16_t f32_to_bf16(float f) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f));
}

// s_waitcnt vmcnt(n) alone; vmcnt is split over bits 3:0 and 15:14
constexpr int kWaitLoads = 0x0F70;
constexpr int wait_loads(int n) { return kWaitLoads | (n & 15) | ((n >> 4) << 14); }

// N consecutive bf16 values, packed two to a register; p need only be 2-byte
// aligned (the memory pipeline takes any alignment).
template <int N>
__device__ __forceinline__ void load_bf16(const uint16_t* p, uint32_t* v) {
  __builtin_memcpy(v, p, 2 * N);
}
__device__ __forceinline__ float unpack_bf16(const uint32_t* v, int j) {
  return bf16_to_f32(static_cast<uint16_t>(v[j / 2] >> (16 * (j & 1))));
}
template <int N>
__device__ __forceinline__ void store_bf16(uint16_t* p, const float (&v)[N]) {
  uint32_t w[N / 2];
#pragma unroll
  for (int j = 0; j < N / 2; ++j)
    w[j] = f32_to_bf16(v[2 * j]) | (static_cast<uint32_t>(f32_to_bf16(v[2 * j + 1])) << 16);
  __builtin_memcpy(p, w, 2 * N);
}

// N consecutive features of a linear product, from element `at` on.
template <int N>
__device__ __forceinline__ void store_features(const LinearArgs& e, int64_t at, const float (&v)[N]) {
  if (e.f32)
    __builtin_memcpy(static_cast<float*>(e.out) + at, v, 4 * N);
  else
    store_bf16<N>(static_cast<uint16_t*>(e.out) + at, v);
}

// The activations of a feed-forward layer: silu(x) = x / (1 + exp(-x)), gelu(x)
// = x erfc(-x / sqrt 2) / 2, and its tanh form x / (1 + exp(-2 u)) with
// u = sqrt(2 / pi) (x + 0.044715 x^3).  Where the exponential overflows the
// quotient is 0; its argument z is rounded to fp32, which costs |z| 2^-24 of a
// value that has itself fallen by exp(z), z < 0.  The hardware's exponential and
// reciprocal are off by a step of fp32 each, which is far below the rounding of a
// bf16 output and shows in an fp32 one as a few steps.
__device__ __forceinline__ float over_exp(float x, float z) {  // x / (1 + exp(-z))
  return x * __builtin_amdgcn_rcpf(1.f + __expf(-z));
}
// All N with one branch: a branch for each took 12 us of 250 sequences' epilogue
// (linear_stream_kernel, the waves two to a SIMD).
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int kind) {
  if (kind == PDA_ACT_NONE) return;
  if (kind == PDA_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = v[j] < 0.f ? 0.f : v[j];  // (a NaN stays)
    return;
  }
  float y[N];
  if (kind == PDA_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = over_exp(v[j], v[j]);
  } else if (kind == PDA_ACT_GELU_TANH) {
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = over_exp(v[j], 1.59576912f * (v[j] + 0.044715f * v[j] * v[j] * v[j]));
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) y[j] = 0.5f * v[j] * erfcf(-0.70710678f * v[j]);
  }
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = v[j] == -__builtin_huge_valf() ? 0.f : y[j];  // the limit, not -inf * 0
}

}  // namespace
}  // namespace pda
