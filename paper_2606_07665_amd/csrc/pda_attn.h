// Device helpers that the attention kernels share (pda_kernels.hip, pda_kv4.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pda_internal.h"

namespace pda {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__device__ __forceinline__ int clamp_len(int L, int max_ctx) {
  return L < 0 ? 0 : (L > max_ctx ? max_ctx : L);
}

// Key range of a sequence.  Its nq query tokens are its last nq tokens:
// query j sits at position L - nq + j and sees keys up to that position, and
// with a sliding window of W > 0 tokens only the W keys ending there.  The
// first key any query sees is seq_start; the steps of the sequence are the
// 32-token steps from the one holding seq_start to the end.  With S > 0 sinks
// (a window only) every query sees the keys t < S as well: the sequence then
// has the sink_steps steps that hold them ahead of the window's, those before
// the window's first step.  (window and sinks are at most the tokens of a
// table, 2^30: nothing here passes 32 bits.)
__device__ __forceinline__ int seq_start(int L, int nq, int window) {
  if (window <= 0) return 0;
  const int s = L - nq + 1 - window;
  return s > 0 ? s : 0;
}

__device__ __forceinline__ int sink_steps(int L, int nq, int window, int sinks) {
  if (window <= 0 || sinks <= 0) return 0;
  const int first = seq_start(L, nq, window);  // keys [0, min(sinks, first)) are seen as sinks
  const int pinned = ((sinks < first ? sinks : first) + kStep - 1) / kStep;
  return pinned < first / kStep ? pinned : first / kStep;
}

__device__ __forceinline__ int seq_steps(int L, int nq, int window, int sinks = 0) {
  return (L + kStep - 1) / kStep - seq_start(L, nq, window) / kStep + sink_steps(L, nq, window, sinks);
}

__device__ __forceinline__ u32x4 ld16(const uint16_t* p) {
  return *reinterpret_cast<const u32x4*>(p);
}

// K and V are read exactly once per call, with raw buffer loads:
//  * non-temporal (cache policy NT): on MI355X a plain streaming read runs at
//    ~7.1 TB/s this way against ~6.1 TB/s with default loads;
//  * the descriptor's base is the page (a wave-uniform 64-bit address) and
//    its size covers only the valid token rows, so rows past the end of the
//    sequence, or a step that does not exist, read as zeros without touching
//    memory.
constexpr int kBufferDword3 = 0x00020000;  // raw buffer, 32-bit data format (gfx9 family)
constexpr int kCachePolicyNT = 2;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_rsrc(const void* base, int bytes) {
  // the base is wave-uniform; passing it through readfirstlane keeps the
  // descriptor in SGPRs (a 64-bit VALU add would otherwise leave it in VGPRs
  // and every load would be wrapped in a waterfall loop)
  const uint64_t a = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(a >> 32));
  void* ub = reinterpret_cast<void*>((static_cast<uint64_t>(hi) << 32) | lo);
  return __builtin_amdgcn_make_buffer_rsrc(ub, 0, uniform(bytes), kBufferDword3);
}
__device__ __forceinline__ u32x4 ld16_stream(__amdgpu_buffer_rsrc_t r, int byte_off) {
  return __builtin_amdgcn_raw_buffer_load_b128(r, byte_off, 0, kCachePolicyNT);
}

// Quotients on the way to the first loads of the fixed split and its
// merge.  The compiler expands a 32-bit integer division into ~25 dependent
// instructions; these divide in fp64 instead: both operands (0 <= a < 2^31,
// 0 < b < 2^31) convert exactly and the quotient a/b, correctly rounded,
// cannot reach the next integer (it is at least 1/b below it, more than the
// rounding error of a quotient below 2^31), so truncation gives
// floor(a / b).  div_small_u is the same for wave-uniform operands: the
// quotient is computed in vector registers (the scalar unit has no fp64)
// and readfirstlane returns it to scalar registers, so that nothing derived
// from it takes vector registers.  (The stream-K prologue keeps the
// compiler's integer division: there the fp64 form measured no faster and
// cost the main loop vector registers.)
__device__ __forceinline__ int div_small(int a, int b) {
  return static_cast<int>(static_cast<double>(a) / static_cast<double>(b));
}
__device__ __forceinline__ int div_small_u(int a, int b) { return uniform(div_small(a, b)); }

// Values with an infinity or a NaN that some query tokens of a sequence see and
// others do not (drafted tokens after a query, the far end of its window): as a
// row of the product P V they would reach every column, 0 * NaN of those that
// do not see them.  Such a row is taken out of the product: its token's
// probabilities times the row are added here to the columns that see it, and
// the row in LDS becomes zeros.  hi, lo: the lane's probabilities as the product
// takes them, element 4 T + i that of token 16 T + 4 (lane / 16) + i; r: the
// token's row in the tile at `rows`; acc: lane (g4, c) holds column c, element i
// of tile dt that of d = 16 dt + 4 g4 + i.
template <int D, int kRowBytes>
__device__ __forceinline__ void add_row_apart(f32x4 (&acc)[D / 16], u32x4 hi, u32x4 lo, unsigned char* rows, int r, bool sees) {
  const int lane = threadIdx.x & 63;
  const int word = 2 * (r >> 4) + ((r & 3) >> 1);
  unsigned h = hi[0], l = lo[0];
#pragma unroll
  for (int k = 1; k < 4; ++k) {
    h = word == k ? hi[k] : h;
    l = word == k ? lo[k] : l;
  }
  const int from = 16 * ((r >> 2) & 3) + (lane & 15);
  h = static_cast<unsigned>(__shfl(static_cast<int>(h), from, 64));
  l = static_cast<unsigned>(__shfl(static_cast<int>(l), from, 64));
  const int shift = r & 1 ? 0 : 16;
  const float p = __builtin_bit_cast(float, (h << shift) & 0xFFFF0000u) + __builtin_bit_cast(float, (l << shift) & 0xFFFF0000u);
  unsigned char* row = rows + r * kRowBytes;
#pragma unroll
  for (int dt = 0; dt < D / 16; ++dt) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(row + 32 * dt + 8 * (lane >> 4));
    f32x4 add;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned w = v[i >> 1];
      const float x = __builtin_bit_cast(float, i & 1 ? w & 0xFFFF0000u : w << 16);
      add[i] = sees ? p * x : 0.f;
    }
    acc[dt] += add;
    __builtin_amdgcn_sched_barrier(0);  // (a tile at a time: rare, and no registers of the loop for it)
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");  // every lane's reads before the zeros
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  if (8 * lane < 2 * D) *reinterpret_cast<u32x2*>(row + 8 * lane) = u32x2{0u, 0u};
}

// Workgroup that owns flattened step x of `total`, when `parts` workgroups
// split [0, total) into ranges [w*total/parts, (w+1)*total/parts).
__device__ __forceinline__ int64_t owner_of(int64_t x, int64_t total, int64_t parts) {
  return ((x + 1) * parts - 1) / total;
}

}  // namespace pda
