// Internal interface of the 4-bit KV cache's kernels (not part of the public ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "pda_internal.h"

namespace pda {

constexpr int kKv4Group = 32;       // elements of a row that share a scale
constexpr int kKv4Threads = 256;    // append and read
constexpr int kKv4MaxTokens = 1 << 20;  // new tokens per sequence of an append or a read

// A 4-bit cache, and the tokens that an append writes to it or a read takes
// from it: the last `tokens` of each sequence.
struct Kv4Args {
  uint8_t* k;         // codes [num_pages, hkv, head_dim / 32, page_size, 16]
  uint8_t* ks;        // scales [num_pages, hkv, head_dim / 32, page_size]
  uint8_t* v;
  uint8_t* vs;
  const int32_t* bt;    // [batch, maxp]
  const int32_t* lens;  // [batch], counting the new tokens
  int batch, tokens, hkv, head_dim, page_shift, num_pages, maxp;
};

hipError_t launch_kv4_append(const Kv4Args& a, const uint16_t* k_new, const uint16_t* v_new, hipStream_t st);
hipError_t launch_kv4_read(const Kv4Args& a, uint16_t* k_out, uint16_t* v_out, hipStream_t st);

// Attention over the cache; `a` as for the bf16 kernel but for the caches,
// which `c` names (a.k and a.v are not read).
hipError_t launch_kv4_attn(const LaunchArgs& a, const Kv4Args& c, hipStream_t st);
size_t kv4_attn_lds_bytes(int head_dim, int batch, int waves);
// Waves of a CU: 12 leave a wave 168 registers, 8 (D = 256) 256.
constexpr int kv4_max_waves(int head_dim) { return head_dim == 256 ? 8 : 12; }

}  // namespace pda
