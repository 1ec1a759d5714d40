// The experts' products of a mixture-of-experts layer for a few tokens, for
// MI355X (gfx950, CDNA4, wave64):
//   out_t = residual_t + sum_j w_tj D_e (act(G_e x_t) * (U_e x_t)),  e = ids_tj.
//
// A token's choice of an expert is a pair.  A segment is up to 16 BT pairs of
// one expert, the columns of its matrix products; the first kernel takes each
// segment through a few row tiles of gate and up weights, the second through
// row tiles of the down weights, and a third adds a token's pairs in order.
#include "pda_ffn.h"

#include <atomic>
#include <type_traits>

#include "pda_device.h"
#include "pda_gemv.h"

namespace pda {
namespace {

// Weights in the packed order of rows_kernel (16 rows x 32 k, 1 KB, straight
// into matrix-core registers), activations through a ring of two steps of
// every wave in LDS, and the W waves dealing the 64-k steps among themselves,
// as there; the rows that a column reads are found by its pair.
enum class Stage { kGateUp, kDown };

constexpr int kMoeWaves = 8;
constexpr int kMoeSlots = 2;  // steps in a wave's ring, and steps per block of weights
__host__ __device__ constexpr int moe_ring_bytes(int bt) { return kMoeWaves * kMoeSlots * bt * 2048; }
__host__ __device__ constexpr int moe_sum_bytes(int rt, int bt) { return kMoeWaves * rt * bt * 1024; }
// ids and counts, before the ring is used
__host__ __device__ constexpr int moe_scratch_bytes() { return (kMaxMoePairs + kMaxExperts) * 4; }
__host__ __device__ constexpr int moe_lds_bytes(int rt, int bt) {
  int n = moe_ring_bytes(bt);
  n = moe_sum_bytes(rt, bt) > n ? moe_sum_bytes(rt, bt) : n;
  return moe_scratch_bytes() > n ? moe_scratch_bytes() : n;
}

// The expert of segment `seg` and its columns' pairs, -1 past the last; false
// if there are fewer segments.  Segments go by expert, then by pair.  Every
// workgroup works this out for itself from the ids.
template <int kCols>
__device__ bool find_segment(const ExpertsArgs& a, int seg, unsigned char* lds, int* found, int* cols) {
  const int pairs = a.tokens * a.top_k;
  int* ids = reinterpret_cast<int*>(lds);
  int* count = ids + kMaxMoePairs;
  const int tid = threadIdx.x;
  for (int e = tid; e < a.experts; e += kMoeWaves * 64) count[e] = 0;
  if (tid == 0) found[0] = -1;
  __syncthreads();
  for (int p = tid; p < pairs; p += kMoeWaves * 64) {
    const int id = a.ids[p];
    ids[p] = id;
    if (id >= 0 && id < a.experts) atomicAdd(&count[id], 1);
  }
  if (tid < kCols) cols[tid] = -1;
  __syncthreads();
  if (tid < 64) {
    // lane l counts the segments of its share of the experts
    const int share = (a.experts + 63) / 64;
    const int e0 = tid * share, e1 = e0 + share < a.experts ? e0 + share : a.experts;
    int n = 0;
    for (int e = e0; e < e1; ++e) n += (count[e] + kCols - 1) / kCols;
    int end = n;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int other = __shfl_up(end, off);
      if (tid >= off) end += other;
    }
    int at = end - n;
    if (seg >= at && seg < end) {
      for (int e = e0; e < e1; ++e) {
        const int k = (count[e] + kCols - 1) / kCols;
        if (seg >= at && seg < at + k) {
          found[0] = e;
          found[1] = (seg - at) * kCols;
        }
        at += k;
      }
    }
  }
  __syncthreads();
  const int expert = uniform(found[0]);
  if (expert < 0) return false;
  if (tid < 64) {
    const int first = uniform(found[1]);
    int seen = 0;
    for (int p0 = 0; p0 < pairs; p0 += 64) {
      const bool is = p0 + tid < pairs && ids[p0 + tid] == expert;
      const uint64_t m = __ballot(is);
      const int rank = seen + __popcll(m & ((uint64_t{1} << tid) - 1)) - first;
      if (is && rank >= 0 && rank < kCols) cols[rank] = p0 + tid;
      seen += __popcll(m);
    }
  }
  __syncthreads();
  return true;
}

template <Stage kStage, int RT, int BT>
__global__ __launch_bounds__(kMoeWaves * 64, RT * BT <= 4 ? 4 : 2) void experts_kernel(ExpertsArgs a, int row_groups) {
  constexpr bool kUp = kStage == Stage::kGateUp;
  constexpr int W = kMoeWaves, DX = kMoeSlots, KB = kMoeSlots;
  constexpr int kSlot = BT * 2048, kLx = 2 * BT, kLw = 2 * RT;
  constexpr uint32_t kOutside = 0x80000000u;  // past any descriptor: reads zero
  static_assert(!kUp || RT % 2 == 0, "gate and up tiles go in pairs");
  extern __shared__ __align__(1024) unsigned char lds[];
  __shared__ int found[2];
  __shared__ int cols[16 * BT];

  const int seg = static_cast<int>(blockIdx.x) / row_groups;
  const int rg = static_cast<int>(blockIdx.x) - seg * row_groups;
  if (!find_segment<16 * BT>(a, seg, lds, found, cols)) return;
  const int64_t expert = uniform(found[0]);

  const int lane = threadIdx.x & 63;
  const int wv = uniform(threadIdx.x >> 6);
  const int col = lane & 15, kblk = lane >> 4;
  const int k = kUp ? a.hidden : a.inter;
  const int n = kUp ? 2 * a.inter : a.hidden;
  const int kt_count = k / kTileK, tiles = n / kTileRows;

  // activations: the row of a column is its token's (kUp) or its pair's
  const int pairs = a.tokens * a.top_k;
  const __amdgpu_buffer_rsrc_t rx =
      make_rsrc(kUp ? a.x : a.h, static_cast<uint32_t>(kUp ? a.tokens : pairs) * static_cast<uint32_t>(k) * 2u);
  const int xpiece = (lane & 7) ^ (lane >> 3);
  uint32_t xrow[kLx];
#pragma unroll
  for (int i = 0; i < kLx; ++i) {
    const int p = cols[8 * i + (lane >> 3)];
    const uint32_t row = static_cast<uint32_t>(kUp ? p / a.top_k : p);
    xrow[i] = p < 0 ? kOutside : row * static_cast<uint32_t>(k) * 2u + xpiece * 16u;
  }
  __syncthreads();  // the ring takes the place of the ids
  unsigned char* ring = lds + wv * (DX * kSlot);

  const uint16_t* w = kUp ? a.w_gate_up : a.w_down;
  __amdgpu_buffer_rsrc_t rw[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    int t = rg * RT + r;
    if constexpr (kUp) {
      const int p = t >> 1;
      t = p < tiles >> 1 ? p + (r & 1) * (tiles >> 1) : tiles;
    }
    t = uniform(t);
    rw[r] = make_rsrc(w + (expert * tiles + (t < tiles ? t : 0)) * kt_count * (kTileRows * kTileK),
                      t < tiles ? kt_count * 1024u : 0u);
  }
  const int steps = ((kt_count + 1) / 2 + W - 1) / W;

  auto issue_x = [&](int slot, int s) __attribute__((always_inline)) {
    const int k0 = (wv + s * W) * kPairK;
    const bool in = k0 + 8 * xpiece < k;
#pragma unroll
    for (int i = 0; i < kLx; ++i) {
      const uint32_t off = in && xrow[i] != kOutside ? xrow[i] + k0 * 2u : kOutside;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rx, (__attribute__((address_space(3))) void*)(ring + slot * kSlot + i * 1024), 16, off, 0, 0, 0);
    }
  };
  u32x4 wa[2][KB][RT][2];
  auto issue_w = [&](int buf, int blk) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < KB; ++i) {
      const int kt = 2 * (wv + (blk * KB + i) * W);
      uint32_t at[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) at[j] = kt + j < kt_count ? static_cast<uint32_t>(kt + j) * 1024u + lane * 16u : kOutside;
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int m = 0; m < 2; ++m)
          wa[buf][i][r][m] = __builtin_amdgcn_raw_buffer_load_b128(rw[r], at[m], 0, kCachePolicyNT);
    }
  };
  f32x4 acc[RT][BT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < BT; ++c) acc[r][c] = f32x4{};
  const int frag0 = (col >> 3) * 1024 + (col & 7) * 128 + ((kblk ^ (col & 7)) * 16);
  u32x4 xb[BT][2];

  issue_w(0, 0);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int s = 0; s < DX; ++s) issue_x(s, s);
  __builtin_amdgcn_sched_barrier(0);

  auto block = [&](int buf, int blk, auto last) __attribute__((always_inline)) {
    constexpr bool kLast = decltype(last)::value;
    if constexpr (!kLast) {
      issue_w(buf ^ 1, blk + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      if constexpr (kLast) {
        if (j == 0) __builtin_amdgcn_s_waitcnt(kWaitLoads);
      } else {
        // younger than the step's activations: the other step's, and this block's request for weights
        constexpr int kYounger = (DX - 1) * kLx + KB * kLw;
        static_assert(kYounger < 64, "vmcnt holds at most 63");
        __builtin_amdgcn_s_waitcnt(wait_loads(kYounger));
      }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int c = 0; c < BT; ++c)
#pragma unroll
        for (int m = 0; m < 2; ++m)
          xb[c][m] = *reinterpret_cast<const u32x4*>(ring + j * kSlot + c * 2048 + (frag0 ^ (m * 64)));
      if constexpr (!kLast) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the slot's operands are in registers
        asm volatile("" ::: "memory");
        issue_x(j, blk * KB + j + DX);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int c = 0; c < BT; ++c)
#pragma unroll
          for (int r = 0; r < RT; ++r)
            acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wa[buf][j][r][m]),
                                                                __builtin_bit_cast(bf16x8, xb[c][m]), acc[r][c], 0, 0, 0);
    }
  };
  const int blocks = (steps + KB - 1) / KB;
  int blk = 0;
  for (; blk + 2 < blocks; blk += 2) {
    block(0, blk, std::false_type{});
    block(1, blk + 1, std::false_type{});
  }
  if (blk + 1 < blocks) {
    block(0, blk, std::false_type{});
    block(1, blk + 1, std::true_type{});
  } else {
    block(0, blk, std::true_type{});
  }

  // ---- the waves' sums meet in LDS
  __builtin_amdgcn_s_waitcnt(kWaitLoads);
  __syncthreads();
  f32x4* red = reinterpret_cast<f32x4*>(lds);  // [W][RT][BT][64 lanes]
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < BT; ++c) red[((wv * RT + r) * BT + c) * 64 + lane] = acc[r][c];
  __syncthreads();
  auto total = [&](int r, int c) __attribute__((always_inline)) {
    f32x4 v = red[(r * BT + c) * 64 + lane];
#pragma unroll
    for (int i = 1; i < W; ++i) v += red[((i * RT + r) * BT + c) * 64 + lane];
    return v;
  };
  constexpr int kItems = (kUp ? RT / 2 : RT) * BT;
  for (int it = wv; it < kItems; it += W) {
    const int r = it / BT, c = it % BT;
    const int p = cols[16 * c + col];
    if constexpr (kUp) {
      const f32x4 g = total(2 * r, c), u = total(2 * r + 1, c);
      const int f = 16 * (rg * (RT / 2) + r) + 4 * kblk;
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = activate(g[j], a.activation) * u[j];
      if (p >= 0 && f < a.inter) store_bf16<4>(a.h + static_cast<int64_t>(p) * a.inter + f, v);
    } else {
      const f32x4 v = total(r, c);
      const int o = 16 * (rg * RT + r) + 4 * kblk;
      if (p >= 0 && o < a.hidden) *reinterpret_cast<f32x4*>(a.y + static_cast<int64_t>(p) * a.hidden + o) = v;
    }
  }
}

// A token's pairs in order, weighted, and the residual: four features a thread.
__global__ __launch_bounds__(256) void combine_kernel(ExpertsArgs a) {
  const int per = a.hidden / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= static_cast<int64_t>(a.tokens) * per) return;
  const int t = static_cast<int>(i / per);
  const int n = 4 * static_cast<int>(i - static_cast<int64_t>(t) * per);
  const int64_t o = static_cast<int64_t>(t) * a.hidden + n;
  uint32_t res[2] = {0u, 0u};
  if (a.residual) load_bf16<4>(a.residual + o, res);
  float v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = unpack_bf16(res, j);
  for (int j = 0; j < a.top_k; ++j) {
    const int p = t * a.top_k + j;
    const int id = a.ids[p];
    if (id < 0 || id >= a.experts) continue;
    const float w = a.weights[p];
    const f32x4 y = *reinterpret_cast<const f32x4*>(a.y + static_cast<int64_t>(p) * a.hidden + n);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += w * y[q];
  }
  store_bf16<4>(a.out + o, v);
}

template <Stage kStage, int RT, int BT>
hipError_t experts_as(const ExpertsArgs& a, hipStream_t st) {
  constexpr int lds = moe_lds_bytes(RT, BT);
  auto* fn = &experts_kernel<kStage, RT, BT>;
  if constexpr (lds > 64 * 1024) {
    // the dynamic-LDS limit is raised once per device (bit = device ordinal)
    static std::atomic<uint64_t> attr_set{0};
    int dev = 0;
    hipError_t err = hipGetDevice(&dev);
    if (err != hipSuccess) return err;
    const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
    if (!bit || !(attr_set.load() & bit)) {
      err = hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
      if (err != hipSuccess) return err;
      attr_set.fetch_or(bit);
    }
  }
  const int pairs = a.tokens * a.top_k;
  const int most = a.experts < pairs ? a.experts : pairs;  // experts that any pair may ask for
  constexpr int kCols = 16 * BT;
  const int segs = (pairs + most * (kCols - 1)) / kCols;
  const int tiles = (kStage == Stage::kGateUp ? 2 * a.inter : a.hidden) / kTileRows;
  const int row_groups = (tiles + RT - 1) / RT;
  hipLaunchKernelGGL(fn, dim3(static_cast<unsigned>(segs) * row_groups), dim3(kMoeWaves * 64), lds, st, a, row_groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_experts(const ExpertsArgs& a, int num_cus, hipStream_t st) {
  (void)num_cus;
  hipError_t e;
  if (a.tokens <= 16) {
    if ((e = experts_as<Stage::kGateUp, 2, 1>(a, st)) != hipSuccess) return e;
    if ((e = experts_as<Stage::kDown, 2, 1>(a, st)) != hipSuccess) return e;
  } else {
    if ((e = experts_as<Stage::kGateUp, 2, 4>(a, st)) != hipSuccess) return e;
    if ((e = experts_as<Stage::kDown, 2, 4>(a, st)) != hipSuccess) return e;
  }
  const int64_t threads = static_cast<int64_t>(a.tokens) * (a.hidden / 4);
  hipLaunchKernelGGL(combine_kernel, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace pda
