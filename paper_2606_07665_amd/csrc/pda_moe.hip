// The experts' products of a mixture-of-experts layer for a few tokens, for
// MI355X (gfx950, CDNA4, wave64):
//   out_t = residual_t + sum_j w_tj D_e (act(G_e x_t) * (U_e x_t)),  e = ids_tj.
//
// A token's choice of an expert is a pair.  A segment is up to 16 BT pairs of
// one expert, the columns of its matrix products.  The first kernel takes each
// segment through the gate and up weights; then one kernel adds up the down
// products of a token's few pairs, or one takes each segment through the down
// weights and another adds a token's pairs.
#include "pda_ffn.h"

#include <type_traits>

#include "pda_device.h"
#include "pda_gemv.h"

namespace pda {
namespace {

enum class Stage { kGateUp, kDown };

constexpr uint32_t kOutside = 0x80000000u;  // past any descriptor: reads zero

// The segment search's ids, counts and list of pairs in LDS.
constexpr int kScratchBytes = (kMaxMoePairs + kMaxExperts + 2 + 128) * 4;

// The expert of segment `seg`, or -1 if there are fewer segments, and the pairs
// of its columns: lane l of every wave holds that of column l + 64 i, -1 past
// the last.  Every workgroup works this out for itself from the ids.
//
// Up to 64 pairs: segments go by first pair, in registers.  A wave holds the
// ids, one a lane, and takes one expert after the other out of the mask of
// pairs that are left; nothing goes through LDS.
template <int kCols>
__device__ __forceinline__ int find_segment_of_few(const ExpertsArgs& a, int seg, int (&cols)[(kCols + 63) / 64]) {
  const int pairs = a.tokens * a.top_k, lane = threadIdx.x & 63;
  int id = lane < pairs ? a.ids[lane] : -1;
  if (id < 0 || id >= a.experts) id = -1;
  uint64_t left = __ballot(id >= 0);
  int at = 0;  // segments before
  while (left) {
    const int expert = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
    const uint64_t same = __ballot(id == expert);
    const int n = (__popcll(same) + kCols - 1) / kCols;
    if (seg < at + n) {
      const int rank = __popcll(same & ((uint64_t{1} << lane) - 1)) - (seg - at) * kCols;
      const int count = __popcll(same) - (seg - at) * kCols;
      // each pair's lane sends its number to the column's; the others to lanes past them, never read
      const bool sent = id == expert && rank >= 0 && rank < kCols;
      const int got = kCols < 64 ? __builtin_amdgcn_ds_permute(4 * (sent ? rank : 63), lane)
                                 : __builtin_amdgcn_ds_permute(4 * (sent ? rank : 63 - __popcll(~same & ((uint64_t{1} << lane) - 1))), lane);
#pragma unroll
      for (int i = 0; i < (kCols + 63) / 64; ++i) cols[i] = -1;
      cols[0] = lane < kCols && lane < count ? got : -1;
      return expert;
    }
    at += n;
    left &= ~same;
  }
  return -1;
}

// More: segments go by expert, then by pair, from counts in LDS (the start of
// `lds`, free again when every wave has passed the next barrier).
template <int kCols, int W>
__device__ __forceinline__ int find_segment_of_many(const ExpertsArgs& a, int seg, unsigned char* lds,
                                                    int (&cols)[(kCols + 63) / 64]) {
  const int pairs = a.tokens * a.top_k;
  int* ids = reinterpret_cast<int*>(lds);
  int* count = ids + kMaxMoePairs;
  int* found = count + kMaxExperts;
  int* list = found + 2;
  const int tid = threadIdx.x;
  for (int e = tid; e < a.experts; e += W * 64) count[e] = 0;
  if (tid == 0) found[0] = -1;
  if (tid < kCols) list[tid] = -1;
  __syncthreads();
  for (int p = tid; p < pairs; p += W * 64) {
    const int id = a.ids[p];
    ids[p] = id;
    if (id >= 0 && id < a.experts) atomicAdd(&count[id], 1);
  }
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
  if (expert < 0) return -1;
  if (tid < 64) {
    const int first = uniform(found[1]);
    int seen = 0;
    for (int p0 = 0; p0 < pairs; p0 += 64) {
      const bool is = p0 + tid < pairs && ids[p0 + tid] == expert;
      const uint64_t m = __ballot(is);
      const int rank = seen + __popcll(m & ((uint64_t{1} << tid) - 1)) - first;
      if (is && rank >= 0 && rank < kCols) list[rank] = p0 + tid;
      seen += __popcll(m);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < (kCols + 63) / 64; ++i) cols[i] = (tid & 63) + 64 * i < kCols ? list[(tid & 63) + 64 * i] : -1;
  return expert;
}

template <int kCols, int W>
__device__ __forceinline__ int find_segment(const ExpertsArgs& a, int seg, unsigned char* lds, int (&cols)[(kCols + 63) / 64]) {
  if (a.tokens * a.top_k <= 64) return find_segment_of_few<kCols>(a, seg, cols);
  return find_segment_of_many<kCols, W>(a, seg, lds, cols);
}

// The pair of column c (the same for every lane, or not).
template <int N>
__device__ __forceinline__ int column(const int (&cols)[N], int c) {
  int p = __shfl(cols[0], c & 63);
#pragma unroll
  for (int i = 1; i < N; ++i) {
    const int q = __shfl(cols[i], c & 63);
    p = c >= 64 * i ? q : p;
  }
  return p;
}

// Weights in the packed order of rows_kernel (16 rows x 32 k, 1 KB, straight
// into matrix-core registers).  A wave takes two row tiles (a gate and up pair,
// or two of the down rows) over the whole k range, or with kSplit the waves of
// a workgroup deal the steps (64 k) of the same two among themselves and add
// their sums in LDS.  The workgroup's activations, gathered by the columns'
// pairs, lie in LDS once for all its waves, kChunkBytes of the k range at a
// time.  Each wave keeps D steps of weights in flight in registers, also while
// a chunk arrives.  The down products' k range may be cut into a.splits parts,
// whose sums the combination adds.
//
// What bounds it is the weights' way from memory, each of them once for up to
// 128 tokens of an expert.  A wave of its own row tiles reads without a pause
// from start to end; the form with the k range dealt over 8 waves and a ring of
// activations for each, which this replaces, spent 2 us of every workgroup's 5
// on its ramp and read the activations again for every 32 rows.  Measured
// (128 experts of 768 x 2048, 8 a token; 64 of 1408, 6 a token; 8 of 14336 x
// 4096, 2 a token), gate and up, then down, us, before -> now: 16 tokens 87 ->
// 74, 63 -> 38 (6.4 and 6.2 TB/s); 58 tokens 211 -> 129, 126 -> 68; 200 tokens
// 682 -> 412, 308 -> 236.
//
// BT = 8 column tiles were as fast as 1 and 4 for few columns (a segment's
// products are compiled for each number of tiles in use) and read an expert of
// more than 64 tokens once: 200 tokens 412 us, with BT = 4 485.  Two workgroups
// of 4 waves a CU beat one of 8 with two chunks in LDS (412 and 404 us there,
// but 35.5 and 41 where 16 experts have 64 tokens); 4 row tiles a wave were no
// faster.
constexpr int kMoeWaves = 4;

template <Stage kStage, int BT, int D, bool kSplit, int kChunkBytes, int kWavesPerSimd>
__global__ __launch_bounds__(kMoeWaves * 64, kWavesPerSimd) void experts_kernel(ExpertsArgs a, int row_groups) {
  constexpr bool kUp = kStage == Stage::kGateUp;
  constexpr int W = kMoeWaves, RT = 2;
  static_assert(kChunkBytes >= kScratchBytes, "the ids fit in a chunk");
  extern __shared__ __align__(1024) unsigned char lds[];

  // part `sp` of the steps (kDown), row group rg of segment seg
  const int sp = kUp ? 0 : static_cast<int>(blockIdx.y);
  const int seg = static_cast<int>(blockIdx.x) / row_groups;
  const int rg = static_cast<int>(blockIdx.x) - seg * row_groups;
  int cols[(16 * BT + 63) / 64];
  const int64_t expert = uniform(find_segment<16 * BT, W>(a, seg, lds, cols));
  if (expert < 0) return;

  const int lane = threadIdx.x & 63;
  const int wv = uniform(threadIdx.x >> 6);
  const int col = lane & 15, kblk = lane >> 4;
  const int k = kUp ? a.hidden : a.inter;
  const int n = kUp ? 2 * a.inter : a.hidden;
  const int kt_count = k / kTileK, tiles = n / kTileRows;
  const int all_steps = (kt_count + 1) / 2;
  const int begin = kUp ? 0 : sp * all_steps / a.splits;
  const int steps = (kUp ? all_steps : (sp + 1) * all_steps / a.splits) - begin;  // of this part
  const int group = kSplit ? rg : rg * W + wv;  // the wave's row tiles, RT * group on
  // the wave's steps of the part: the q-th is q * kStride + first
  constexpr int kStride = kSplit ? W : 1;
  const int first = kSplit ? wv : 0;
  const int count = steps > first ? (steps - first + kStride - 1) / kStride : 0;

  // weights first: the loads are in flight while the activations come
  const uint16_t* w = kUp ? a.w_gate_up : a.w_down;
  __amdgpu_buffer_rsrc_t rw[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    int t = group * RT + r;
    if constexpr (kUp) {
      const int p = t >> 1;
      t = p < tiles >> 1 ? p + (r & 1) * (tiles >> 1) : tiles;
    }
    t = uniform(t);
    rw[r] = make_rsrc(w + (expert * tiles + (t < tiles ? t : 0)) * kt_count * (kTileRows * kTileK),
                      t < tiles ? kt_count * 1024u : 0u);
  }
  u32x4 wa[D][RT][2];
  auto issue_w = [&](int slot, int q) __attribute__((always_inline)) {
    // (k tiles past the end lie outside; so do those of the next part)
    const int s = q * kStride + first;
    const uint32_t at = s < steps ? static_cast<uint32_t>(begin + s) * 2048u + lane * 16u : kOutside;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int m = 0; m < 2; ++m)
        wa[slot][r][m] = __builtin_amdgcn_raw_buffer_load_b128(rw[r], at + m * 1024u, 0, kCachePolicyNT);
  };
#pragma unroll
  for (int j = 0; j < D; ++j) issue_w(j, j);
  __builtin_amdgcn_sched_barrier(0);

  const int pairs = a.tokens * a.top_k;
  const __amdgpu_buffer_rsrc_t rx =
      make_rsrc(kUp ? a.x : a.h, static_cast<uint32_t>(kUp ? a.tokens : pairs) * static_cast<uint32_t>(k) * 2u);
  // activations go into LDS 8 rows x 128 bytes a wave load, lane l fetching
  // the 16-byte piece (l % 8) ^ (l / 8) of row l / 8: operand reads without
  // bank conflicts
  const int xpiece = (lane & 7) ^ (lane >> 3);
  uint32_t xrow[2 * BT];
#pragma unroll
  for (int i = 0; i < 2 * BT; ++i) {
    const int p = column(cols, 8 * i + (lane >> 3));
    const uint32_t row = static_cast<uint32_t>(kUp ? p / a.top_k : p);
    xrow[i] = p < 0 ? kOutside : row * static_cast<uint32_t>(k) * 2u + xpiece * 16u;
  }
  const int frag0 = (col >> 3) * 1024 + (col & 7) * 128 + ((kblk ^ (col & 7)) * 16);

  // groups of 8 columns in use: pairs come first
  int used8 = 1;
#pragma unroll
  for (int c = 1; c < 2 * BT; ++c) used8 += uniform(column(cols, 8 * c)) >= 0 ? 1 : 0;

  // NT column tiles are in use
  auto products = [&](auto nt) __attribute__((always_inline)) {
    constexpr int NT = decltype(nt)::value;
    constexpr int kSlot = NT * 2048;                                 // a step's activations
    constexpr int kQ = kChunkBytes / kSlot / (kStride * D) * D;      // steps of a wave in a chunk
    static_assert(kQ >= D, "a chunk holds every step in flight");
    f32x4 acc[RT][NT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int c = 0; c < NT; ++c) acc[r][c] = f32x4{};
    // the chunk from the waves' step q0 on
    auto issue_chunk = [&](int q0) __attribute__((always_inline)) {
      const int s0 = q0 * kStride;
      const int s1 = s0 + kQ * kStride < steps ? s0 + kQ * kStride : steps;
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i) {
        // (columns without a pair keep what the LDS holds: nobody reads their sums)
        if (i >= used8) break;
        for (int s = s0 + wv; s < s1; s += W) {
          const uint32_t k0 = static_cast<uint32_t>(begin + s) * kPairK;
          const uint32_t off = static_cast<int>(k0) + 8 * xpiece < k && xrow[i] != kOutside ? xrow[i] + k0 * 2u : kOutside;
          __builtin_amdgcn_raw_ptr_buffer_load_lds(
              rx, (__attribute__((address_space(3))) void*)(lds + (s - s0) * kSlot + i * 1024), 16, off, 0, 0, 0);
        }
      }
    };
    __syncthreads();  // the ids are done with
    // a step's products: the weights of slot j, the activations at `at`
    auto multiply = [&](int j, const unsigned char* at) __attribute__((always_inline)) {
      u32x4 xb[NT][2];
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int m = 0; m < 2; ++m) xb[c][m] = *reinterpret_cast<const u32x4*>(at + c * 2048 + (frag0 ^ (m * 64)));
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int r = 0; r < RT; ++r)
            acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wa[j][r][m]),
                                                                __builtin_bit_cast(bf16x8, xb[c][m]), acc[r][c], 0, 0, 0);
    };
    if constexpr (!kSplit && NT >= 3) {
      // a whole chunk of many columns is only a few steps, and no weights are in
      // flight behind it when it has come: two steps at a time in two places, the next
      // ones on their way, in whole rounds without a branch (what lies past the end is
      // zeros).  us: 80 tokens of 5 over 8 experts of 1056 (3584 features) 68.1 -> 64.5,
      // 128 of 2 over 8 of 14336 (4096) 575.7 -> 561.1, fewer columns level.
      static_assert(D == 4 && W == 4 && 4 * kSlot <= kChunkBytes, "two places of two steps");
      uint32_t xgroup[NT];  // the wave's share: half of the groups of one of two steps
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int p = column(cols, 8 * ((wv >> 1) * NT + i) + (lane >> 3));
        const uint32_t row = static_cast<uint32_t>(kUp ? p / a.top_k : p);
        xgroup[i] = p < 0 ? kOutside : row * static_cast<uint32_t>(k) * 2u + xpiece * 16u;
      }
      auto issue_two = [&](int q0, int place) __attribute__((always_inline)) {
        const int s = q0 + (wv & 1);
        const uint32_t k0 = static_cast<uint32_t>(begin + s) * kPairK;
        const bool in = s < steps && static_cast<int>(k0) + 8 * xpiece < k;
        unsigned char* to = lds + (2 * place + (wv & 1)) * kSlot + (wv >> 1) * (NT * 1024);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const uint32_t off = in && xgroup[i] != kOutside ? xgroup[i] + k0 * 2u : kOutside;
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void*)(to + i * 1024), 16, off, 0, 0, 0);
        }
      };
      issue_two(0, 0);
      __builtin_amdgcn_s_waitcnt(kWaitLoads);
      __syncthreads();
      for (int q1 = 0; q1 < steps; q1 += D) {
#pragma unroll
        for (int ph = 0; ph < 2; ++ph) {
          issue_two(q1 + 2 * ph + 2, ph ^ 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int q = 2 * ph; q < 2 * ph + 2; ++q) {
            multiply(q, lds + q * kSlot);
            issue_w(q, q1 + q + D);
            __builtin_amdgcn_sched_barrier(0);
          }
          asm volatile("" ::: "memory");
          __builtin_amdgcn_s_waitcnt(wait_loads(4 * RT));  // all but the weights after the activations
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
        }
      }
    } else {
      issue_chunk(0);
      __builtin_amdgcn_s_waitcnt(kWaitLoads);
      __syncthreads();
      const int all = (steps + kStride - 1) / kStride;  // the most steps of a wave
      for (int q0 = 0; q0 < all; q0 += kQ) {
        const int end = q0 + kQ < count ? q0 + kQ : count;
        const unsigned char* from = lds + first * kSlot;
        auto step = [&](int j, int q) __attribute__((always_inline)) { multiply(j, from + (q - q0) * (kStride * kSlot)); };
        // whole rounds without a branch, so that the waits count the loads of
        // every step in flight; then the last steps
        int q = q0;
        for (; q + D <= end; q += D) {
#pragma unroll
          for (int j = 0; j < D; ++j) {
            step(j, q + j);
            issue_w(j, q + j + D);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
#pragma unroll
        for (int j = 0; j < D; ++j)
          if (q + j < end) step(j, q + j);
        if (q0 + kQ >= all) break;
        __syncthreads();
        issue_chunk(q0 + kQ);
        __builtin_amdgcn_s_waitcnt(kWaitLoads);
        __syncthreads();
      }
    }

    // A column's pair and the four rows 4 kblk .. of row tile (or pair) r.
    // h is rounded to bf16, the operand of the next product's matrix instructions
    // (its halves in two would double the activations' way through LDS and the
    // products).  The output is the fp64 one of these rounded h, rounded once, at 99 to
    // 100% of all places; against one without the rounding its root mean square error
    // is 1.41 times that of the last rounding alone, with a residual 1.09 to 1.23
    // times (1, 16 and 61 tokens of 6 to 8 experts, 200 of 2).
    auto emit = [&](int r, int p, f32x4 v, f32x4 up) __attribute__((always_inline)) {
      if (p < 0) return;
      if constexpr (kUp) {
        const float scale = a.weighted_h ? a.weights[p] : 1.f;
        const int f = 16 * (group * (RT / 2) + r) + 4 * kblk;
        float h[4] = {v[0], v[1], v[2], v[3]};
        activate(h, a.activation);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[j] = scale * h[j] * up[j];
        if (f < a.inter) store_bf16<4>(a.h + static_cast<int64_t>(p) * a.inter + f, h);
      } else {
        const int o = 16 * (group * RT + r) + 4 * kblk;
        if (o < a.hidden) *reinterpret_cast<f32x4*>(a.y + (static_cast<int64_t>(sp) * pairs + p) * a.hidden + o) = v;
      }
    };
    int of[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) of[c] = column(cols, 16 * c + col);
    constexpr int kR = kUp ? RT / 2 : RT;
    if constexpr (kSplit) {
      static_assert(W * RT * NT * 1024 <= kChunkBytes, "the waves' sums fit in a chunk");
      f32x4* red = reinterpret_cast<f32x4*>(lds);  // [W][RT][NT][64 lanes]
      __syncthreads();
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < NT; ++c) red[((wv * RT + r) * NT + c) * 64 + lane] = acc[r][c];
      __syncthreads();
      auto total = [&](int r, int c) __attribute__((always_inline)) {
        f32x4 v = red[(r * NT + c) * 64 + lane];
#pragma unroll
        for (int i = 1; i < W; ++i) v += red[((i * RT + r) * NT + c) * 64 + lane];
        return v;
      };
#pragma unroll
      for (int r = 0; r < kR; ++r)
#pragma unroll
        for (int c = 0; c < NT; ++c)
          if ((r * NT + c) % W == wv) {
            if constexpr (kUp)
              emit(r, of[c], total(2 * r, c), total(2 * r + 1, c));
            else
              emit(r, of[c], total(r, c), f32x4{});
          }
    } else {
#pragma unroll
      for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int r = 0; r < kR; ++r) {
          if constexpr (kUp)
            emit(r, of[c], acc[2 * r][c], acc[2 * r + 1][c]);
          else
            emit(r, of[c], acc[r][c], f32x4{});
        }
    }
  };
  const int used = (used8 + 1) / 2;
  if constexpr (BT >= 8) {
    if (used == 8) return products(std::integral_constant<int, 8>{});
    if (used == 7) return products(std::integral_constant<int, 7>{});
    if (used == 6) return products(std::integral_constant<int, 6>{});
    if (used == 5) return products(std::integral_constant<int, 5>{});
  }
  if constexpr (BT >= 4) {
    if (used == 4) return products(std::integral_constant<int, 4>{});
    if (used == 3) return products(std::integral_constant<int, 3>{});
  }
  if constexpr (BT >= 2) {
    if (used == 2) return products(std::integral_constant<int, 2>{});
  }
  products(std::integral_constant<int, 1>{});
}

// The second product of few pairs (up to 64, of up to 8 tokens), whole in one
// kernel: h carries the pair's weight, the columns are the tokens, and a
// workgroup adds up every expert's part of 8 rows, which the waves deal among
// themselves by their (expert, 64 k) steps, a run of them each.  A token that
// has not chosen an expert reads zeros in its steps (outside the descriptor, no
// traffic), and takes nothing from their sums: zeros times a weight that is not
// finite are none.  The sums' order follows from the slots of the whole batch, so
// that a token's last bits may depend on the others' choices; the same ids give
// the same bits.
//
// A matrix instruction multiplies both k tiles of a step at once: rows 0-7 of
// its operand and columns 0-7 of the other hold the first, rows and columns
// 8-15 the second; of its results the two blocks on the diagonal are the
// products, and their sum is the step's.  So 8 rows fill it, and twice as many
// workgroups share the weights than with 16: 2048 rows over 8 experts of 768
// 7.2 us, with 16 rows 9.2; 4 tokens 22.5 and 28.  The other form takes 8 us
// and its combination 4 more, 24.3 with 4 tokens, 40.2 here and there with 8.
template <int W, int D>
__global__ __launch_bounds__(W * 64, W / 4) void experts_join_kernel(ExpertsArgs a) {
  __shared__ f32x4 red[W][64];
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  const int col = lane & 15, kblk = lane >> 4;
  const int token = col & 7;
  const int pairs = a.tokens * a.top_k;
  int id = lane < pairs ? a.ids[lane] : -1;
  if (id < 0 || id >= a.experts) id = -1;
  const int kt_count = a.inter / kTileK, steps_each = (kt_count + 1) / 2;
  const int tile = static_cast<int>(blockIdx.x) >> 1, row8 = (static_cast<int>(blockIdx.x) & 1) * 8;  // rows 8 on or not
  const int tiles = a.hidden / kTileRows;
  const int token0 = (lane < pairs ? lane : 0) / a.top_k * a.top_k;  // the first pair of this lane's token
  // the token's own earlier pairs, and the pairs of the column's token
  const uint64_t before = ((uint64_t{1} << lane) - 1) & ~((uint64_t{1} << token0) - 1);
  const uint64_t of_col = token < a.tokens ? ((uint64_t{1} << a.top_k) - 1) << (token * a.top_k) : 0;

  // slots: an expert and one pair of each token that chose it (a second pair
  // of the same token and expert comes in a slot of its own)
  auto next_slot = [&](uint64_t& left, int& expert) -> uint64_t {
    expert = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
    const uint64_t same = __ballot(id == expert) & left;
    const uint64_t slot = __ballot(((same >> lane) & 1) && (same & before) == 0);
    left &= ~slot;
    return slot;
  };
  const uint64_t chosen_pairs = __ballot(id >= 0);
  int slots = 0;
  for (uint64_t left = chosen_pairs; left; ++slots) {
    int e;
    next_slot(left, e);
  }
  const int total = slots * steps_each;
  const int s0 = static_cast<int>(static_cast<int64_t>(total) * wv / W);
  const int s1 = static_cast<int>(static_cast<int64_t>(total) * (wv + 1) / W);

  const __amdgpu_buffer_rsrc_t rh = make_rsrc(a.h, static_cast<uint32_t>(pairs) * static_cast<uint32_t>(a.inter) * 2u);
  f32x4 acc = f32x4{}, sum = f32x4{};  // of the slot, of those before it
  // what the wave loads next: the slot's descriptor and row, the step of it
  uint64_t left = chosen_pairs;
  int at = s0, slot_end = 0;
  __amdgpu_buffer_rsrc_t rw = make_rsrc(a.w_down, 0u);
  uint32_t row = kOutside;
  const uint32_t wlane = kblk * 256u + (row8 + (col & 7)) * 16u;
  u32x4 wa[D], xb[D];
  auto issue = [&](int j) __attribute__((always_inline)) {
    while (at >= slot_end && left) {  // on to the slot of step `at`
      int e;
      const uint64_t slot = next_slot(left, e);
      slot_end += steps_each;
      if (at >= slot_end) continue;
      const uint64_t mine = slot & of_col;
      row = mine ? static_cast<uint32_t>(__builtin_ctzll(mine)) * static_cast<uint32_t>(a.inter) * 2u + kblk * 16u : kOutside;
      rw = make_rsrc(a.w_down + (static_cast<int64_t>(e) * tiles + tile) * kt_count * (kTileRows * kTileK), kt_count * 1024u);
    }
    const int kt = 2 * (at - (slot_end - steps_each)) + (col >> 3);
    const bool in = at < s1 && kt < kt_count;
    wa[j] = __builtin_amdgcn_raw_buffer_load_b128(rw, in ? kt * 1024u + wlane : kOutside, 0, kCachePolicyNT);
    xb[j] = __builtin_amdgcn_raw_buffer_load_b128(rh, in && row != kOutside ? row + kt * 64u : kOutside, 0, 0);
    ++at;
  };
#pragma unroll
  for (int j = 0; j < D; ++j) issue(j);
  __builtin_amdgcn_sched_barrier(0);
  // what it multiplies next
  uint64_t left_now = chosen_pairs;
  int end_now = 0;
  bool chosen = false;  // the column's token has chosen the slot's expert
  auto join = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] = chosen ? sum[q] + acc[q] : sum[q];
    acc = f32x4{};
  };
  for (int s = s0; s < s1; s += D) {
#pragma unroll
    for (int j = 0; j < D; ++j) {
      if (s + j >= end_now) {
        join();
        while (s + j >= end_now && left_now) {
          int e;
          chosen = (next_slot(left_now, e) & of_col) != 0;
          end_now += steps_each;
        }
      }
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wa[j]), __builtin_bit_cast(bf16x8, xb[j]), acc,
                                                    0, 0, 0);
      issue(j);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  join();
  red[wv][lane] = sum;
  __syncthreads();
  if (wv != 0) return;
  f32x4 all = red[0][lane];
#pragma unroll
  for (int i = 1; i < W; ++i) all += red[i][lane];
#pragma unroll
  for (int q = 0; q < 4; ++q) all[q] += __shfl_xor(all[q], 40);  // the other block: column + 8, rows + 8
  if (col >= 8 || kblk >= 2 || token >= a.tokens) return;
  const int64_t out = static_cast<int64_t>(token) * a.hidden + 16 * tile + row8 + 4 * kblk;
  float v[4] = {all[0], all[1], all[2], all[3]};
  if (a.residual) {
    uint32_t res[2];
    load_bf16<4>(a.residual + out, res);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += unpack_bf16(res, j);
  }
  store_bf16<4>(a.out + out, v);
}

// A token's pairs in order, each the sum of its parts, weighted, and the
// residual: four features a thread.  Four pairs are requested at a time, before
// their ids and weights are there (16 tokens of 8 pairs, 2048 features: 4.8 us
// pair by pair); one without an expert was written by nobody and is left out.
constexpr int kCombineThreads = 64;
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(ExpertsArgs a) {
  const int per = a.hidden / 4;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kCombineThreads + threadIdx.x;
  if (i >= static_cast<int64_t>(a.tokens) * per) return;
  const int t = static_cast<int>(i / per);
  const int n = 4 * static_cast<int>(i - static_cast<int64_t>(t) * per);
  const int64_t o = static_cast<int64_t>(t) * a.hidden + n;
  const int64_t part = static_cast<int64_t>(a.tokens) * a.top_k * a.hidden;
  uint32_t res[2] = {0u, 0u};
  if (a.residual) load_bf16<4>(a.residual + o, res);
  f32x4 v{};
  for (int j0 = 0; j0 < a.top_k; j0 += 4) {
    int id[4];
    float w[4];
    f32x4 y[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int p = t * a.top_k + (j0 + q < a.top_k ? j0 + q : a.top_k - 1);
      y[q] = *reinterpret_cast<const f32x4*>(a.y + static_cast<int64_t>(p) * a.hidden + n);
      id[q] = j0 + q < a.top_k ? a.ids[p] : -1;
      w[q] = a.weights[p];
    }
    for (int s = 1; s < a.splits; ++s) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int p = t * a.top_k + (j0 + q < a.top_k ? j0 + q : a.top_k - 1);
        y[q] += *reinterpret_cast<const f32x4*>(a.y + s * part + static_cast<int64_t>(p) * a.hidden + n);
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bool chosen = id[q] >= 0 && id[q] < a.experts;
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = chosen ? v[c] + w[q] * y[q][c] : v[c];
    }
  }
  float out[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) out[c] = a.residual ? v[c] + unpack_bf16(res, c) : v[c];
  store_bf16<4>(a.out + o, out);
}

template <Stage kStage, int BT, int D, bool kSplit, int kChunkBytes, int kWavesPerSimd>
hipError_t experts_as(const ExpertsArgs& a, hipStream_t st) {
  auto* fn = &experts_kernel<kStage, BT, D, kSplit, kChunkBytes, kWavesPerSimd>;
  static_assert(kChunkBytes <= 64 * 1024, "within the default limit of dynamic LDS");
  constexpr int kEach = 2 * (kSplit ? 1 : kMoeWaves);
  const int tiles = (kStage == Stage::kGateUp ? 2 * a.inter : a.hidden) / kTileRows;
  const int row_groups = (tiles + kEach - 1) / kEach;
  const dim3 grid(static_cast<unsigned>(moe_most_segments(a.tokens * a.top_k, a.experts, 16 * BT)) * row_groups,
                  kStage == Stage::kDown ? a.splits : 1);
  hipLaunchKernelGGL(fn, grid, dim3(kMoeWaves * 64), kChunkBytes, st, a, row_groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_experts(const ExpertsArgs& args, const ExpertsPlan& p, hipStream_t st) {
  ExpertsArgs a = args;
  a.weighted_h = p.joined;
  a.splits = p.splits;
  hipError_t e = p.shared_up ? experts_as<Stage::kGateUp, kMoeFewCols / 16, 2, true, 32 * 1024, 4>(a, st)
                             : experts_as<Stage::kGateUp, kMoeCols / 16, 4, false, 64 * 1024, 2>(a, st);
  if (e != hipSuccess) return e;
  if (p.joined) {
    constexpr int kJoinWaves = 8;
    hipLaunchKernelGGL((experts_join_kernel<kJoinWaves, 4>), dim3(static_cast<unsigned>(a.hidden / 8)), dim3(kJoinWaves * 64), 0,
                       st, a);
    return hipGetLastError();
  }
  e = p.shared_down ? experts_as<Stage::kDown, kMoeFewCols / 16, 2, true, 32 * 1024, 4>(a, st)
                    : experts_as<Stage::kDown, kMoeCols / 16, 4, false, 64 * 1024, 2>(a, st);
  if (e != hipSuccess) return e;
  const int64_t threads = static_cast<int64_t>(a.tokens) * (a.hidden / 4);
  hipLaunchKernelGGL(combine_kernel, dim3(static_cast<unsigned>((threads + kCombineThreads - 1) / kCombineThreads)),
                     dim3(kCombineThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace pda
