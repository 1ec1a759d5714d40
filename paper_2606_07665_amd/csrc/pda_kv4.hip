// The 4-bit KV cache on MI355X (gfx950): what writes it, what reads it back
// and the paged decode attention over it.
//
// Format (OCP microscaling FP4).  A token's key (or value) of one kv head is
// D / 32 groups of 32 elements.  A group has a byte s and 32 E2M1 codes (sign,
// two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) and stands
// for code * 2^(s - 127).  s = max(E - 2, 0) with E the largest biased bf16
// exponent in the group, so its largest element lies in [4, 8) units; codes
// are rounded to nearest, ties to even, and stop at 6.  (Taking the next unit
// wherever the largest element passes 6 would double the other elements'
// steps: more error over the group than the one clipped element saves.)  A
// group with an infinity or a NaN gets s = 255, which stands for NaN.
// gfx950 converts two codes and a scale to two bf16 values, and back, in one
// instruction at full rate, exactly as defined here for every scale (0 and
// 255 among them).
//
// Layout.  Codes [page, kv head, group, token slot, 16 bytes] and scales
// [page, kv head, group, token slot]: the 16 tokens x 128 elements that a
// wave multiplies at a time are then 64 consecutive 16-byte chunks in lane
// order, 1 KB, and their scales 64 consecutive bytes.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "pda_attn.h"
#include "pda_internal.h"
#include "pda_kv4.h"

namespace pda {
namespace {

__device__ __forceinline__ float scale_of(unsigned s) { return __builtin_bit_cast(float, s << 23); }

// Eight codes (the lowest four bits first) and their scale -> eight bf16.
__device__ __forceinline__ bf16x8 decode8(unsigned w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  const bf16x4 lo = __builtin_shufflevector(a, b, 0, 1, 2, 3), hi = __builtin_shufflevector(c, d, 0, 1, 2, 3);
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// ------------------------------------------------------------ append, read
// Eight lanes take two neighbouring groups of one token, 8 elements (16 bytes
// in bf16, 4 in codes) a lane, so that a token's 128 bytes of bf16 are one
// line.  kTile = 8: a wave takes the same two groups of the 8 tokens of an
// aligned run of slots, whose codes are then whole lines as well; kTile = 1:
// a wave takes 16 groups of one token, for calls whose runs would be mostly
// empty.  blockIdx.y: sequence; blockIdx.z: 0 keys, 1 values.
struct Kv4Lane {
  int t;          // position in the sequence
  int j;          // token of the call
  int g, grp;     // kv head, group
  unsigned page;  // its token's page; one outside the pool: none
  bool in;        // the call has this token
};

template <int D, int kTile>
__device__ __forceinline__ Kv4Lane kv4_lane(const Kv4Args& a) {
  constexpr int kGroups = D / kKv4Group;
  constexpr int kPairs = kGroups / 2;
  const unsigned u = (blockIdx.x * kKv4Threads + threadIdx.x) / 8;  // token and pair of groups
  const unsigned pairs = a.hkv * kPairs;
  const unsigned r = u / kTile;
  const unsigned run = r / pairs;
  const unsigned hp = r - run * pairs;
  const int b = blockIdx.y;
  const int L = clamp_len(a.lens[b], a.maxp << a.page_shift);
  const int start = L - a.tokens;  // position of the call's first token
  Kv4Lane p;
  p.t = kTile == 1 ? start + static_cast<int>(run) : (start & ~(kTile - 1)) + static_cast<int>(run * kTile + u % kTile);
  p.j = p.t - start;
  p.in = p.j >= 0 && p.j < a.tokens;
  p.g = hp / kPairs;
  p.grp = (hp % kPairs) * 2 + ((threadIdx.x & 7) >> 2);
  p.page = ~0u;
  if (p.in && p.t >= 0) p.page = static_cast<unsigned>(a.bt[static_cast<int64_t>(b) * a.maxp + (p.t >> a.page_shift)]);
  return p;
}

// Whether there is a page: an entry outside the pool (a page that was lacking, or
// was released) is none; clamped into the pool it would be another sequence's.
__device__ __forceinline__ bool kv4_paged(const Kv4Args& a, const Kv4Lane& p) {
  return p.page < static_cast<unsigned>(a.num_pages);
}

// Index of the group's 16 bytes of codes, and of its scale.
template <int D>
__device__ __forceinline__ int64_t kv4_chunk(const Kv4Args& a, const Kv4Lane& p) {
  const int64_t group = (static_cast<int64_t>(p.page) * a.hkv + p.g) * (D / kKv4Group) + p.grp;
  return (group << a.page_shift) + (p.t & ((1 << a.page_shift) - 1));
}

// The bf16 row of a lane: element index of its 8 elements.
template <int D>
__device__ __forceinline__ int64_t kv4_row(const Kv4Args& a, const Kv4Lane& p) {
  return ((static_cast<int64_t>(blockIdx.y) * a.tokens + p.j) * a.hkv + p.g) * D + p.grp * kKv4Group + 8 * (threadIdx.x & 3);
}

template <int D, int kTile>
__global__ __launch_bounds__(kKv4Threads) void kv4_append_kernel(Kv4Args a, const uint16_t* __restrict__ k_new,
                                                                 const uint16_t* __restrict__ v_new) {
  const Kv4Lane p = kv4_lane<D, kTile>(a);
  // (a run past the last token, a lane before the first, or no page: the four
  // lanes of the exchange below stay together, as they are of one token; the
  // values are asked for together with the page id, not behind the branch on it)
  if (!p.in || p.t < 0) return;
  u32x4 x = ld16((blockIdx.z ? v_new : k_new) + kv4_row<D>(a, p));
  asm volatile("" : "+v"(x) : "s"(a.k), "s"(a.ks), "s"(a.v), "s"(a.vs));
  if (!kv4_paged(a, p)) return;
  const int64_t chunk = kv4_chunk<D>(a, p);
  // the group's largest biased exponent: of 8 elements in the lane, then of
  // its 4 lanes
  unsigned e = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned lo = (x[i] >> 7) & 255, hi = (x[i] >> 23) & 255;
    e = max(e, max(lo, hi));
  }
  e = max(e, static_cast<unsigned>(__builtin_amdgcn_mov_dpp(static_cast<int>(e), 0xB1, 0xF, 0xF, true)));  // lane ^ 1
  e = max(e, static_cast<unsigned>(__builtin_amdgcn_mov_dpp(static_cast<int>(e), 0x4E, 0xF, 0xF, true)));  // lane ^ 2
  const unsigned s = e == 255 ? 255 : (e > 2 ? e - 2 : 0);
  const float unit = scale_of(s);
  unsigned w = 0;
  const unsigned x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x0), unit, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x1), unit, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x2), unit, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x3), unit, 3);
  if (s == 255) w = 0;
  reinterpret_cast<unsigned*>((blockIdx.z ? a.v : a.k) + 16 * chunk)[threadIdx.x & 3] = w;
  if ((threadIdx.x & 3) == 0) (blockIdx.z ? a.vs : a.ks)[chunk] = static_cast<uint8_t>(s);
}

template <int D, int kTile>
__global__ __launch_bounds__(kKv4Threads) void kv4_read_kernel(Kv4Args a, uint16_t* __restrict__ k_out,
                                                               uint16_t* __restrict__ v_out) {
  const Kv4Lane p = kv4_lane<D, kTile>(a);
  if (!p.in) return;
  bf16x8 y = {};
  if (kv4_paged(a, p)) {
    const int64_t chunk = kv4_chunk<D>(a, p);
    const unsigned w = reinterpret_cast<const unsigned*>((blockIdx.z ? a.v : a.k) + 16 * chunk)[threadIdx.x & 3];
    y = decode8(w, scale_of((blockIdx.z ? a.vs : a.ks)[chunk]));
  }
  *reinterpret_cast<u32x4*>((blockIdx.z ? v_out : k_out) + kv4_row<D>(a, p)) = __builtin_bit_cast(u32x4, y);
}

// --------------------------------------------------------------- attention
// Eight bf16 values times zero: a NaN where they are not finite.
__device__ __forceinline__ u32x4 times_zero(u32x4 x) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = ((x[i] & 0x7F80u) == 0x7F80u ? 0x7FC0u : 0u) | ((x[i] & 0x7F800000u) == 0x7F800000u ? 0x7FC00000u : 0u);
  return x;
}

typedef const __attribute__((address_space(1))) uint8_t global_u8;
typedef const __attribute__((address_space(1))) u32x4 global_u32x4;

template <int D>
struct Shape4 {
  static constexpr int kParts = D == 256 ? 2 : 1;      // 128-wide parts of a key (K's loads and products per tile)
  static constexpr int kQK = D / 32;                   // products of K and q per tile
  static constexpr int kVLoads = D / 64;               // 16-byte loads per lane of a step's V
  static constexpr int kRing = 2;                      // steps of loads in flight per wave
  static constexpr int kDT = D / 16;                   // 16-wide d tiles of the output
  static constexpr int kRowBytes = 2 * D + 32;         // a V row in LDS, padded as in the bf16 kernel
  static constexpr int kTileBytes = kStep * kRowBytes;
  static constexpr int kAccBytes = 64 * kDT * 16;
  static_assert(kAccBytes <= kTileBytes, "accumulator exchange reuses the tile");
};
template <int D>
__host__ __device__ constexpr int ml_offset4(int waves) { return waves * Shape4<D>::kTileBytes; }
template <int D>
__host__ __device__ constexpr int pref_offset4(int waves) { return ml_offset4<D>(waves) + waves * 16 * 2 * 4; }

// What is not a pointer: those are arguments of their own, so that the compiler
// knows what is only read and takes page ids through the scalar cache.
struct Attn4 {
  int batch, hq, hkv, group, hgs, page_shift, num_pages, maxp, min_steps, nq, window, sinks, chunks, chunk_steps;
  float scale;  // in log2 units, > 0
  // q as the products take it: its bits exclusive or `flip`, the signs turned for
  // a negative scale; for a zero one (`zero`) times_zero of them, and a scale of 1
  unsigned flip;
  int zero;
};

constexpr float kLazy = 8.f;  // see the online softmax
// The largest scale of a value under which a probability of 2^kLazy leaves room
// for the sum of a table's 2^30 tokens in fp32: 30 + 8 + log2(6) + 214 - 127 < 128.
constexpr unsigned kLazyScale = 214;

// One pass over the cache with the split, the columns and the partials of the
// bf16 kernel (pda_kernels.hip): a wave takes 32-token steps of one kv head,
// the columns of its products are (query token, head of the group) pairs.
// What differs is how a step gets to the matrix cores:
//  * K: lane (r, g4) loads token r's group g4 (16 bytes: 32 elements) of a
//    16-token tile.  Converted, its four runs of 8 elements are the A operand
//    of four v_mfma_f32_16x16x32_bf16 as they stand, since the order of d
//    inside a product is free as long as q's operand has the same: K does not
//    pass through LDS.  (The matrix cores also multiply E2M1 codes with their
//    scales directly, q as two E4M3 parts: 32 conversions a step fewer, the
//    same time, and scores off by ~2^-15 of themselves, which is why not.)
//  * V: loaded the same way, converted with its scales to bf16 rows in LDS
//    and read back transposed, as in the bf16 kernel.
//
// A quarter of the bf16 kernel's bytes leaves a step ~1300 cycles of a SIMD at
// 7 TB/s, and it takes (D = 128, counters) 176 vector, 26 matrix and 24 LDS
// instructions: the time goes where a wave waits.  So:
//  * 12 waves a CU (3 a SIMD, 168 registers each), each with the loads of two
//    steps in flight, as three workgroups of 4 waves where the prefix over the
//    batch leaves LDS for them: one takes up its next sequence while the others
//    stream.  4 x 131072 tokens, 64:8 heads: 16 waves with one step in flight
//    and vector page ids 131 us a call, scalar page ids 115, 8 waves with four
//    steps 120, 12 waves with two 107; a batch of 64, U[128, 8192] at 32:8
//    heads: 85, 70, 75, 63; loads alone, nothing computed: 97 and 54 + the merge.
//  * every loop value that is the same for the wave is kept in scalar registers
//    (divisions and LDS reads leave theirs in vector ones).
template <int D, bool kFixed>
__global__ __launch_bounds__(64 * kv4_max_waves(D), kv4_max_waves(D) / 4) void attn4_kernel(
    const uint16_t* __restrict__ q, const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_scales,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_scales, const int32_t* __restrict__ bt,
    const int32_t* __restrict__ lens, uint16_t* __restrict__ out, float* __restrict__ ws_acc, float* __restrict__ ws_ml,
    int32_t* __restrict__ ws_pref, Attn4 p) {
  using S = Shape4<D>;
  extern __shared__ __align__(16) unsigned char smem[];
  const int nthreads = blockDim.x;
  const int nwaves = nthreads >> 6;
  const int hgs = p.hgs, nq = p.nq, group = p.group, window = p.window, sinks = p.sinks;
  const int phases = nwaves / hgs;
  const int ngroups = p.hkv / hgs;
  const int ncols = group * nq;
  int32_t* pref = reinterpret_cast<int32_t*>(smem + pref_offset4<D>(nwaves));
  int32_t* lens_s = pref + p.batch + 1;
  float* ml_x = reinterpret_cast<float*>(smem + ml_offset4<D>(nwaves));
  int32_t* scan = reinterpret_cast<int32_t*>(smem);
  const int tid = threadIdx.x;
  const int page = 1 << p.page_shift;
  const int max_ctx = p.maxp << p.page_shift;
  // What a sequence counts for in the stream-K ranges: its steps, and four for
  // each step phase ahead of them, for taking up another piece (page ids, then
  // the first loads, q's operand, the exchange of the phases: ~5 us of a
  // workgroup, where a step takes 1.5).  Batches of 101 (Zipf) and 64 (uniform)
  // sequences: 168 and 62 us without, 139 and 59 with two, 124 and 59 with four.
  const int extra = 4 * phases;
  auto extent = [&](int steps) { return steps + (steps > 0 ? extra : 0); };

  if constexpr (!kFixed) {
    // prefix over the batch of what each sequence counts for
#pragma unroll 8
    for (int b = tid; b < p.batch; b += nthreads) lens_s[b] = clamp_len(lens[b], max_ctx);
    __syncthreads();
    const int per = (p.batch + nthreads - 1) / nthreads;
    const int lo = tid * per;
    const int hi = min(p.batch, lo + per);
    int sum = 0;
    for (int b = lo; b < hi; ++b) sum += extent(seq_steps(lens_s[b], nq, window, sinks));
    int incl = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int v = __shfl_up(incl, off, 64);
      if ((tid & 63) >= off) incl += v;
    }
    if ((tid & 63) == 63) scan[tid >> 6] = incl;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < (tid >> 6); ++w) before += scan[w];
    int run = before + incl - sum;
    for (int b = lo; b < hi; ++b) {
      pref[b] = run;
      run += extent(seq_steps(lens_s[b], nq, window, sinks));
    }
    if (tid == nthreads - 1) pref[p.batch] = before + incl;
    __syncthreads();
    if (blockIdx.x == 0) {  // the merge kernel's copy, and the zero rows of empty sequences
      for (int b = tid; b <= p.batch; b += nthreads) ws_pref[b] = pref[b];
      const int row16 = nq * p.hq * D / 8;
      const int ln = tid & 63;
      for (int c = (tid >> 6) * 64; c < p.batch; c += nwaves * 64) {
        uint64_t empty = __ballot(c + ln < p.batch && pref[c + ln + 1] == pref[c + ln]);
        while (empty) {
          const int j = __builtin_ctzll(empty);
          empty &= empty - 1;
          u32x4* orow = reinterpret_cast<u32x4*>(out + static_cast<int64_t>(c + j) * nq * p.hq * D);
          for (int i = ln; i < row16; i += 64) orow[i] = u32x4{0u, 0u, 0u, 0u};
        }
      }
    }
    __syncthreads();  // the scan area becomes the tiles
  }

  const int lane = tid & 63;
  const int wid = uniform(tid >> 6);
  const int hi_w = uniform(wid % hgs);  // kv head of this wave within the group
  const int ph = uniform(wid / hgs);    // step phase of this wave
  const int g4 = lane >> 4;    // lane group: MFMA k block / C row block
  const int c = lane & 15;     // MFMA row (A) / column (B, C)
  const int qj = c < ncols ? c / group : nq - 1;
  const int qh = c - (c / group) * group;
  const int blk = blockIdx.x;
  int32_t* ws_split = ws_pref + p.batch + 1;

  int b, hg, s0, nb;
  int fx_a[S::kRing] = {}, fx_b[S::kRing] = {};  // fixed split: page ids of the first steps
  int64_t x = 0, xend, total = 1, beff = 1;
  if constexpr (kFixed) {
    const int e = div_small_u(blk, p.chunks);
    b = div_small_u(e, ngroups);
    hg = e - b * ngroups;
    s0 = (blk - e * p.chunks) * p.chunk_steps;
    // without a window the first steps' page ids do not depend on the length:
    // both are requested together (entries past the sequence's pages are
    // clamped into the pool like any other, and masked)
    if (window == 0) {
#pragma unroll
      for (int i = 0; i < S::kRing; ++i) {
        const int t = (s0 + ph + i * phases) * kStep;
        const int ja = t >> p.page_shift, jb = (t + 16) >> p.page_shift;
        fx_a[i] = bt[static_cast<int64_t>(b) * p.maxp + (ja < p.maxp ? ja : p.maxp - 1)];
        fx_b[i] = bt[static_cast<int64_t>(b) * p.maxp + (jb < p.maxp ? jb : p.maxp - 1)];
      }
    }
    nb = seq_steps(clamp_len(uniform(lens[b]), max_ctx), nq, window, sinks);
    if (s0 >= nb) {  // a chunk past the sequence's end
      if (nb == 0 && s0 == 0) {  // an empty sequence: zero rows
        const int row16 = hgs * group * D / 8;
        for (int j = 0; j < nq; ++j) {
          u32x4* orow = reinterpret_cast<u32x4*>(
              out + ((static_cast<int64_t>(b) * nq + j) * p.hq + hg * hgs * group) * D);
          for (int i = tid; i < row16; i += nthreads) orow[i] = u32x4{0u, 0u, 0u, 0u};
        }
      }
      return;
    }
    xend = nb - s0 < p.chunk_steps ? nb - s0 : p.chunk_steps;
  } else {
    total = static_cast<int64_t>(uniform(pref[p.batch])) * ngroups;
    const int64_t per_block_min = static_cast<int64_t>(p.min_steps) * phases;
    beff = (total + per_block_min - 1) / per_block_min;
    beff = beff < gridDim.x ? beff : gridDim.x;
    if (blk >= beff) {  // (also where the whole batch is empty)
      if (tid == 0) ws_split[blk] = -1;
      return;
    }
    x = (static_cast<int64_t>(blk) * total) / beff;
    xend = (static_cast<int64_t>(blk + 1) * total) / beff;
    const int y = static_cast<int>(x / ngroups);  // the largest b with pref[b] <= y holds x
    int lo = 0, hi = p.batch - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (uniform(pref[mid]) <= y) lo = mid; else hi = mid - 1;
    }
    b = lo;
    nb = uniform(pref[b + 1]) - uniform(pref[b]);
    const int rel = static_cast<int>(x - static_cast<int64_t>(uniform(pref[b])) * ngroups);
    hg = rel / nb;
    s0 = rel - hg * nb;
    if (tid == 0) ws_split[blk] = (s0 > 0 && owner_of(x - s0, total, beff) == blk - 1) ? b * ngroups + hg : -1;
  }

  int left = static_cast<int>(xend - x);  // steps of the workgroup (fewer than 2^31: a call has no more)
  unsigned char* tile = smem + wid * S::kTileBytes;
  const int head_bytes = (D / 2) << p.page_shift;  // codes of a kv head's page; its scales: head_bytes / 16
  const unsigned page_bytes = static_cast<unsigned>(head_bytes) * p.hkv;  // at most 2^27
  // K: this lane's codes and scale within a tile: token c, group g4 (and g4 + 4
  // at D = 256; at D = 64 lanes g4 and g4 + 2 share a group, half each)
  const unsigned ksoff = ((D == 64 ? g4 & 1 : g4) << p.page_shift) + c;
  const int dof = D == 64 ? 32 * (g4 & 1) + 16 * (g4 >> 1) : 32 * g4;  // its first d
  // V: load i takes token c of tile vtile(i), group vgrp(i)
  auto vtile = [&](int i) { return D == 64 ? g4 >> 1 : D == 256 ? i >> 1 : i; };
  auto vgrp = [&](int i) { return D == 64 ? g4 & 1 : D == 256 ? g4 + 4 * (i & 1) : g4; };

  while (true) {
    b = uniform(b);
    hg = uniform(hg);
    s0 = uniform(s0);
    nb = uniform(nb);
    left = uniform(left);
    const int s1 = left < nb - s0 ? s0 + left : nb;
    const int L = uniform(kFixed ? clamp_len(lens[b], max_ctx) : lens_s[b]);
    const int npages = (L + page - 1) >> p.page_shift;
    const int lo_seq = uniform(seq_start(L, nq, window));
    const int pinned = window > 0 ? min(sinks, lo_seq) : 0;  // keys [0, pinned) are seen as sinks
    const int nsink = uniform(sink_steps(L, nq, window, sinks));
    const int sb = lo_seq / kStep - nsink;  // absolute step of index i >= nsink: i + sb
    const int lead = kFixed ? 0 : nb - seq_steps(L, nq, window, sinks);
    const int t0 = max(s0 - lead, 0), t1 = max(s1 - lead, 0);
    // The wave's steps of the piece: sw, sw + phases, ...  One with none takes a
    // step all the same, of a sequence of no tokens: everything in it is masked
    // (skipping it cost the loop 60 registers in spills).
    const int sw = uniform(t0 + ph);
    const int steps = sw < t1 ? (t1 - sw + phases - 1) / phases : 0;
    const int nsteps = uniform(steps > 0 ? steps : 1);
    const int Lw = steps > 0 ? L : 0;
    const int hi_c = Lw - nq + 1 + qj;  // this column sees keys [lo_c, hi_c) and [0, min(hi_c, sinks))
    const int lo_c = window > 0 ? max(0, hi_c - window) : 0;
    const int hi_min = Lw - nq + 1;
    const int lo_max = window > 0 ? max(0, Lw - window) : 0;
    const int32_t* bt_row = bt + static_cast<int64_t>(b) * p.maxp;
    const int g = uniform(hg * hgs + hi_w);

    f32x4 acc[S::kDT];
#pragma unroll
    for (int dt = 0; dt < S::kDT; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -__builtin_inff();
    float seen = -__builtin_inff();  // the largest score of this lane's tokens, unscaled
    f32x4 l_acc = {0.f, 0.f, 0.f, 0.f};  // the column's sum of probabilities, in every row

    // first token of the wave's k-th step (clamped to its last)
    auto token_of = [&](int k) {
      const int i = sw + (k < nsteps ? k : nsteps - 1) * phases;
      return (i < nsink ? i : i + sb) * kStep;
    };
    // page ids of the two tiles of the step at token t
    auto load_pids = [&](int t, int& pa, int& pb) {
      const int ja = t >> p.page_shift, jb = (t + 16) >> p.page_shift;
      pa = bt_row[ja < npages ? ja : npages - 1];
      pb = bt_row[jb < npages ? jb : npages - 1];
    };
    // Where a tile's codes lie from the head's first page on (its scales: a
    // sixteenth of that).  A tile that no query sees -- past the end, or between
    // the sinks and the window, where its page may have been released -- is
    // read from the page that its id is clamped to and masked: that is at most
    // two tiles a piece, and spares every other one a descriptor.
    auto tile_at = [&](int t, int id) {
      const unsigned raw = static_cast<unsigned>(uniform(id));
      const unsigned pid = raw < static_cast<unsigned>(p.num_pages) ? raw : p.num_pages - 1;
      return static_cast<uint64_t>(pid) * page_bytes + 16 * (t & (page - 1));
    };
    const uint8_t* kg = k_codes + static_cast<int64_t>(g) * head_bytes;
    const uint8_t* vg = v_codes + static_cast<int64_t>(g) * head_bytes;
    const uint8_t* ksg = k_scales + static_cast<int64_t>(g) * (head_bytes >> 4);
    const uint8_t* vsg = v_scales + static_cast<int64_t>(g) * (head_bytes >> 4);
    const unsigned part = 4u << p.page_shift;  // scales between the 128-wide parts of a key
    // a scalar base and a 32-bit offset per lane, as the loads take them (left
    // to itself the compiler adds the tile's place to a pointer per lane)
    auto at_scalar = [](const uint8_t* x) {
      asm volatile("" : "+s"(x));
      return (global_u8*)x;
    };
    struct Set {  // a step's codes and scales
      u32x4 kw[2][S::kParts], vw[S::kVLoads];
      unsigned ks[2][S::kParts], vs[S::kVLoads];
    };
    // Loads of a step past the wave's last have `only` = 0: every lane asks for
    // the first 16 bytes of the last step's tile, one request instead of a
    // branch (at whose join the compiler would wait for the path with fewer
    // loads in flight).
    auto load_k = [&](const uint64_t (&at)[2], unsigned only, Set& r) {
      const unsigned o = ksoff & only;
#pragma unroll
      for (int T = 0; T < 2; ++T)
#pragma unroll
        for (int i = 0; i < S::kParts; ++i) {
          r.kw[T][i] = __builtin_nontemporal_load((global_u32x4*)(at_scalar(kg + at[T] + 16 * i * part) + 16 * o));
          r.ks[T][i] = at_scalar(ksg + (at[T] >> 4) + i * part)[o];
        }
    };
    auto load_v = [&](const uint64_t (&at)[2], unsigned only, Set& r) {
      const unsigned o = ksoff & only;
#pragma unroll
      for (int i = 0; i < S::kVLoads; ++i) {
        if constexpr (D == 64) {  // a lane for each token of the step and group
          const uint64_t from = g4 >> 1 ? at[1] : at[0];
          r.vw[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vg + from + 16 * o));
          r.vs[i] = (vsg + (from >> 4))[o];
        } else {
          const int T = D == 256 ? i >> 1 : i, h = D == 256 ? i & 1 : 0;
          r.vw[i] = __builtin_nontemporal_load((global_u32x4*)(at_scalar(vg + at[T] + 16 * h * part) + 16 * o));
          r.vs[i] = at_scalar(vsg + (at[T] >> 4) + h * part)[o];
        }
      }
    };
    auto lds_order = [&]() {  // LDS writes of this wave before its reads, and back
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };

    // Loads run kRing steps ahead: a set's registers are loaded again as soon as
    // its step has used them, K after the products with q, V after its rows are
    // in LDS.  Page ids (scalar loads) run one step further.
    // q's rows are requested first: vector loads arrive in order.
    u32x4 qraw[S::kQK];
    {
      // (a padding column reads a row inside q, and is zeroed below)
      const uint16_t* qrow = q + ((static_cast<int64_t>(b) * nq + qj) * p.hq + g * group + qh) * D + dof;
#pragma unroll
      for (int i = 0; i < S::kQK; ++i) qraw[i] = ld16(qrow + 128 * (i >> 2) + 8 * (i & 3));
    }
    Set ring[S::kRing];
    int pa, pb;
#pragma unroll
    for (int i = 0; i < S::kRing; ++i) {
      int t = token_of(i);
      if (kFixed && window == 0) {
        t = (sw + i * phases) * kStep;
        pa = fx_a[i];
        pb = fx_b[i];
      } else {
        load_pids(t, pa, pb);
      }
      const uint64_t at[2] = {tile_at(t, pa), tile_at(t + 16, pb)};
      const unsigned only = i < nsteps ? ~0u : 0u;
      load_k(at, only, ring[i]);
      load_v(at, only, ring[i]);
    }
    load_pids(token_of(S::kRing), pa, pb);
    // q as the B operand: column c, elements 8 j .. +7 of the lane's part of d
    bf16x8 qop[S::kQK];
#pragma unroll
    for (int i = 0; i < S::kQK; ++i) {
      const u32x4 x = p.zero ? times_zero(qraw[i]) : qraw[i] ^ p.flip;
      qop[i] = __builtin_bit_cast(bf16x8, c < ncols ? x : u32x4{0u, 0u, 0u, 0u});
    }
    {
      auto step = [&](int k, Set& r) {
        const int t = token_of(k);
        const bool edge = (t + kStep > hi_min) | ((t < lo_max) & (t + kStep > sinks));  // some key is masked
        // S^T = K Q^T: rows = tokens 16 T + 4 g4 + i, column c
        f32x4 sacc[2];
#pragma unroll
        for (int T = 0; T < 2; ++T) {
          sacc[T] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < S::kQK; ++i) {
            const u32x4 w = r.kw[T][i >> 2];
            const unsigned word = D == 64 ? (g4 > 1 ? w[2 + (i & 1)] : w[i & 1]) : w[i & 3];
            sacc[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(word, scale_of(r.ks[T][i >> 2])), qop[i], sacc[T], 0, 0, 0);
          }
        }
        const int ta = token_of(k + S::kRing);
        const uint64_t at[2] = {tile_at(ta, pa), tile_at(ta + 16, pb)};
        const unsigned only = k + S::kRing < nsteps ? ~0u : 0u;
        load_k(at, only, r);
        load_pids(token_of(k + S::kRing + 1), pa, pb);
        // V rows that no query of the sequence sees (only where some key is
        // masked): zeros, never NaN * 0
        unsigned apart = 0;  // tokens of the step that add_row_apart takes
        if (edge) {
#pragma unroll
          for (int i = 0; i < S::kVLoads; ++i) {
            const int tok = t + 16 * vtile(i) + c;
            const bool live = (tok < Lw) & ((tok >= lo_seq) | (tok < pinned));
            r.vs[i] = live ? r.vs[i] : 0;  // (2^-127 times codes that are finite, times a probability of zero)
            // (from a unit of 2^126 on a value may be an infinity, 255 is NaN)
            const bool all = (tok < hi_min) & ((tok >= lo_max) | (tok < sinks));
            uint64_t odd = __ballot((r.vs[i] >= 253) & !all);
            if (odd) {
              odd |= odd >> 16;
              if constexpr (D != 64) odd |= odd >> 32;
              apart |= (static_cast<unsigned>(odd) & 0xFFFF) << (D == 64 ? 0 : 16 * vtile(i));
              if constexpr (D == 64) apart |= static_cast<unsigned>(odd >> 32) << 16;
            }
          }
        }
        lds_order();  // the previous step's reads of the tile are done
#pragma unroll
        for (int i = 0; i < S::kVLoads; ++i) {
          unsigned char* row = tile + (16 * vtile(i) + c) * S::kRowBytes + 64 * vgrp(i);
          const float unit = scale_of(r.vs[i]);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            *reinterpret_cast<u32x4*>(row + 16 * j) = __builtin_bit_cast(u32x4, decode8(r.vw[i][j], unit));
        }
        unsigned top = r.vs[0];
#pragma unroll
        for (int i = 1; i < S::kVLoads; ++i) top = max(top, r.vs[i]);
        const bool large = top > kLazyScale;
        load_v(at, only, r);
        // Online softmax in log2 units, against a reference m_run of each column
        // that follows its maximum only when a score passes it by 2^kLazy: the
        // probabilities are then at most 2^kLazy, which costs fp32 and the hi +
        // lo pairs nothing, and most steps neither reduce a maximum across
        // lanes nor rescale the accumulator.  Where the step has values so large
        // that 2^kLazy of them could leave fp32 (`large`) the reference is the
        // maximum itself, as in the bf16 kernel.
        if (edge) {
#pragma unroll
          for (int T = 0; T < 2; ++T)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int tok = t + 16 * T + 4 * g4 + i;
              const bool masked = (tok >= hi_c) | ((tok < lo_c) & (tok >= sinks));
              sacc[T][i] = masked ? -__builtin_inff() : sacc[T][i];
            }
        }
        const float mx0 = fmaxf(fmaxf(sacc[0][0], sacc[0][1]), fmaxf(sacc[0][2], sacc[0][3]));
        const float mx1 = fmaxf(fmaxf(sacc[1][0], sacc[1][1]), fmaxf(sacc[1][2], sacc[1][3]));
        seen = fmaxf(seen, fmaxf(mx0, mx1));
        if (__any((seen * p.scale > m_run + kLazy) | large)) {  // (no key yet: m_run = -inf)
          seen = fmaxf(seen, __shfl_xor(seen, 16));
          seen = fmaxf(seen, __shfl_xor(seen, 32));
          const float m_new = fmaxf(m_run, seen * p.scale);
          // (a column that has still seen no key keeps 0 in its place)
          const float alpha = m_run == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
          m_run = m_new;
          l_acc *= alpha;
#pragma unroll
          for (int dt = 0; dt < S::kDT; ++dt) acc[dt] *= alpha;
        }
        const float m_ref = m_run == -__builtin_inff() ? 0.f : m_run;
        // p = hi + lo, two bf16 values: the products carry it to ~2^-17
        unsigned hi_w2[4], lo_w2[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x2 pf;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int e = 2 * i + j;
            pf[j] = __builtin_amdgcn_exp2f(fmaf(sacc[e >> 2][e & 3], p.scale, -m_ref));
          }
          hi_w2[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(pf, bf16x2));
          const f32x2 rest = {pf[0] - __builtin_bit_cast(float, hi_w2[i] << 16),
                              pf[1] - __builtin_bit_cast(float, hi_w2[i] & 0xFFFF0000u)};
          lo_w2[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(rest, bf16x2));
        }
        const bf16x8 pop = __builtin_bit_cast(bf16x8, u32x4{hi_w2[0], hi_w2[1], hi_w2[2], hi_w2[3]});
        const bf16x8 pop_lo = __builtin_bit_cast(bf16x8, u32x4{lo_w2[0], lo_w2[1], lo_w2[2], lo_w2[3]});
        // their sum is a product with a row of ones (the matrix cores have time)
        const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
        l_acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pop, l_acc, 0, 0, 0);
        l_acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pop_lo, l_acc, 0, 0, 0);
        lds_order();
        while (apart) {
          const int row = __builtin_ctz(apart), tok = t + row;
          apart &= apart - 1;
          add_row_apart<D, S::kRowBytes>(acc, __builtin_bit_cast(u32x4, pop), __builtin_bit_cast(u32x4, pop_lo), tile, row,
                                         (tok < hi_c) & ((tok >= lo_c) | (tok < sinks)));
          lds_order();
        }
        const unsigned char* r0 = tile + (4 * g4 + (c >> 2)) * S::kRowBytes + 8 * (c & 3);
        const unsigned char* r1 = r0 + 16 * S::kRowBytes;
#pragma unroll
        for (int dt = 0; dt < S::kDT; ++dt) {
          const i16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(r0 + 32 * dt));
          const i16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(r1 + 32 * dt));
          const bf16x8 va = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pop, acc[dt], 0, 0, 0);
          acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pop_lo, acc[dt], 0, 0, 0);
        }
      };
      for (int k = 0;;) {
        step(k, ring[0]);
        if (++k >= nsteps) break;
        if constexpr (S::kRing > 1) {
          step(k, ring[1]);
          if (++k >= nsteps) break;
        }
      }
      lds_order();
    }

    // ---- finish the piece: combine the phases of each kv head, then write
    const float l_tot = l_acc[0];
    float big_m = m_run, den = l_tot;
    if (phases > 1) {
      f32x4* accx = reinterpret_cast<f32x4*>(smem);  // [wave][dt][lane], reuses the tiles
      __syncthreads();
#pragma unroll
      for (int dt = 0; dt < S::kDT; ++dt) accx[(wid * S::kDT + dt) * 64 + lane] = acc[dt];
      if (g4 == 0) {
        ml_x[(wid * 16 + c) * 2 + 0] = m_run;
        ml_x[(wid * 16 + c) * 2 + 1] = l_tot;
      }
      __syncthreads();
      if (ph == 0) {
        big_m = -__builtin_inff();
        for (int w = 0; w < phases; ++w) big_m = fmaxf(big_m, ml_x[((w * hgs + hi_w) * 16 + c) * 2]);
        den = 0.f;
#pragma unroll
        for (int dt = 0; dt < S::kDT; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < phases; ++w) {
          const int wp = w * hgs + hi_w;
          const float mp = ml_x[(wp * 16 + c) * 2];
          const float f = mp == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mp - big_m);  // no step: weight 0
          den += f * ml_x[(wp * 16 + c) * 2 + 1];
#pragma unroll
          for (int dt = 0; dt < S::kDT; ++dt) acc[dt] += f * accx[(wp * S::kDT + dt) * 64 + lane];
        }
      }
    }
    if (ph == 0 && c < ncols) {
      if (s0 == 0 && s1 == nb) {
        const float inv = den > 0.f ? 1.0f / den : 0.f;  // a query that sees no key: zero row
        uint16_t* orow = out + ((static_cast<int64_t>(b) * nq + qj) * p.hq + g * group + qh) * D + 4 * g4;
#pragma unroll
        for (int dt = 0; dt < S::kDT; ++dt) {
          bf16x4 o;
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = static_cast<__bf16>(acc[dt][i] * inv);
          *reinterpret_cast<u32x2*>(orow + 16 * dt) = __builtin_bit_cast(u32x2, o);
        }
      } else {
        const int64_t slot = kFixed ? static_cast<int64_t>(blk) : static_cast<int64_t>(blk) + static_cast<int64_t>(b) * ngroups + hg;
        const int64_t row = (slot * hgs + hi_w) * ncols + c;
        float* arow = ws_acc + row * D + 4 * g4;
#pragma unroll
        for (int dt = 0; dt < S::kDT; ++dt) *reinterpret_cast<f32x4*>(arow + 16 * dt) = acc[dt];
        if (g4 == 0) *reinterpret_cast<f32x2*>(ws_ml + row * 2) = f32x2{big_m, den};
      }
    }
    if (phases > 1) __syncthreads();  // the exchange area is a tile again

    left -= s1 - s0;
    if (kFixed || left <= 0) break;
    s0 = 0;
    if (++hg == ngroups) {
      hg = 0;
      do {
        ++b;
        nb = uniform(pref[b + 1]) - uniform(pref[b]);
      } while (nb == 0);
    }
  }
}

template <int D, bool kFixed>
hipError_t launch_attn4(const LaunchArgs& a, const Kv4Args& c, hipStream_t st) {
  static std::atomic<uint64_t> attr_set{0};  // the dynamic-LDS limit, raised once per device
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
  if (!bit || !(attr_set.load() & bit)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(&attn4_kernel<D, kFixed>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, kMaxLdsBytes);
    if (e != hipSuccess) return e;
    attr_set.fetch_or(bit);
  }
  Attn4 p;
  p.batch = a.batch;
  p.hq = a.hq;
  p.hkv = a.hkv;
  p.group = a.group;
  p.hgs = a.hgs;
  p.page_shift = a.page_shift;
  p.num_pages = a.num_pages;
  p.maxp = a.maxp;
  p.min_steps = a.min_steps;
  p.nq = a.nq;
  p.window = a.window;
  p.sinks = a.sinks;
  p.chunks = a.chunks;
  p.chunk_steps = a.chunk_steps;
  const float s = a.scale * kLog2e;
  p.scale = s == 0.f ? 1.f : s < 0.f ? -s : s;
  p.zero = s == 0.f;
  p.flip = s < 0.f ? 0x80008000u : 0u;
  hipLaunchKernelGGL((attn4_kernel<D, kFixed>), dim3(a.grid), dim3(64 * a.waves), kv4_attn_lds_bytes(D, a.batch, a.waves),
                     st, a.q, c.k, c.ks, c.v, c.vs, a.bt, a.lens, a.out, a.ws_acc, a.ws_ml, a.ws_pref, p);
  return hipGetLastError();
}

// Threads of an append or a read: a lane for 8 elements of each token (or of
// each aligned run of 8 tokens that the call may touch).
template <int kTile>
dim3 kv4_grid(const Kv4Args& a) {
  const int64_t runs = kTile == 1 ? a.tokens : (a.tokens + 2 * kTile - 2) / kTile;
  const int64_t threads = runs * kTile * a.hkv * (a.head_dim / 8);
  return dim3(static_cast<unsigned>((threads + kKv4Threads - 1) / kKv4Threads), a.batch, 2);
}

template <int kTile>
hipError_t append4(const Kv4Args& a, const uint16_t* k, const uint16_t* v, hipStream_t st) {
  const dim3 grid = kv4_grid<kTile>(a), block(kKv4Threads);
  if (a.head_dim == 128) hipLaunchKernelGGL((kv4_append_kernel<128, kTile>), grid, block, 0, st, a, k, v);
  else if (a.head_dim == 256) hipLaunchKernelGGL((kv4_append_kernel<256, kTile>), grid, block, 0, st, a, k, v);
  else hipLaunchKernelGGL((kv4_append_kernel<64, kTile>), grid, block, 0, st, a, k, v);
  return hipGetLastError();
}

template <int kTile>
hipError_t read4(const Kv4Args& a, uint16_t* k, uint16_t* v, hipStream_t st) {
  const dim3 grid = kv4_grid<kTile>(a), block(kKv4Threads);
  if (a.head_dim == 128) hipLaunchKernelGGL((kv4_read_kernel<128, kTile>), grid, block, 0, st, a, k, v);
  else if (a.head_dim == 256) hipLaunchKernelGGL((kv4_read_kernel<256, kTile>), grid, block, 0, st, a, k, v);
  else hipLaunchKernelGGL((kv4_read_kernel<64, kTile>), grid, block, 0, st, a, k, v);
  return hipGetLastError();
}

}  // namespace

// Runs of 8 tokens from 8 tokens a call on.
hipError_t launch_kv4_append(const Kv4Args& a, const uint16_t* k_new, const uint16_t* v_new, hipStream_t st) {
  return a.tokens >= 8 ? append4<8>(a, k_new, v_new, st) : append4<1>(a, k_new, v_new, st);
}

hipError_t launch_kv4_read(const Kv4Args& a, uint16_t* k_out, uint16_t* v_out, hipStream_t st) {
  return a.tokens >= 8 ? read4<8>(a, k_out, v_out, st) : read4<1>(a, k_out, v_out, st);
}

hipError_t launch_kv4_attn(const LaunchArgs& a, const Kv4Args& c, hipStream_t st) {
  if (a.chunks > 0) {
    if (a.head_dim == 128) return launch_attn4<128, true>(a, c, st);
    if (a.head_dim == 256) return launch_attn4<256, true>(a, c, st);
    return launch_attn4<64, true>(a, c, st);
  }
  if (a.head_dim == 128) return launch_attn4<128, false>(a, c, st);
  if (a.head_dim == 256) return launch_attn4<256, false>(a, c, st);
  return launch_attn4<64, false>(a, c, st);
}

size_t kv4_attn_lds_bytes(int head_dim, int batch, int waves) {
  const int base = head_dim == 256 ? pref_offset4<256>(waves) : head_dim == 128 ? pref_offset4<128>(waves) : pref_offset4<64>(waves);
  return static_cast<size_t>(base) + (2 * static_cast<size_t>(batch) + 1) * sizeof(int32_t);
}

}  // namespace pda
