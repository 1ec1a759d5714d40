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
  int64_t chunk;  // index of the group's 16 bytes of codes, and of its scale
  bool in;        // the call has this token (chunk is valid only where t >= 0)
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
  p.chunk = 0;
  if (p.in && p.t >= 0) {
    const unsigned raw = static_cast<unsigned>(a.bt[static_cast<int64_t>(b) * a.maxp + (p.t >> a.page_shift)]);
    const int64_t page = raw < static_cast<unsigned>(a.num_pages) ? raw : a.num_pages - 1;
    p.chunk = (((page * a.hkv + p.g) * kGroups + p.grp) << a.page_shift) + (p.t & ((1 << a.page_shift) - 1));
  }
  return p;
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
  // (a run past the last token, or a lane before the first: its four lanes
  // stay together for the exchange below, as they are of one token)
  if (!p.in || p.t < 0) return;
  const u32x4 x = ld16((blockIdx.z ? v_new : k_new) + kv4_row<D>(a, p));
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
  reinterpret_cast<unsigned*>((blockIdx.z ? a.v : a.k) + 16 * p.chunk)[threadIdx.x & 3] = w;
  if ((threadIdx.x & 3) == 0) (blockIdx.z ? a.vs : a.ks)[p.chunk] = static_cast<uint8_t>(s);
}

template <int D, int kTile>
__global__ __launch_bounds__(kKv4Threads) void kv4_read_kernel(Kv4Args a, uint16_t* __restrict__ k_out,
                                                               uint16_t* __restrict__ v_out) {
  const Kv4Lane p = kv4_lane<D, kTile>(a);
  if (!p.in) return;
  bf16x8 y = {};
  if (p.t >= 0) {
    const unsigned w = reinterpret_cast<const unsigned*>((blockIdx.z ? a.v : a.k) + 16 * p.chunk)[threadIdx.x & 3];
    y = decode8(w, scale_of((blockIdx.z ? a.vs : a.ks)[p.chunk]));
  }
  *reinterpret_cast<u32x4*>((blockIdx.z ? v_out : k_out) + kv4_row<D>(a, p)) = __builtin_bit_cast(u32x4, y);
}

// --------------------------------------------------------------- attention
template <int D>
struct Shape4 {
  static constexpr int kParts = D == 256 ? 2 : 1;      // loads of codes per 16-token tile (K and V each)
  static constexpr int kWords = D == 64 ? 2 : 4;       // 32-bit words of codes per load and lane
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

struct Attn4 {
  const uint16_t* q;
  const uint8_t *k, *ks, *v, *vs;
  const int32_t *bt, *lens;
  uint16_t* out;
  float *ws_acc, *ws_ml;
  int32_t* ws_pref;
  int batch, hq, hkv, group, hgs, page_shift, num_pages, maxp, min_steps, nq, window, sinks, chunks, chunk_steps;
  float scale;  // in log2 units, >= 0
  unsigned flip;  // 0x80008000 where the caller's scale is negative: q's signs are turned
};

// One pass over the cache with the split, the columns and the partials of the
// bf16 kernel (pda_kernels.hip): a wave takes 32-token steps of one kv head,
// the columns of its products are (query token, head of the group) pairs.
// What differs is how a step gets to the matrix cores:
//  * K: lane (r, g4) loads token r's group g4 (16 bytes: 32 elements) of a
//    16-token tile.  Converted, its four runs of 8 elements are the A operand
//    of four v_mfma_f32_16x16x32_bf16 as they stand, since the order of d
//    inside a product is free as long as q's operand has the same: K does not
//    pass through LDS.
//  * V: loaded the same way, converted with its scales to bf16 rows in LDS
//    and read back transposed, as in the bf16 kernel.
template <int D, bool kFixed>
__global__ __launch_bounds__(64 * kv4_max_waves(D), 2 * kKv4WorkgroupsPerCu * kv4_max_waves(D) / 8) void attn4_kernel(Attn4 p) {
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
  const int extra = (phases > 1 || D == 256) ? phases : 0;
  auto extent = [&](int steps) { return steps + (steps > 0 && steps < 8 * phases ? extra : 0); };

  if constexpr (!kFixed) {
    // prefix over the batch of what each sequence counts for
#pragma unroll 8
    for (int b = tid; b < p.batch; b += nthreads) lens_s[b] = clamp_len(p.lens[b], max_ctx);
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
      for (int b = tid; b <= p.batch; b += nthreads) p.ws_pref[b] = pref[b];
      const int row16 = nq * p.hq * D / 8;
      const int ln = tid & 63;
      for (int c = (tid >> 6) * 64; c < p.batch; c += nwaves * 64) {
        uint64_t empty = __ballot(c + ln < p.batch && pref[c + ln + 1] == pref[c + ln]);
        while (empty) {
          const int j = __builtin_ctzll(empty);
          empty &= empty - 1;
          u32x4* orow = reinterpret_cast<u32x4*>(p.out + static_cast<int64_t>(c + j) * nq * p.hq * D);
          for (int i = ln; i < row16; i += 64) orow[i] = u32x4{0u, 0u, 0u, 0u};
        }
      }
    }
    __syncthreads();  // the scan area becomes the tiles
  }

  const int lane = tid & 63;
  const int wid = uniform(tid >> 6);
  const int hi_w = wid % hgs;  // kv head of this wave within the group
  const int ph = wid / hgs;    // step phase of this wave
  const int g4 = lane >> 4;    // lane group: MFMA k block / C row block
  const int c = lane & 15;     // MFMA row (A) / column (B, C)
  const int qj = c < ncols ? c / group : nq - 1;
  const int qh = c - (c / group) * group;
  const int blk = blockIdx.x;
  int32_t* ws_split = p.ws_pref + p.batch + 1;

  int b, hg, s0, nb;
  int64_t x = 0, xend, total = 1, beff = 1;
  if constexpr (kFixed) {
    const int e = div_small_u(blk, p.chunks);
    b = div_small_u(e, ngroups);
    hg = e - b * ngroups;
    s0 = (blk - e * p.chunks) * p.chunk_steps;
    nb = seq_steps(clamp_len(uniform(p.lens[b]), max_ctx), nq, window, sinks);
    if (s0 >= nb) {  // a chunk past the sequence's end
      if (nb == 0 && s0 == 0) {  // an empty sequence: zero rows
        const int row16 = hgs * group * D / 8;
        for (int j = 0; j < nq; ++j) {
          u32x4* orow = reinterpret_cast<u32x4*>(
              p.out + ((static_cast<int64_t>(b) * nq + j) * p.hq + hg * hgs * group) * D);
          for (int i = tid; i < row16; i += nthreads) orow[i] = u32x4{0u, 0u, 0u, 0u};
        }
      }
      return;
    }
    xend = nb - s0 < p.chunk_steps ? nb - s0 : p.chunk_steps;
  } else {
    total = static_cast<int64_t>(pref[p.batch]) * ngroups;
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

  unsigned char* tile = smem + wid * S::kTileBytes;
  const int64_t head_bytes = static_cast<int64_t>(D / 2) << p.page_shift;  // codes of a kv head's page
  const int64_t head_scales = static_cast<int64_t>(D / kKv4Group) << p.page_shift;
  // this lane's codes and scale within a tile: token c, group g4 (and g4 + 4
  // at D = 256; at D = 64 half a group)
  const int grp0 = D == 64 ? g4 >> 1 : g4;
  const int soff = (grp0 << p.page_shift) + c;
  const int coff = 16 * soff + (D == 64 ? 8 * (g4 & 1) : 0);
  const int dof = D == 64 ? 16 * g4 : 32 * g4;  // d of the lane's first element

  while (true) {
    const int64_t remaining = xend - x;
    const int s1 = remaining < nb - s0 ? s0 + static_cast<int>(remaining) : nb;
    const int L = uniform(kFixed ? clamp_len(p.lens[b], max_ctx) : lens_s[b]);
    const int npages = (L + page - 1) >> p.page_shift;
    const int lo_seq = uniform(seq_start(L, nq, window));
    const int pinned = window > 0 ? min(sinks, lo_seq) : 0;  // keys [0, pinned) are seen as sinks
    const int nsink = uniform(sink_steps(L, nq, window, sinks));
    const int sb = lo_seq / kStep - nsink;  // absolute step of index i >= nsink: i + sb
    const int lead = kFixed ? 0 : nb - seq_steps(L, nq, window, sinks);
    const int t0 = max(s0 - lead, 0), t1 = max(s1 - lead, 0);
    const int hi_c = L - nq + 1 + qj;  // this column sees keys [lo_c, hi_c) and [0, sinks)
    const int lo_c = window > 0 ? max(0, hi_c - window) : 0;
    const int hi_min = L - nq + 1;
    const int lo_max = window > 0 ? max(0, L - window) : 0;
    const int32_t* bt_row = p.bt + static_cast<int64_t>(b) * p.maxp;
    const int g = hg * hgs + hi_w;

    bf16x8 qop[D / 32];
    {
      const uint16_t* qrow = p.q + ((static_cast<int64_t>(b) * nq + qj) * p.hq + g * group + qh) * D + dof;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        u32x4 w = {0u, 0u, 0u, 0u};
        if (c < ncols) w = ld16(qrow + (D == 256 ? 128 * (i >> 2) + 8 * (i & 3) : 8 * i)) ^ p.flip;
        qop[i] = __builtin_bit_cast(bf16x8, w);
      }
    }
    f32x4 acc[S::kDT];
#pragma unroll
    for (int dt = 0; dt < S::kDT; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -__builtin_inff();
    float l_lane = 0.f;

    const int sw = t0 + ph;
    const int nsteps = sw < t1 ? (t1 - sw + phases - 1) / phases : 0;
    auto token_of = [&](int k) {  // first token of the wave's k-th step (clamped to its last)
      k = k < nsteps ? k : nsteps - 1;
      const int i = sw + k * phases;
      return (i < nsink ? i : i + sb) * kStep;
    };
    struct Codes {
      unsigned w[2][S::kParts][S::kWords];  // [tile][part][word]
      unsigned s[2][S::kParts];
    };
    // page ids of a step's two tiles
    auto load_pids = [&](int k, int& pa, int& pb) {
      const int t = token_of(k);
      int ja = t >> p.page_shift, jb = (t + 16) >> p.page_shift;
      ja = ja < npages ? ja : npages - 1;
      jb = jb < npages ? jb : npages - 1;
      pa = bt_row[ja];
      pb = bt_row[jb];
    };
    auto load = [&](int k, int pa, int pb, const uint8_t* codes, const uint8_t* scales, Codes& r) {
      const int t = token_of(k);
#pragma unroll
      for (int T = 0; T < 2; ++T) {
        const int tt = t + 16 * T;
        // a tile past the end, or wholly between the sinks and the window (its
        // page may have been released), is not read
        const bool dead = k >= nsteps || tt >= L || (tt >= pinned && tt + 16 <= lo_seq);
        const unsigned raw = static_cast<unsigned>(uniform(T ? pb : pa));
        const int64_t pid = raw < static_cast<unsigned>(p.num_pages) ? raw : p.num_pages - 1;
        const int slot = tt & (page - 1);
        const int64_t hp = pid * p.hkv + g;
        const __amdgpu_buffer_rsrc_t rc = page_rsrc(codes + hp * head_bytes + 16 * slot, dead ? 0 : static_cast<int>(head_bytes) - 16 * slot);
        const __amdgpu_buffer_rsrc_t rs = page_rsrc(scales + hp * head_scales + slot, dead ? 0 : static_cast<int>(head_scales) - slot);
#pragma unroll
        for (int i = 0; i < S::kParts; ++i) {
          const int po = 4 * i << p.page_shift;
          if constexpr (S::kWords == 4) {
            const u32x4 w = ld16_stream(rc, coff + 16 * po);
#pragma unroll
            for (int j = 0; j < 4; ++j) r.w[T][i][j] = w[j];
          } else {
            const u32x2 w = __builtin_amdgcn_raw_buffer_load_b64(rc, coff, 0, kCachePolicyNT);
            r.w[T][i][0] = w[0];
            r.w[T][i][1] = w[1];
          }
          r.s[T][i] = __builtin_amdgcn_raw_buffer_load_b8(rs, soff + po, 0, 0);
        }
      }
    };
    auto lds_order = [&]() {  // LDS writes of this wave before its reads, and back
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };

    if (nsteps > 0) {
      Codes kr, vr;
      int pa, pb, pa1, pb1;
      load_pids(0, pa, pb);
      load_pids(1, pa1, pb1);
      load(0, pa, pb, p.k, p.ks, kr);
      load(0, pa, pb, p.v, p.vs, vr);
      for (int k = 0; k < nsteps; ++k) {
        const int t = token_of(k);
        const bool edge = t + kStep > hi_min || (t < lo_max && t + kStep > sinks);  // some key is masked
        // S^T = K Q^T: rows = tokens 16 T + 4 g4 + i, column c
        f32x4 sacc[2];
#pragma unroll
        for (int T = 0; T < 2; ++T) {
          sacc[T] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < S::kParts; ++i)
#pragma unroll
            for (int j = 0; j < S::kWords; ++j)
              sacc[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(kr.w[T][i][j], scale_of(kr.s[T][i])),
                                                                 qop[i * S::kWords + j], sacc[T], 0, 0, 0);
        }
        load_pids(k + 2, pa, pb);
        load(k + 1, pa1, pb1, p.k, p.ks, kr);
        // V rows that no query of the sequence sees: zeros, never NaN * 0
        if (t + kStep > L || (t < lo_seq && t + kStep > pinned)) {
#pragma unroll
          for (int T = 0; T < 2; ++T) {
            const int tok = t + 16 * T + c;
            const bool live = tok < L && (tok >= lo_seq || tok < pinned);
#pragma unroll
            for (int i = 0; i < S::kParts; ++i) {
              vr.s[T][i] = live ? vr.s[T][i] : 0;
#pragma unroll
              for (int j = 0; j < S::kWords; ++j) vr.w[T][i][j] = live ? vr.w[T][i][j] : 0;
            }
          }
        }
        lds_order();  // the previous step's reads of the tile are done
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int i = 0; i < S::kParts; ++i)
#pragma unroll
            for (int j = 0; j < S::kWords; ++j)
              *reinterpret_cast<u32x4*>(tile + (16 * T + c) * S::kRowBytes + 2 * (dof + 128 * i + 8 * j)) =
                  __builtin_bit_cast(u32x4, decode8(vr.w[T][i][j], scale_of(vr.s[T][i])));
        load(k + 1, pa1, pb1, p.v, p.vs, vr);
        // online softmax in log2 units
        float sv[2][4];
        float mx = -__builtin_inff();
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float s = sacc[T][i] * p.scale;
            if (edge) {
              const int tok = t + 16 * T + 4 * g4 + i;
              if (tok >= hi_c || (tok < lo_c && tok >= sinks)) s = -__builtin_inff();
            }
            sv[T][i] = s;
            mx = fmaxf(mx, s);
          }
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m_run, mx);
        const float m_ref = m_new == -__builtin_inff() ? 0.f : m_new;  // a column that has seen no key yet
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_ref);
        m_run = m_new;
        bf16x8 pop, pop_lo;  // p = hi + lo: the products carry it to ~2^-17
        float psum = 0.f;
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float pf = __builtin_amdgcn_exp2f(sv[T][i] - m_ref);
            const __bf16 hi = static_cast<__bf16>(pf);
            pop[4 * T + i] = hi;
            pop_lo[4 * T + i] = static_cast<__bf16>(pf - static_cast<float>(hi));
            psum += pf;
          }
        l_lane = l_lane * alpha + psum;
#pragma unroll
        for (int dt = 0; dt < S::kDT; ++dt) acc[dt] *= alpha;
        lds_order();
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
        pa1 = pa;
        pb1 = pb;
      }
      lds_order();
    }

    // ---- finish the piece: combine the phases of each kv head, then write
    float l_tot = l_lane + __shfl_xor(l_lane, 16);
    l_tot += __shfl_xor(l_tot, 32);
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
        const float inv = den > 0.f ? 1.0f / den : (den == 0.f ? 0.f : den);  // no key: a zero row; NaN stays
        uint16_t* orow = p.out + ((static_cast<int64_t>(b) * nq + qj) * p.hq + g * group + qh) * D + 4 * g4;
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
        float* arow = p.ws_acc + row * D + 4 * g4;
#pragma unroll
        for (int dt = 0; dt < S::kDT; ++dt) *reinterpret_cast<f32x4*>(arow + 16 * dt) = acc[dt];
        if (g4 == 0) *reinterpret_cast<f32x2*>(p.ws_ml + row * 2) = f32x2{big_m, den};
      }
    }
    if (phases > 1) __syncthreads();  // the exchange area is a tile again

    x += s1 - s0;
    if (kFixed || x >= xend) break;
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
  p.q = a.q;
  p.k = c.k;
  p.ks = c.ks;
  p.v = c.v;
  p.vs = c.vs;
  p.bt = a.bt;
  p.lens = a.lens;
  p.out = a.out;
  p.ws_acc = a.ws_acc;
  p.ws_ml = a.ws_ml;
  p.ws_pref = a.ws_pref;
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
  p.scale = s < 0.f ? -s : s;
  p.flip = s < 0.f ? 0x80008000u : 0u;
  hipLaunchKernelGGL((attn4_kernel<D, kFixed>), dim3(a.grid), dim3(64 * a.waves), kv4_attn_lds_bytes(D, a.batch, a.waves),
                     st, p);
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
