// Linear products of more than 32 sequences with many output features, for
// MI355X (gfx950, CDNA4, wave64), and the plan of every linear product.
#include <atomic>
#include <cmath>

#include "pda_device.h"
#include "pda_gemv.h"

namespace pda {
namespace {

constexpr uint32_t kOutside = 0x80000000u;  // past any descriptor: reads zero

// y = x W^T over a packed W (16 rows x 32 k, 1 KB, straight into matrix-core
// registers), with the whole epilogue, or one of a.splits parts of the k range.
// A wave takes two row tiles (with a gate a pair) and all column tiles, NT of
// them, over the part; the workgroup's activations lie in LDS once for its W
// waves, kQ steps (64 k) at a time in two places, so that the next ones arrive
// while the waves multiply.  Each wave keeps D steps of weights in flight.
//
// rows_kernel, whose waves deal the k range among themselves, reads 64 rows of
// activations for every 128 rows of weights or fewer, and its waves' sums bound
// its tiles; here every activation in LDS meets all of a workgroup's rows, and a
// workgroup reads all sequences once.  What bounds this form is the CU: operand
// reads of LDS (NT KB for every 2 KB of weights) and matrix instructions take
// about 0.08 us a step and column tile for 256 rows and overlap little, so with
// few row tiles rows_kernel, which needs no parts of k, stays ahead (the choice:
// stream_splits, with both sides' times).
//
// Each row group starts its part of the k range at a place of its own: rows of
// 16 or 32 KB otherwise meet in the same channels (us, all from the same place ->
// so: 80 x 8192 -> 16384 54.5 -> 52.4, 250 94 -> 92; but 128 59.8 -> 61.9 and 80 x
// 8192 -> 12288 47.2 -> 48.5; other k and rows within 1%).  Four row tiles a wave halve the LDS reads, but
// their sums and operands go past the 256 plain registers (101 sequences 46 us
// as before, 200 twice as long).
template <bool kGated, int RT, int NT, int W, int D, int kQ, int kWavesPerSimd>
__global__ __launch_bounds__(W * 64, kWavesPerSimd) void linear_stream_kernel(RowsArgs a, LinearArgs e) {
  constexpr int kSlot = NT * 2048;  // a step's activations
  constexpr int kChunk = kQ * kSlot;
  static_assert(D % kQ == 0, "a round is whole chunks");
  extern __shared__ __align__(1024) unsigned char lds[];

  // part `sp` of the steps, row group rg: parts go to the XCDs by turns, so that
  // their activations are in few L2s
  const int sp = static_cast<int>(blockIdx.x) % a.splits;
  const int rg = static_cast<int>(blockIdx.x) / a.splits;
  const int lane = threadIdx.x & 63;
  const int wv = uniform(threadIdx.x >> 6);
  const int col = lane & 15, kblk = lane >> 4;
  const int kt_count = a.k / kTileK, tiles = a.n / kTileRows;
  const int all_steps = (kt_count + 1) / 2;
  const int begin = sp * all_steps / a.splits;
  const int steps = (sp + 1) * all_steps / a.splits - begin;
  const int group = rg * W + wv;  // the wave's RT row tiles
  // the q-th step: each row group starts at a place of its own
  const int rot = static_cast<int>(static_cast<int64_t>(rg) * steps * a.splits / static_cast<int>(gridDim.x));
  auto step_of = [&](int q) __attribute__((always_inline)) {
    const int s = q + rot;
    return begin + (s < steps ? s : s - steps);
  };

  // row tile r of the wave: with a gate, even ones are the gate's and odd ones
  // their up rows, tiles / 2 on
  auto tile_of = [&](int r) __attribute__((always_inline)) {
    const int t = group * RT + r;
    if constexpr (!kGated) return t;
    return t >> 1 < tiles >> 1 ? (t >> 1) + (r & 1) * (tiles >> 1) : tiles;
  };
  __amdgpu_buffer_rsrc_t rw[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int t = uniform(tile_of(r));
    rw[r] = make_rsrc(a.wp + static_cast<int64_t>(t < tiles ? t : 0) * kt_count * (kTileRows * kTileK),
                      t < tiles ? kt_count * 1024u : 0u);
  }
  u32x4 wa[D][RT][2];
  auto issue_w = [&](int slot, int q) __attribute__((always_inline)) {
    // (k tiles past the end lie outside; so do the steps of the next part)
    const uint32_t at = (q < steps ? static_cast<uint32_t>(step_of(q)) * 2048u : kOutside) + lane * 16u;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int m = 0; m < 2; ++m)
        wa[slot][r][m] = __builtin_amdgcn_raw_buffer_load_b128(rw[r], at + m * 1024u, 0, kCachePolicyNT);
  };
#pragma unroll
  for (int j = 0; j < D; ++j) issue_w(j, j);
  __builtin_amdgcn_sched_barrier(0);

  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x, static_cast<uint32_t>(a.batch) * a.k * 2u);
  const int xpiece = (lane & 7) ^ (lane >> 3);
  const uint32_t xlane = static_cast<uint32_t>(lane >> 3) * a.k * 2u + xpiece * 16u;
  const uint32_t xgroup = static_cast<uint32_t>(a.k) * 16u;  // bytes of 8 rows
  const int groups8 = (a.batch + 7) / 8;
  // the chunk from step q0 on; its 1 KB pieces (8 rows x 64 k) are dealt to the waves
  auto issue_chunk = [&](int q0, unsigned char* to) __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
      const uint32_t k0 = static_cast<uint32_t>(step_of(q0 + q)) * kPairK;
      const bool in = q0 + q < steps && static_cast<int>(k0) + 8 * xpiece < a.k;
#pragma unroll
      for (int i = 0; i < (2 * NT + W - 1) / W; ++i) {
        const int g = i * W + wv;
        const uint32_t off = in && g < groups8 ? xlane + g * xgroup + k0 * 2u : kOutside;
        // (past the last piece into the spare one: as many loads for every wave)
        unsigned char* piece = g < 2 * NT ? to + q * kSlot + g * 1024 : lds + 2 * kChunk;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void*)piece, 16, off, 0, 0, 0);
      }
    }
  };
  const int frag0 = (col >> 3) * 1024 + (col & 7) * 128 + ((kblk ^ (col & 7)) * 16);
  f32x4 acc[RT][NT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int c = 0; c < NT; ++c) acc[r][c] = f32x4{};

  issue_chunk(0, lds);
  __builtin_amdgcn_s_waitcnt(kWaitLoads);
  __syncthreads();
  // rounds of D steps, kQ to a chunk, the chunks in two places by turns; the
  // next chunk arrives while the waves multiply.  Whole rounds, without a branch
  // (what lies past the end is zeros): where one leaves in the middle, the compiler's
  // waits count the fewest loads of any way, and two steps of weights are in flight
  // and not four (8192 -> 16384, us: 112 sequences 60.7 -> 58.1, 250 97.4 -> 95.0; 200
  // lose 2%, 84.1 -> 86.0).
  constexpr int kPhases = D / kQ;
  constexpr int kPlaces = kPhases % 2 == 0 ? 1 : 2;  // rounds until the places repeat
  for (int q1 = 0; q1 < steps; q1 += kPlaces * D) {
#pragma unroll
    for (int ph = 0; ph < kPlaces * kPhases; ++ph) {
      const int q0 = q1 + ph * kQ;
      const int place = ph & 1, slot = ph % kPhases * kQ;
      const unsigned char* from = lds + place * kChunk;
      issue_chunk(q0 + kQ, lds + (place ^ 1) * kChunk);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int q = 0; q < kQ; ++q) {
        // (steps past the end multiply zeros)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          u32x4 xb[NT];
#pragma unroll
          for (int c = 0; c < NT; ++c) xb[c] = *reinterpret_cast<const u32x4*>(from + q * kSlot + c * 2048 + (frag0 ^ (m * 64)));
#pragma unroll
          for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int r = 0; r < RT; ++r)
              acc[r][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wa[slot + q][r][m]),
                                                                  __builtin_bit_cast(bf16x8, xb[c]), acc[r][c], 0, 0, 0);
        }
        issue_w(slot + q, q0 + q + D);
        __builtin_amdgcn_sched_barrier(0);
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(wait_loads(2 * RT * kQ));  // all but the loads after the chunk's
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
  }

  if (a.splits > 1) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int t = tile_of(r);
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        const int b = 16 * c + col;
        if (b < a.batch && t < tiles)
          *reinterpret_cast<f32x4*>(a.y + (static_cast<int64_t>(sp) * a.batch + b) * a.n + 16 * t + 4 * kblk) = acc[r][c];
      }
    }
    return;
  }
  // The sums go through LDS, [sequence][row of the workgroup] in fp32, so that
  // eight features a thread are written in one loop: straight from the products'
  // registers, 8 bytes a lane, 2048 -> 57344 with 250 sequences took 98 us, so 85
  // (and 71 with one branch for the eight activations).  The sums of parts, 16
  // bytes a lane, gain nothing from it (they lose 3%).
  constexpr int kRow = W * RT * 64;  // bytes of a sequence
  constexpr int kFit = 2 * kChunk / (16 * kRow);
  constexpr int kPass = kFit < NT ? kFit : NT;  // column tiles at a time
  static_assert(kPass >= 1, "a column tile fits in the chunks");
  // 16-byte pieces, by turns so that neither way meets in a bank
  auto at = [&](int row, int piece) __attribute__((always_inline)) {
    return reinterpret_cast<f32x4*>(lds + row * kRow + ((piece ^ (row & 7)) * 16));
  };
  const int tid = threadIdx.x;
#pragma unroll
  for (int c0 = 0; c0 < NT; c0 += kPass) {
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int c = 0; c < kPass; ++c)
        if (c0 + c < NT) *at(16 * c + col, (wv * RT + r) * 4 + kblk) = acc[r][c0 + c];
    __syncthreads();
    const int last = a.batch - 16 * c0 < 16 * kPass ? a.batch - 16 * c0 : 16 * kPass;
    constexpr int kEach = kGated ? 2 * W : 4 * W;  // threads a sequence, 8 features each
    const int q = tid % kEach, n = rg * (8 * kEach) + 8 * q;
    if (n >= e.features) continue;
    const int piece = kGated ? (q >> 1) * 8 + (q & 1) * 2 : 2 * q;
    uint32_t bias[4] = {0u, 0u, 0u, 0u}, bias_up[4] = {0u, 0u, 0u, 0u};
    if (e.bias) {
      load_bf16<8>(e.bias + n, bias);
      if constexpr (kGated) load_bf16<8>(e.bias + e.features + n, bias_up);
    }
    for (int row = tid / kEach; row < last; row += W * 64 / kEach) {
      const int64_t o = static_cast<int64_t>(16 * c0 + row) * e.features + n;
      uint32_t res[4];
      if (e.residual) load_bf16<8>(e.residual + o, res);
      const f32x4 y[2] = {*at(row, piece), *at(row, piece + 1)};
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = y[j / 4][j % 4] + unpack_bf16(bias, j);
      activate(v, e.activation);
      if constexpr (kGated) {
        const f32x4 up[2] = {*at(row, piece + 4), *at(row, piece + 5)};
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= up[j / 4][j % 4] + unpack_bf16(bias_up, j);
      }
      if (e.residual) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += unpack_bf16(res, j);
      }
      store_features(e, o, v);
    }
  }
}

template <bool kGated, int RT, int NT, int W, int D, int kQ, int kWavesPerSimd>
hipError_t linear_stream_as(const RowsArgs& a, const LinearArgs& e, hipStream_t st) {
  auto* fn = &linear_stream_kernel<kGated, RT, NT, W, D, kQ, kWavesPerSimd>;
  constexpr int lds = 2 * kQ * NT * 2048 + 1024;
  if constexpr (lds > 64 * 1024) {
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
  const int groups = (a.n / kTileRows + RT * W - 1) / (RT * W);
  hipLaunchKernelGGL(fn, dim3(static_cast<unsigned>(groups * a.splits)), dim3(W * 64), lds, st, a, e);
  return hipGetLastError();
}

// The forms: 4 waves, two workgroups a CU, up to 128 sequences; then 8 waves
// (more rows share the activations).
constexpr int stream_waves(int batch) { return batch <= 128 ? 4 : 8; }

template <bool kGated>
hipError_t linear_stream_any(const RowsArgs& a, const LinearArgs& e, hipStream_t st) {
  const int nt = (a.batch + 15) / 16;
  if (nt <= 4) return linear_stream_as<kGated, 2, 4, 4, 4, 2, 2>(a, e, st);
  if (nt <= 5) return linear_stream_as<kGated, 2, 5, 4, 4, 2, 2>(a, e, st);
  if (nt <= 6) return linear_stream_as<kGated, 2, 6, 4, 4, 2, 2>(a, e, st);
  if (nt <= 7) return linear_stream_as<kGated, 2, 7, 4, 4, 2, 2>(a, e, st);
  if (nt <= 8) return linear_stream_as<kGated, 2, 8, 4, 4, 2, 2>(a, e, st);
  if (nt <= 10) return linear_stream_as<kGated, 2, 10, 8, 4, 2, 2>(a, e, st);
  if (nt <= 13) return linear_stream_as<kGated, 2, 13, 8, 4, 2, 2>(a, e, st);
  if (nt <= 16) return linear_stream_as<kGated, 2, 16, 8, 2, 2, 2>(a, e, st);
  return hipErrorInvalidValue;
}

int stream_groups(int waves, int rows) { return (rows / kTileRows + 2 * waves - 1) / (2 * waves); }

// Most parts of the k range: 512 rows to a CU, parts together, which bounds the
// workspace of their sums (1/2 MB a sequence); more were not the shortest anywhere.
int stream_most_splits(int waves, int rows, int num_cus) {
  const int most = 16 / waves * num_cus / stream_groups(waves, rows);
  return most < 1 ? 1 : most < kMaxStreamSplits ? most : kMaxStreamSplits;
}

// How a product of more than 32 sequences runs: by rows_kernel (0), or by
// linear_stream_kernel in so many parts of the k range, whichever these models
// of the measured times say is shorter, in us of a chip of 256 CUs.  Each joins, as
// the root of the squares, its products and the read of the weights:
//   rows_kernel: whole groups of 64 sequences at 3.6e8 outputs x k a us, the read
//     at 6.4 TB/s; 4.4, and 2.4 a million outputs of those groups.
//   here: the busiest CU's workgroups, 0.036 for 64 k of 128 rows and a column
//     tile (the weights count as 5 more), the read at 6.5 TB/s, less by the root of
//     the CUs without a workgroup; 4.7; whole, 0.12 for the epilogue of 128 rows and a
//     column tile, in parts 5.4 for the second kernel and the parts' sums, written
//     and read, at 3 MB a us.
// With weights out of every cache the models are 8% off, and the choice over 199
// products (80 to 250 sequences, k 256 to 8192, 10240 to 57344 rows) is 0.4% behind
// the best of rows_kernel and 1, 2, 3, 4 and 6 parts on average, 12% at most;
// rows_kernel always is 29% behind.  Over 105 of 36 to 64 sequences, not in parts,
// 0.3%, and 13.2% (us, rows_kernel, whole, 3 parts: 80, 256 -> 57344 30.9, 12.5, -;
// 101, 5120 -> 20480 with GELU -, 64.0, 54.5; 250, 2048 -> 28672 75.0, 62.7, 83.2, in
// two 58.8; 64, 4096 -> 20480 40.0, 44.4, 45.7).
//
// Below 40 rows a CU (10240) it is rows_kernel without a look at the models.  With k
// up to 8192 that is right (8192 rows: 0.7% behind the best over 30 products of 80 to
// 250 sequences, 1.9% over 15 of 36 to 64).  It is not just below the bound and with
// longer k, where parts are ahead, the more the longer (us, rows_kernel, best number of
// parts: 10224 rows, 4096 of k, 200 sequences 43.1, 43.0; 8192, 80 46.4, 37.4, 200 74.9,
// 62.7; 14336, 200 124, 91; 8192 rows, 14336 of k, 80 59.0, 48.1, 200 87.3, 77.8;
// 28672, 80 111, 82, 200 174, 142; 4096 rows, 14336 of k, 80 34.3, 33.3, 200 51.1,
// 69.1; 28672, 80 58.7, 52.2, 200 94.7, 115).
int stream_splits(int batch, int rows, int k, int num_cus) {
  if (batch <= 32 || rows < 40 * num_cus) return 0;
  const double scale = 256.0 / num_cus, weights = scale * rows * k, outputs = scale * rows * ((batch + 63) / 64 * 64);
  auto joined = [](double a, double b) { return std::sqrt(a * a + b * b); };
  double best = joined(outputs * k / 3.6e8, weights * 2 / 6.4e6) + 2.4e-6 * outputs + 4.4;
  int splits = 0;
  const int waves = stream_waves(batch), groups = stream_groups(waves, rows), cols = (batch + 15) / 16;
  const int most = batch <= 64 ? 1 : stream_most_splits(waves, rows, num_cus);
  for (int s = 1; s <= most; ++s) {
    const double busiest = (groups * s + num_cus - 1) / num_cus * (waves / 4);
    const double used = groups * s < num_cus ? std::sqrt(static_cast<double>(groups * s) / num_cus) : 1.0;
    const double t = joined(busiest * 0.036 * (cols + 5) * k / kPairK / s, weights * 2 / 6.5e6 / used) + 4.7 +
                     (s == 1 ? busiest * 0.12 * cols : scale * s * batch * rows * 4 / 3e6 + 5.4);
    if (t < best) best = t, splits = s;
  }
  return splits;
}

// Products with few output features (a router's) of more than 16 sequences by
// rows_kernel in small tiles, each column group with workgroups of its own: what
// bounds them is a workgroup's way through its activations and weights, not the
// chip, and the forms that take up to 64 sequences together leave most CUs idle.
// One row and one column tile a workgroup while there is a CU for each, then two
// row tiles, then two of both.  Past one round of workgroups, or where a
// workgroup's way is long, the planner's forms, which share it or split k, are
// level or ahead.  us a product, the planner's form -> these, weights cold:
//   one of each: 20 sequences, 4096 -> 256 6.8 -> 5.5, 8192 -> 512 7.9 -> 10.1;
//     200, 2048 -> 256 9.1 -> 4.7, 14336 -> 256 19.7 -> 16.9;
//   two row tiles: 24, 4096 -> 2560 8.1 -> 9.1; 64, 4096 -> 2048 11.7 -> 9.3; 128,
//     8192 -> 1024 16.4 -> 14.4, 14336 -> 1024 19.9 -> 22.8;
//   two of both: 40, 4096 -> 4096 12.3 -> 11.4, -> 4640 (304 workgroups) 14.2 ->
//     17.0; 128, 4096 -> 2048 16.2 -> 12.0; 64, 8192 -> 4096 21.5 -> 23.1.
bool few_rows_plan(int batch, int rows, int k, int num_cus, bool gated, RowsPlan* out) {
  const int cols = (batch + 15) / 16, tiles = rows / kTileRows;
  if (cols < 2) return false;
  const int64_t ones = static_cast<int64_t>(tiles) * cols, pairs = static_cast<int64_t>((tiles + 1) / 2) * cols;
  RowsPlan p{};
  p.rt = !gated && ones <= num_cus ? 1 : 2;
  p.bt = pairs <= num_cus ? 1 : 2;
  if (cols <= p.bt || pairs > 2 * num_cus) return false;
  if (cols == 2 && (p.rt == 2 || k > 6144)) return false;
  if (p.rt == 2 && k > (p.bt == 1 ? 8192 : 4096)) return false;
  p.waves = 8;
  p.kb = 2;
  p.fused = true;
  p.row_groups = (tiles + p.rt - 1) / p.rt;
  p.col_groups = (cols + p.bt - 1) / p.bt;
  p.splits = 1;
  p.split_grid = p.grid = (p.row_groups + 7) / 8 * 8 * p.col_groups;
  if (p.grid > num_cus) return false;
  *out = p;
  return true;
}

}  // namespace

RowsPlan plan_linear(int batch, int rows, int k, int num_cus, bool gated) {
  RowsPlan few;
  if (few_rows_plan(batch, rows, k, num_cus, gated, &few)) return few;
  const int splits = stream_splits(batch, rows, k, num_cus);
  if (!splits) return plan_rows(batch, rows, k, num_cus, gated ? Fusable::kPairs : Fusable::kAny, kMaxRowsSplits);
  RowsPlan p{};
  p.stream = true;
  p.waves = stream_waves(batch);
  p.rt = 2 * p.waves;
  p.bt = (batch + 15) / 16;
  p.row_groups = stream_groups(p.waves, rows);
  p.col_groups = 1;
  p.splits = splits;
  p.split_grid = p.row_groups;
  p.grid = p.row_groups * p.splits;
  p.fused = p.splits == 1;
  return p;
}

int64_t linear_most_floats(int batch, int rows, int num_cus) {
  int64_t most = rows_most_floats(batch, rows, num_cus, kMaxRowsSplits);
  if (batch <= 64) return most;  // (streamed whole)
  for (const int b : {batch < 128 ? batch : 128, batch}) {
    const int splits = stream_most_splits(stream_waves(b), rows, num_cus);
    const int64_t n = splits > 1 ? static_cast<int64_t>(splits) * b * rows : 0;
    most = n > most ? n : most;
  }
  return most;
}

hipError_t launch_linear(const RowsArgs& args, const RowsPlan& p, const LinearArgs& e, bool gated, hipStream_t st) {
  RowsArgs a = args;
  hipError_t err;
  if (p.stream) {
    a.splits = p.splits;
    err = gated ? linear_stream_any<true>(a, e, st) : linear_stream_any<false>(a, e, st);
  } else {
    err = p.fused ? launch_rows_linear(a, p, e, gated, st) : launch_rows(a, p, st);
  }
  if (err != hipSuccess || p.fused) return err;
  return launch_linear_epilogue(e, a.y, p.splits, a.batch, gated, st);
}

}  // namespace pda
