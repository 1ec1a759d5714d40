// C-ABI host side of the paged decode attention library: argument checks
// (before any HIP call), the split planner, per-(device, stream) workspaces
// and optional event timing.  The kernels live in pda_kernels.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>
#include <map>
#include <mutex>
#include <string>
#include <utility>
#include <vector>

#include "pda.h"
#include "pda_append.h"
#include "pda_ffn.h"
#include "pda_probe.h"
#include "pda_gemv.h"
#include "pda_internal.h"
#include "pda_kv4.h"
#include "pda_pages.h"

namespace {

thread_local std::string g_err;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

int hip_fail(hipError_t e, const char* what) {
  return fail(PDA_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

int env_int(const char* name, int dflt, int lo, int hi) {
  const char* s = std::getenv(name);
  if (!s || !*s) return dflt;
  long v = std::strtol(s, nullptr, 10);
  if (v < lo) v = lo;
  if (v > hi) v = hi;
  return static_cast<int>(v);
}

// Tunables of the planner: defaults, environment overrides, pda_set_option.
constexpr int kMaxBlocksPerCu = 8;
constexpr int kMaxMinSteps = 1 << 30;
std::atomic<int> g_blocks_per_cu{-1};
std::atomic<int> g_min_steps{-1};
std::atomic<int> g_compute_path{-1};
std::atomic<int> g_fused_merge{-1};
std::atomic<int> g_kv_group{-1};
std::atomic<int> g_fixed_split{-1};

int blocks_per_cu() {
  int v = g_blocks_per_cu.load();
  if (v < 0) {
    v = env_int("PDA_BLOCKS_PER_CU", 1, 1, kMaxBlocksPerCu);
    g_blocks_per_cu.store(v);
  }
  return v;
}
// Fewest 32-token steps per wave the caller fixed (0 = the planner's choice).
int min_steps_option() {
  int v = g_min_steps.load();
  if (v < 0) {
    v = env_int("PDA_MIN_STEPS", 0, 0, kMaxMinSteps);
    g_min_steps.store(v);
  }
  return v;
}

int compute_path() {
  int v = g_compute_path.load();
  if (v < 0) {
    v = env_int("PDA_COMPUTE_PATH", 0, 0, 1);
    g_compute_path.store(v);
  }
  return v;
}

int fused_merge() {
  int v = g_fused_merge.load();
  if (v < 0) {
    v = env_int("PDA_FUSED_MERGE", 0, 0, 2);
    g_fused_merge.store(v);
  }
  return v;
}

// Most kv heads one attention workgroup reads together (0 = the plan's own choice).
int kv_group_cap() {
  int v = g_kv_group.load();
  if (v < 0) {
    v = env_int("PDA_KV_GROUP", 0, 0, pda::kMaxWaves);
    g_kv_group.store(v);
  }
  return v;
}

// 1 (default): latency-bound calls take the fixed split; 0: every call
// takes the stream-K split.
int fixed_split() {
  int v = g_fixed_split.load();
  if (v < 0) {
    v = env_int("PDA_FIXED_SPLIT", 1, 0, 1);
    g_fixed_split.store(v);
  }
  return v;
}

bool is_pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
int log2i(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

int check_shape(int32_t batch, int32_t hq, int32_t hkv, int32_t d, int32_t p, int32_t maxp) {
  if (batch < 0) return fail(PDA_ERR_SHAPE, "batch must be >= 0 (got %d)", batch);
  if (hq <= 0 || hkv <= 0) return fail(PDA_ERR_SHAPE, "head counts must be positive (q %d, kv %d)", hq, hkv);
  if (hq % hkv) return fail(PDA_ERR_SHAPE, "num_q_heads %d is not a multiple of num_kv_heads %d", hq, hkv);
  if (hkv > PDA_MAX_KV_HEADS)
    return fail(PDA_ERR_UNSUPPORTED, "num_kv_heads %d exceeds %d", hkv, PDA_MAX_KV_HEADS);
  if (hq / hkv > PDA_MAX_GROUP)
    return fail(PDA_ERR_UNSUPPORTED, "query group %d exceeds %d", hq / hkv, PDA_MAX_GROUP);
  if (d != 64 && d != 128 && d != 256) return fail(PDA_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128, 256)", d);
  if (p <= 0 || maxp <= 0) return fail(PDA_ERR_SHAPE, "page_size and max_pages_per_seq must be positive");
  if (!is_pow2(p) || p > PDA_MAX_PAGE_SIZE)
    return fail(PDA_ERR_UNSUPPORTED, "page_size %d (supported: powers of two up to %d)", p, PDA_MAX_PAGE_SIZE);
  if (batch > PDA_MAX_BATCH) return fail(PDA_ERR_UNSUPPORTED, "batch %d exceeds %d", batch, PDA_MAX_BATCH);
  const int64_t max_ctx = static_cast<int64_t>(maxp) * p;
  if (max_ctx > (int64_t{1} << 30)) return fail(PDA_ERR_SHAPE, "max_pages_per_seq * page_size too large");
  const int64_t steps = static_cast<int64_t>(batch) * ((max_ctx + pda::kStep - 1) / pda::kStep);
  if (steps >= (int64_t{1} << 31))
    return fail(PDA_ERR_UNSUPPORTED, "batch * max context exceeds 2^36 tokens");
  return PDA_OK;
}

// Attention-only limits on top of check_shape.
int check_attention(int32_t batch, int32_t hq, int32_t hkv, int32_t d, int32_t p, int32_t maxp) {
  int rc = check_shape(batch, hq, hkv, d, p, maxp);
  if (rc) return rc;
  if (d == 256 && batch > PDA_MAX_BATCH_D256)
    return fail(PDA_ERR_UNSUPPORTED, "batch %d exceeds %d at head_dim 256", batch, PDA_MAX_BATCH_D256);
  return PDA_OK;
}

// The compute path's own limits (PDA_OPT_COMPUTE_PATH): the vector-ALU
// variant takes D = 128, pages of >= 16 tokens and <= 8 columns, and its LDS
// tiles bound the batch.  *valu_cols = 0 (matrix cores) or 4 / 8.
int check_compute_path(int32_t d, int32_t p, int cols, int32_t batch, int* valu_cols) {
  *valu_cols = 0;
  if (compute_path() != 1) return PDA_OK;
  if (d != 128 || p < 16 || cols > 8)
    return fail(PDA_ERR_UNSUPPORTED,
                "the vector-ALU compute path takes head_dim 128, page_size >= 16 and at most 8 columns "
                "(got head_dim %d, page_size %d, %d columns)", d, p, cols);
  if (pda::attn_lds_bytes(d, batch, pda::max_waves(d), true) > static_cast<size_t>(pda::kMaxLdsBytes))
    return fail(PDA_ERR_UNSUPPORTED, "batch %d needs more LDS than a workgroup has on the vector-ALU path", batch);
  *valu_cols = cols <= 4 ? 4 : 8;
  return PDA_OK;
}

struct Plan {
  int grid = 0;
  int waves = 0;   // per workgroup
  int hgs = 0;     // kv heads per workgroup
  int min_steps = 0;   // fewest 32-token steps per wave
  bool fused = false;  // split sequences merged by their last workgroup
  int chunks = 0;       // > 0: fixed split, chunks per (sequence, kv-head group)
  int chunk_steps = 0;  // 32-token steps per chunk of the fixed split
  int64_t slots = 0;
  int64_t off_acc = 0, off_ml = 0, off_pref = 0, bytes = 0;
};

int64_t align256(int64_t x) { return (x + 255) & ~int64_t{255}; }

// Largest divisor of hkv that is at most max_waves: the kv heads a workgroup
// reads together from every page.
int heads_per_group(int hkv, int max_waves) {
  for (int d = max_waves; d > 1; --d)
    if (hkv % d == 0) return d;
  return 1;
}

// The same for workgroups of more than 8 waves, of which at least three in
// four should have work: 8 heads go to 12 waves as 4 heads x 3 step phases.
int heads_of_waves(int hkv, int max_waves, int most) {
  for (int d = std::min(max_waves, most); d > 1; --d)
    if (hkv % d == 0 && 4 * d * (max_waves / d) >= 3 * max_waves) return d;
  return 1;
}

// What the planner has to know of the kernel that a plan is for.
struct Form {
  int max_waves;        // waves of a workgroup at most
  int per_cu;           // workgroups of a compute unit that run together
  int64_t token_bytes;  // K and V of a token and kv head
  bool options;         // the compute path and the fused merge apply
  bool light;           // 4-bit steps: small calls by small_plan_light, whole sequences by plan_whole_light
};
Form bf16_form(int d, bool sinks = false) { return {pda::max_waves(d), 1, static_cast<int64_t>(d) * 4, !sinks, false}; }
// Workgroups of 4 waves, as many as fill a CU's registers, where their LDS (the
// tiles, and the prefix over the batch) allows it; one of all the waves, or
// what fits, where it does not.
Form kv4_form(int d, int batch) {
  int waves = 4, per_cu = pda::kv4_max_waves(d) / 4;
  if (per_cu * pda::kv4_attn_lds_bytes(d, batch, waves) > static_cast<size_t>(pda::kMaxLdsBytes)) {
    per_cu = 1;
    for (waves = pda::kv4_max_waves(d); waves > 4; waves -= 4)
      if (pda::kv4_attn_lds_bytes(d, batch, waves) <= static_cast<size_t>(pda::kMaxLdsBytes)) break;
  }
  return {waves, per_cu, static_cast<int64_t>(d) * 17 / 16, false, true};
}

// Workgroups: one wave per kv head of a group of hgs, times step phases up
// to max_waves waves (8; 4 at D = 256); as many workgroups as fill the
// device (blocks_per_cu per CU), but none with fewer than min_steps 32-token
// steps per wave when every sequence has steps_seq steps.  Partial
// slots: one per (workgroup, sequence piece), at most grid + batch * kv-head
// groups, each holding `cols` (query token, head) rows per kv head.
Plan plan_for(const Form& form, int hgs, int32_t batch, int32_t hkv, int32_t d, int64_t steps_seq, int num_cus,
              int cols, int min_steps) {
  Plan pl;
  const int max_waves = form.max_waves;
  pl.hgs = hgs;
  pl.min_steps = min_steps;
  const int phases = max_waves / pl.hgs;
  pl.waves = pl.hgs * phases;
  const int64_t ngroups = hkv / pl.hgs;
  const int64_t steps_max = static_cast<int64_t>(batch) * ngroups * steps_seq;
  const int64_t per_block = static_cast<int64_t>(min_steps) * phases;
  int64_t blocks = (steps_max + per_block - 1) / per_block;
  const int64_t target = static_cast<int64_t>(num_cus) * blocks_per_cu() * form.per_cu;
  if (blocks > target) blocks = target;
  if (blocks < 1) blocks = 1;
  pl.grid = static_cast<int>(blocks);
  pl.slots = static_cast<int64_t>(pl.grid) + static_cast<int64_t>(batch) * ngroups;
  const int64_t rows = pl.slots * pl.hgs * cols;
  pl.off_acc = 0;
  pl.off_ml = align256(rows * d * 4);
  pl.off_pref = pl.off_ml + align256(rows * 2 * 4);
  // steps prefix [batch + 1], then the split list [grid] (see the kernels)
  pl.bytes = pl.off_pref + align256((static_cast<int64_t>(batch) + 1 + pl.grid) * 4);
  return pl;
}

// Most 32-token steps a sequence can have: what the page table holds, or with
// a sliding window the steps that window + num_queries - 1 tokens touch, and
// those of the sinks.
int64_t most_steps(int32_t p, int32_t maxp, int num_queries, int window, int sinks = 0) {
  const int64_t table = (static_cast<int64_t>(maxp) * p + pda::kStep - 1) / pda::kStep;
  if (window <= 0) return table;
  const int64_t seen = (static_cast<int64_t>(window) + num_queries - 1 + pda::kStep - 1) / pda::kStep + 1 +
                       (static_cast<int64_t>(sinks) + pda::kStep - 1) / pda::kStep;
  return std::min(table, seen);
}

// The fixed split of a latency-bound call with the kv-head grouping and
// step count of `base`: every (sequence, kv-head group) is cut into the same
// number of chunks of whole 32-token steps, as many as the stream-K plan
// would give it at the page table's largest context (but at least 2 and
// within the device's workgroups), so each workgroup knows its piece from
// its index.  Where the stream-K plan takes a single workgroup, every pair is
// one chunk: whole sequences, one workgroup each, nothing to merge.  Returns
// a plan with grid 0 where it does not apply: more pairs than half the
// device's workgroups (the stream-K split balances those better).  One
// partial slot per workgroup.
Plan plan_fixed(const Form& form, const Plan& base, int32_t batch, int32_t hkv, int32_t d, int64_t steps_seq, int num_cus,
                int cols) {
  Plan pl = base;
  pl.grid = 0;
  const int phases = pl.waves / pl.hgs;
  const int64_t seqs = static_cast<int64_t>(batch) * (hkv / pl.hgs);
  const int64_t target = static_cast<int64_t>(num_cus) * blocks_per_cu() * form.per_cu;
  const int64_t per_block = static_cast<int64_t>(pl.min_steps) * phases;
  if (base.grid < 1 || 2 * seqs > target) return pl;
  int64_t chunks = 1;
  if (base.grid > 1) {
    chunks = std::min((steps_seq + per_block - 1) / per_block, target / seqs);
    chunks = std::max<int64_t>(chunks, 1);
  }
  const int64_t chunk_steps = (steps_seq + chunks - 1) / chunks;
  chunks = (steps_seq + chunk_steps - 1) / chunk_steps;  // no chunk wholly past the largest context
  if (base.grid > 1 && chunks < 2) return pl;
  pl.grid = static_cast<int>(seqs * chunks);
  pl.chunks = static_cast<int>(chunks);
  pl.chunk_steps = static_cast<int>(chunk_steps);
  pl.slots = pl.grid;
  const int64_t rows = pl.slots * pl.hgs * cols;
  pl.off_acc = 0;
  pl.off_ml = align256(rows * d * 4);
  pl.off_pref = pl.off_ml + align256(rows * 2 * 4);
  pl.bytes = pl.off_pref + align256((static_cast<int64_t>(batch) + 1 + pl.grid) * 4);
  return pl;
}

// The split plan of a call.  The default reads all kv heads of a group of up to 8
// together (the faster access order for long streams) and merges split
// sequences in a separate kernel.  With PDA_OPT_FUSED_MERGE = 1, a grid of
// several workgroups with little partial data per sequence merges inside
// the attention kernel instead: with the largest kv-head group for which
// the most partial data one sequence can have, grid x hgs x cols x d fp32,
// fits pda::kFusedMergeBytes (a single request then takes one kv head per
// workgroup); a latency-bound call with the fixed split keeps it, its
// sequences merged by the last of their chunks (1 x 4096 tokens, 32:8
// heads: 14.0 us per call against 11.7 us with the merge kernel).  On
// MI355X the in-kernel hand-off (write-through stores, their
// acknowledgement, the arrival atomic, coherent reloads) costs more than
// the merge kernel's launch, so the option is off by default.
// Calls whose K and V (bounded by the page table) fit in this many bytes are
// latency-bound: they take the small-call rules of make_plan.
constexpr int64_t kSmallCallBytes = int64_t{128} << 20;
// Most pieces a small call cuts one (sequence, kv-head group) into.
constexpr int64_t kSmallCallPieces = 32;
constexpr int kDefaultMinSteps = 2;

// Small calls over a 4-bit cache, whose steps are a quarter of the bytes.  A
// workgroup takes the fewest kv heads with which the fixed split still applies,
// its waves as step phases that are joined in LDS.  A wave takes as many steps as
// leave a workgroup a CU, up to four, since another workgroup costs its partials
// and its place in the merge; and as many, up to four too, as leave the merge of
// a sequence 64 pieces (32 at head size 256, which are as wide).  us per call with
// 1, 2, 3, 4 steps, the taken one in brackets: 1 x 4096 tokens at 32:8 heads
// [9.0] 9.8 10.5 11.4, 1 x 8192 12.2 [10.1] 10.8 11.4, 1 x 12000 15.1 12.9 [11.0]
// 11.6, 1 x 16384 15.6 13.9 15.0 [11.8], 1 x 32768 19.0 19.0 19.0 [16.5]; for the
// merge: 1 x 12000 at 32:2 12.1 [10.7] 10.7 11.4, 1 x 32768 21.3 14.7 13.7 [13.2].
// Where a workgroup a step and group of heads fit the CUs and leave the merge no
// more than 32 pieces there is nothing to join in LDS: 1 x 1024 tokens at 32:8
// 8.6 -> 8.0, two sequences of 40 to 614 at 12:4, D = 256 10.3 -> 9.4.
constexpr int kLightMostSteps = 4;
Plan small_plan_light(const Form& form, const Plan& dflt, int32_t batch, int32_t hkv, int32_t d, int64_t steps_seq,
                      int num_cus, int cols, int cap, int ms_opt) {
  const int64_t target = static_cast<int64_t>(num_cus) * blocks_per_cu() * form.per_cu;
  int h = dflt.hgs;
  if (ms_opt == 0 && steps_seq <= 32 && steps_seq * batch * (hkv / h) <= num_cus)
    return plan_for(form, h, batch, hkv, d, steps_seq, num_cus, cols, 1);
  if (cap == 0)
    for (h = 1; h < dflt.hgs; ++h)
      if (hkv % h == 0 && 2 * static_cast<int64_t>(batch) * (hkv / h) <= target) break;
  const int phases = form.max_waves / h;
  auto per_wave = [&](int64_t steps, int64_t workgroups) {
    const int64_t n = workgroups * phases;
    return static_cast<int>(std::min<int64_t>(kLightMostSteps, (steps + n - 1) / n));
  };
  const int ms = std::max({1, per_wave(steps_seq * batch * (hkv / h), num_cus), per_wave(steps_seq, d == 256 ? 32 : 64)});
  return plan_for(form, h, batch, hkv, d, steps_seq, num_cus, cols, ms_opt > 0 ? ms_opt : ms);
}

Plan make_split_plan(const Form& form, int32_t batch, int32_t hkv, int32_t d, int64_t steps_seq, int num_cus, int cols) {
  const int cap = kv_group_cap();
  const int ms_opt = min_steps_option();
  // A split piece leaves a partial of cols x head_dim fp32 per kv head it
  // covers; with more than 8 columns (several query tokens) those writes
  // cost more than the longer token rows save, so at most 4 kv heads go
  // together (multiq: 191.4 -> 188.3 us per call; long70b and ragged, at 8
  // columns or fewer, run slower with 4).  Over a 4-bit cache, whose steps are
  // shorter beside the same partials, at most 2 (101 Zipf sequences with three
  // queries at 40:8 heads 124.5 -> 119.3, 64 x U[128, 8192] with four at 32:8 71.2
  // -> 70.2; at 4 columns 60.4 -> 63.3).
  const int dflt_most = cols > 8 ? std::min(form.light ? 2 : 4, form.max_waves) : form.max_waves;
  const int most = cap > 0 && cap < form.max_waves ? cap : dflt_most;
  const int together = form.max_waves > 8 ? heads_of_waves(hkv, form.max_waves, most) : heads_per_group(hkv, most);
  Plan dflt = plan_for(form, together, batch, hkv, d, steps_seq, num_cus, cols, ms_opt > 0 ? ms_opt : kDefaultMinSteps);
  // Small calls (each 32-token step's K and V is a few KB; the whole call
  // is a chain of latencies):
  //  - a plan that splits the work but leaves CUs idle gives each wave one
  //    step instead of two, doubling the workgroups (graph replay of 20
  //    calls over cold K/V: 1 x 1024 tokens 15.1 -> 12.5 us, 4 x 1024
  //    15.9 -> 13.6, 8 x 512 15.7 -> 13.8);
  //  - fewer kv heads per workgroup when a sequence's heads would be cut
  //    into more than kSmallCallPieces pieces: the same workgroups then take
  //    longer runs of fewer heads, so less partial data and a lighter merge
  //    (1 x 4096 tokens, 32:8 heads, 15.6 -> 14.4 us with 2 heads per
  //    workgroup; 1 x 16384 25.1 -> 21.9 with 1; 1 x 8192, 64:8 heads,
  //    20.7 -> 16.8 with 1).  Large calls keep 8 heads, whose 2 KB token
  //    rows stream faster (long70b: 319.8 us per call with 8, 321.2 with 4,
  //    329.6 with 2, 351.8 with 1).
  //  - the fixed split (plan_fixed) unless PDA_OPT_FIXED_SPLIT is 0: the
  //    first K/V loads leave ~2 us earlier and the merge needs no prefix
  //    (1 x 4096 tokens, 32:8 heads, cold K/V: attention kernel 14.8 ->
  //    11.4 us by events, 16.7 -> 11.9 us per call replayed from a graph).
  const int64_t kv_bytes = static_cast<int64_t>(batch) * steps_seq * pda::kStep * hkv * form.token_bytes;
  const bool small = kv_bytes <= kSmallCallBytes;
  if (small && form.light) {
    dflt = small_plan_light(form, dflt, batch, hkv, d, steps_seq, num_cus, cols, cap, ms_opt);
  } else if (small) {
    if (ms_opt == 0 && dflt.grid > 1 && dflt.grid < static_cast<int64_t>(num_cus) * blocks_per_cu() * form.per_cu)
      dflt = plan_for(form, dflt.hgs, batch, hkv, d, steps_seq, num_cus, cols, 1);
    if (cap == 0) {
      for (int h = dflt.hgs; h >= 1; --h) {
        if (hkv % h) continue;
        if (h == 1 || static_cast<int64_t>(dflt.grid) * h <= kSmallCallPieces * batch * hkv) {
          if (h != dflt.hgs) dflt = plan_for(form, h, batch, hkv, d, steps_seq, num_cus, cols, dflt.min_steps);
          break;
        }
      }
    }
  }
  // (the vector-ALU variant, a measurement aid, keeps the merge kernel)
  if (dflt.grid == 1 || !form.options || !fused_merge() || compute_path() != 0) {
    if (small && fixed_split() && (!form.options || compute_path() == 0)) {
      const Plan f = plan_fixed(form, dflt, batch, hkv, d, steps_seq, num_cus, cols);
      if (f.grid > 0) return f;
    }
    return dflt;
  }
  // a latency-bound call keeps the fixed split, merged in the kernel
  if (small && fixed_split()) {
    Plan f = plan_fixed(form, dflt, batch, hkv, d, steps_seq, num_cus, cols);
    if (f.grid > 1 && f.chunks > 1 && f.grid <= pda::kMaxFusedGrid) {
      f.fused = true;
      return f;
    }
  }
  if (fused_merge() == 2) {  // every plan that has something to merge (tests)
    Plan c = dflt;
    c.fused = c.grid <= pda::kMaxFusedGrid && c.bytes < (int64_t{1} << 31);
    return c;
  }
  for (int h = dflt.hgs; h >= 1; --h) {
    if (hkv % h) continue;
    Plan c = plan_for(form, h, batch, hkv, d, steps_seq, num_cus, cols, dflt.min_steps);
    const int64_t most_bytes = static_cast<int64_t>(c.grid) * h * cols * d * 4;
    if (c.grid > 1 && c.grid <= pda::kMaxFusedGrid && most_bytes <= pda::kFusedMergeBytes &&
        c.bytes < (int64_t{1} << 31)) {
      c.fused = true;
      return c;
    }
  }
  return dflt;
}

// A workgroup for h kv heads of each sequence.
Plan whole_of(const Form& form, Plan pl, int h, int32_t batch, int32_t hkv, int64_t steps_seq) {
  pl.hgs = h;
  pl.waves = h * (form.max_waves / h);
  pl.grid = static_cast<int>(static_cast<int64_t>(batch) * (hkv / h));
  pl.chunks = 1;
  pl.chunk_steps = static_cast<int>(steps_seq);
  pl.fused = false;
  return pl;  // (the split plan's workspace, unused, is kept: the same calls fit the same scratch)
}

// Whole sequences, one workgroup per (sequence, kv-head group) and nothing to
// merge, for calls whose sequences are all short: the fewest kv heads a
// workgroup that give every pair a CU of its own.  It is the fixed split with
// one chunk per pair.  Taken where even the longest sequence the table (or
// the window) allows ends before a split plan's merge would: a workgroup
// takes about 6 us + its K/V bytes at 42 KB/us, a split plan at least 9 us
// (its merge kernel and boundary are 4 of them), and 13 where the pairs are
// too many for the fixed split, since its workgroups then take several
// sequences one after another.  Replayed from a graph over cold K/V, split ->
// whole: 16 x 160 tokens, 32:8 heads 10.5 -> 8.2 us; 64 x 64 10.9 -> 8.5; 256
// x 64 19.9 -> 14.7; 32:2 heads, 128 x 64 17.9 -> 7.8, 256 x 256 22.3 ->
// 15.9.  With longer sequences a few long ones among short ones would cost
// more whole.
Plan plan_whole(const Form& form, const Plan& split, int32_t batch, int32_t hkv, int64_t steps_seq, int num_cus) {
  Plan pl = split;
  pl.grid = 0;
  const int max_waves = form.max_waves;
  const bool streamed = 2 * static_cast<int64_t>(batch) * (hkv / heads_per_group(hkv, max_waves)) > num_cus;
  const int64_t most_kb = streamed ? 300 : 150;
  for (int h = 1; h <= max_waves; ++h) {
    if (hkv % h || static_cast<int64_t>(batch) * (hkv / h) > num_cus) continue;
    if (steps_seq * pda::kStep * h * form.token_bytes > most_kb * 1024) break;
    return whole_of(form, split, h, batch, hkv, steps_seq);
  }
  return pl;
}

// The same over a 4-bit cache, by the steps of a wave: up to four (two at head
// size 256) where the device has room for a split, up to eight where the heads of
// the batch alone are three in eight of its CUs (more than half at head size 256);
// a workgroup a CU if that holds them, else as many as run together.  us per call, split -> whole: 1 x 256
// tokens at 32:8 heads 8.2 -> 6.4, 1 x 512 8.1 -> 8.1, 1 x 1024 8.6 -> 11.4;
// 64 x 512 15.1 -> 12.0, 64 x 1024 21.9 -> 18.1, 150 x 500 25.8 -> 21.9, 256 x 256
// 29.1 -> 16.4; 12:4, D = 256, 16 x 256 10.4 -> 9.2, 16 x 512 10.8 -> 12.0, 24 x
// 1000 14.6 -> 17.2, 64 x 1024 22.9 -> 18.7.
Plan plan_whole_light(const Form& form, const Plan& split, int32_t batch, int32_t hkv, int32_t d, int64_t steps_seq,
                      int num_cus) {
  const int64_t pairs = static_cast<int64_t>(batch) * hkv;
  const bool many = d == 256 ? 2 * pairs > num_cus : 8 * pairs >= 3 * static_cast<int64_t>(num_cus);
  const int most = many ? 8 : d == 256 ? 2 : 4;
  for (const int64_t room : {static_cast<int64_t>(num_cus), static_cast<int64_t>(num_cus) * form.per_cu})
    for (int h = 1; h <= form.max_waves; ++h) {
      if (hkv % h || pairs / h > room) continue;
      if (steps_seq > most * (form.max_waves / h)) break;
      return whole_of(form, split, h, batch, hkv, steps_seq);
    }
  Plan none = split;
  none.grid = 0;
  return none;
}

// The plan of a call: the split plan, or whole sequences where that is
// faster, unless an option asks for a particular split.
Plan make_plan(const Form& form, int32_t batch, int32_t hkv, int32_t d, int64_t steps_seq, int num_cus, int cols) {
  const Plan split = make_split_plan(form, batch, hkv, d, steps_seq, num_cus, cols);
  if (split.chunks == 1 || !fixed_split() || (form.options && (compute_path() != 0 || fused_merge())) || kv_group_cap() ||
      min_steps_option() || blocks_per_cu() != 1)
    return split;
  const Plan whole = form.light ? plan_whole_light(form, split, batch, hkv, d, steps_seq, num_cus)
                                : plan_whole(form, split, batch, hkv, steps_seq, num_cus);
  return whole.grid > 0 ? whole : split;
}

// Workspace that any plan of these sizes may need, and of any smaller batch or
// table, fewer columns and every window: what a call asks for, so that calls
// of one shape that plan differently (by their windows) use one workspace,
// also under capture.  A plan has at most per_cu workgroups per compute unit and
// one per (sequence, kv head, step), each with one slot of up to max_waves kv
// heads beside one per (sequence, kv-head group).  (A 4-bit plan of a batch of
// thousands may have up to 4 waves a compute unit fewer than that of a smaller
// one: those rows are in the quarter that workspace_for adds.)
int64_t workspace_bytes(const Form& form, int32_t batch, int32_t hkv, int32_t d, int32_t p, int32_t maxp, int num_cus,
                        int cols) {
  const int64_t target = static_cast<int64_t>(num_cus) * blocks_per_cu() * form.per_cu;
  const int64_t pairs = static_cast<int64_t>(batch) * hkv;
  const int64_t steps = pairs * most_steps(p, maxp, 1, 0);
  const int64_t rows = (std::min(target * form.max_waves, steps) + pairs) * cols;
  return align256(rows * d * 4) + align256(rows * 2 * 4) + align256((batch + 1 + std::min(target, steps)) * 4);
}

int device_cus(int dev, int* cus) {
  static std::mutex mu;
  static std::map<int, int> cache;
  std::lock_guard<std::mutex> lock(mu);
  auto it = cache.find(dev);
  if (it != cache.end()) {
    *cus = it->second;
    return PDA_OK;
  }
  int n = 0;
  hipError_t e = hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return hip_fail(e, "hipDeviceGetAttribute(multiprocessor count)");
  cache[dev] = n;
  *cus = n;
  return PDA_OK;
}

// ---------------------------------------------------------------- workspaces
// Per (device, stream): one buffer for split partials and the steps prefix.
struct Workspace {
  void* ptr = nullptr;
  int64_t bytes = 0;
  int32_t* cnt = nullptr;  // arrival counters of the fused merge, zero between calls
  std::vector<void*> outgrown;  // smaller buffers that captured graphs may hold
};
std::mutex g_ws_mu;
std::map<std::pair<int, hipStream_t>, Workspace> g_ws;

// A buffer of at least `least` bytes, which this call writes.  One that has to
// grow takes `most` bytes (and a quarter), what every call that `most` covers
// writes; one that holds `least` alone grows to that as well, so that those
// calls can be captured later, but early: not while the stream is being
// captured, not where it cannot, and keeping the old buffer, which a graph
// captured before may write to, until pda_release_workspaces.  (Each buffer is
// at least 5/4 of the one before: four times the last one are kept at most.)
int workspace_for(int dev, hipStream_t st, int64_t least, int64_t most, void** out) {
  most = std::max(most, least);  // never less than this call writes, whatever its caller worked out
  std::lock_guard<std::mutex> lock(g_ws_mu);
  Workspace& ws = g_ws[{dev, st}];
  *out = ws.ptr;
  if (ws.bytes >= most) return PDA_OK;
  const bool fits = ws.bytes >= least;
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  hipError_t e = hipStreamIsCapturing(st, &cap);
  if (fits && (e != hipSuccess || cap != hipStreamCaptureStatusNone)) {
    if (e != hipSuccess) (void)hipGetLastError();
    return PDA_OK;
  }
  if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
  if (cap != hipStreamCaptureStatusNone)
    return fail(PDA_ERR_HIP, "workspace must grow to %lld bytes while the stream is being captured; "
                "call pda_workspace_reserve before capture", static_cast<long long>(most));
  const int64_t grow = most + most / 4;
  if (fits) {
    // another thread's capture must not see this allocation
    hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
    if (hipThreadExchangeStreamCaptureMode(&mode) != hipSuccess) {
      (void)hipGetLastError();
      return PDA_OK;
    }
    void* p = nullptr;
    e = hipMalloc(&p, static_cast<size_t>(grow));
    (void)hipThreadExchangeStreamCaptureMode(&mode);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return PDA_OK;
    }
    if (ws.ptr) ws.outgrown.push_back(ws.ptr);
    *out = ws.ptr = p;
    ws.bytes = grow;
    return PDA_OK;
  }
  if (ws.ptr) {
    e = hipStreamSynchronize(st);  // in-flight calls may still use the old buffer
    if (e != hipSuccess) return hip_fail(e, "hipStreamSynchronize");
    if ((e = hipFree(ws.ptr)) != hipSuccess) return hip_fail(e, "hipFree");
    ws.ptr = nullptr;
    ws.bytes = 0;
  }
  if ((e = hipMalloc(&ws.ptr, static_cast<size_t>(grow))) != hipSuccess) {
    ws.ptr = nullptr;
    return hip_fail(e, "hipMalloc(workspace)");
  }
  ws.bytes = grow;
  *out = ws.ptr;
  return PDA_OK;
}

// The fused merge's arrival counters of (device, stream): a buffer of their
// own (the GEMV calls share the workspace), cleared once when allocated;
// every call leaves them at zero.
int counters_for(int dev, hipStream_t st, int32_t** out) {
  std::lock_guard<std::mutex> lock(g_ws_mu);
  Workspace& ws = g_ws[{dev, st}];
  if (!ws.cnt) {
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    hipError_t e = hipStreamIsCapturing(st, &cap);
    if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
    if (cap != hipStreamCaptureStatusNone)
      return fail(PDA_ERR_HIP, "the merge counters must be allocated while the stream is being captured; "
                  "call pda_workspace_reserve before capture");
    void* p = nullptr;
    const size_t bytes = static_cast<size_t>(pda::kMaxFusedGrid) * sizeof(int32_t);
    if ((e = hipMalloc(&p, bytes)) != hipSuccess) return hip_fail(e, "hipMalloc(merge counters)");
    if ((e = hipMemsetAsync(p, 0, bytes, st)) != hipSuccess) {
      (void)hipFree(p);
      return hip_fail(e, "hipMemsetAsync(merge counters)");
    }
    ws.cnt = static_cast<int32_t*>(p);
  }
  *out = ws.cnt;
  return PDA_OK;
}

// ---------------------------------------------------------------- profiling
// Events around the two kernels of a call: kind 0 is attention (split,
// merge), kind 1 the prelude (GEMV, epilogue), kind 2 o_proj (GEMV, epilogue).
struct Rec {
  hipEvent_t a, b, c;
  int kind;
};
std::mutex g_prof_mu;
bool g_prof_on = false;
std::vector<Rec> g_prof_recs;
std::vector<hipEvent_t> g_prof_pool;

hipEvent_t prof_event() {
  if (!g_prof_pool.empty()) {
    hipEvent_t e = g_prof_pool.back();
    g_prof_pool.pop_back();
    return e;
  }
  hipEvent_t e = nullptr;
  if (hipEventCreate(&e) != hipSuccess) return nullptr;
  return e;
}

// A record with three events when profiling is on, else one with none.
Rec prof_begin(int kind) {
  std::lock_guard<std::mutex> lock(g_prof_mu);
  if (!g_prof_on) return Rec{nullptr, nullptr, nullptr, kind};
  Rec r{prof_event(), prof_event(), prof_event(), kind};
  if (!r.a || !r.b || !r.c) return Rec{nullptr, nullptr, nullptr, kind};
  return r;
}

void prof_push(const Rec& r) {
  std::lock_guard<std::mutex> lock(g_prof_mu);
  g_prof_recs.push_back(r);
}

// Sum the two intervals of every record of `kind`, release them.
int prof_read(int kind, double* first_ms, double* second_ms, int64_t* calls) {
  std::lock_guard<std::mutex> lock(g_prof_mu);
  double s = 0, m = 0;
  int64_t n = 0;
  int rc = PDA_OK;
  std::vector<Rec> keep;
  for (const Rec& r : g_prof_recs) {
    if (r.kind != kind) {
      keep.push_back(r);
      continue;
    }
    float t1 = 0, t2 = 0;
    hipError_t e = hipEventSynchronize(r.c);
    if (e == hipSuccess) e = hipEventElapsedTime(&t1, r.a, r.b);
    if (e == hipSuccess) e = hipEventElapsedTime(&t2, r.b, r.c);
    if (e != hipSuccess) rc = hip_fail(e, "reading profile events");
    s += t1;
    m += t2;
    ++n;
    g_prof_pool.push_back(r.a);
    g_prof_pool.push_back(r.b);
    g_prof_pool.push_back(r.c);
  }
  g_prof_recs.swap(keep);
  *first_ms = s;
  *second_ms = m;
  *calls = n;
  return rc;
}

// ---------------------------------------------------------------- validation
// The tokens of a sequence that a call touches: all of them, what its queries
// see under a window with sinks, or the last so many (an append, a read back).
struct Touched {
  int32_t num_queries = 1, window = 0, sinks = 0;
  int32_t tokens = 0;  // > 0: the last so many
  // Of a sequence of `len` tokens: [0, pinned) and [first, len).
  void of(int64_t len, int64_t* pinned, int64_t* first) const {
    const int64_t before = tokens > 0 ? len - tokens : window > 0 ? len - num_queries + 1 - window : 0;
    *first = std::max<int64_t>(before, 0);
    *pinned = tokens > 0 ? 0 : std::min<int64_t>(sinks, *first);
  }
};

// Host-side check of the device page tables and lengths (debugging aid):
// synchronises the stream and copies both to the host.  Pages without a
// touched token may have been released: any entry.
int validate_paging(const int32_t* block_table, const int32_t* context_lens, int32_t batch, int32_t maxp,
                    int32_t page_size, int32_t num_pages, const Touched& touched, hipStream_t st) {
  std::vector<int32_t> lens(batch), bt(static_cast<size_t>(batch) * maxp);
  hipError_t e = hipMemcpyAsync(lens.data(), context_lens, lens.size() * 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess)
    e = hipMemcpyAsync(bt.data(), block_table, bt.size() * 4, hipMemcpyDeviceToHost, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return hip_fail(e, "reading block_table / context_lens for validation");
  const int64_t max_ctx = static_cast<int64_t>(maxp) * page_size;
  for (int32_t b = 0; b < batch; ++b) {
    if (lens[b] < 0 || lens[b] > max_ctx)
      return fail(PDA_ERR_SHAPE, "context_lens[%d] = %d outside [0, %lld]", b, lens[b],
                  static_cast<long long>(max_ctx));
    int64_t pinned, first;
    touched.of(lens[b], &pinned, &first);
    const int32_t pages = (lens[b] + page_size - 1) / page_size;
    for (int32_t j = 0; j < pages; ++j) {
      const int64_t t = static_cast<int64_t>(j) * page_size;
      if (t >= pinned && t + page_size <= first) continue;
      const int32_t id = bt[static_cast<size_t>(b) * maxp + j];
      if (id < 0 || id >= num_pages)
        return fail(PDA_ERR_SHAPE, "block_table[%d][%d] = %d outside [0, %d)", b, j, id, num_pages);
    }
  }
  return PDA_OK;
}

// PDA_DEBUG_VALIDATE=1: check the paging inputs before every attention or
// append call (skipped while the stream is being captured).
bool debug_validate() {
  static const bool on = env_int("PDA_DEBUG_VALIDATE", 0, 0, 1) == 1;
  return on;
}

int maybe_validate(const int32_t* block_table, const int32_t* context_lens, int32_t batch, int32_t maxp,
                   int32_t page_size, int32_t num_pages, const Touched& touched, hipStream_t st) {
  if (!debug_validate()) return PDA_OK;
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(st, &cap) != hipSuccess || cap != hipStreamCaptureStatusNone) return PDA_OK;
  return validate_paging(block_table, context_lens, batch, maxp, page_size, num_pages, touched, st);
}

Touched last_tokens(int32_t n) {
  Touched t;
  t.tokens = n;
  return t;
}

// ---------------------------------------------------------------- descriptors
const char* dtype_name(int32_t dt) {
  switch (dt) {
    case PDA_DTYPE_BF16: return "bf16";
    case PDA_DTYPE_F16: return "fp16";
    case PDA_DTYPE_F32: return "fp32";
    case PDA_DTYPE_I32: return "int32";
    case PDA_DTYPE_I64: return "int64";
    default: return "unknown";
  }
}

// Rank and extents of one descriptor (not NULL).
int check_rank(const pda_tensor& t, const char* name, int32_t ndim) {
  if (t.ndim != ndim) return fail(PDA_ERR_SHAPE, "%s: %d dimensions, expected %d", name, t.ndim, ndim);
  for (int i = 0; i < ndim; ++i)
    if (t.shape[i] < 0 || t.shape[i] > INT32_MAX)
      return fail(PDA_ERR_SHAPE, "%s: extent %lld of dimension %d out of range", name,
                  static_cast<long long>(t.shape[i]), i);
  return PDA_OK;
}

bool desc_empty(const pda_tensor& t) {
  for (int i = 0; i < t.ndim; ++i)
    if (t.shape[i] == 0) return true;
  return false;
}

// Dense row-major strides (extent-1 dimensions and empty tensors excepted).
int check_dense(const pda_tensor& t, const char* name) {
  if (desc_empty(t)) return PDA_OK;
  int64_t want = 1;
  for (int i = t.ndim - 1; i >= 0; --i) {
    if (t.shape[i] != 1 && t.stride[i] != want)
      return fail(PDA_ERR_LAYOUT, "%s: stride %lld in dimension %d, a dense row-major tensor has %lld", name,
                  static_cast<long long>(t.stride[i]), i, static_cast<long long>(want));
    if (want > (int64_t{1} << 50) / (t.shape[i] > 0 ? t.shape[i] : 1))
      return fail(PDA_ERR_SHAPE, "%s: too many elements", name);
    want *= t.shape[i];
  }
  return PDA_OK;
}

// ---------------------------------------------------------------- prelude
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int check_prelude(const pda_prelude_dims* dm) {
  if (!dm) return fail(PDA_ERR_NULL, "dims is NULL");
  const pda_prelude_dims& d = *dm;
  if (d.batch < 0) return fail(PDA_ERR_SHAPE, "batch must be >= 0 (got %d)", d.batch);
  if (d.batch > pda::kMaxGemvBatch)
    return fail(PDA_ERR_UNSUPPORTED, "prelude batch %d exceeds %d", d.batch, pda::kMaxGemvBatch);
  if (d.hidden <= 0 || d.num_q_heads <= 0 || d.num_kv_heads <= 0)
    return fail(PDA_ERR_SHAPE, "hidden and head counts must be positive");
  if (d.hidden % pda::kTileK || d.hidden > 65536)
    return fail(PDA_ERR_UNSUPPORTED, "hidden %d (supported: multiples of 32 up to 65536)", d.hidden);
  if (d.num_q_heads % d.num_kv_heads)
    return fail(PDA_ERR_SHAPE, "num_q_heads %d is not a multiple of num_kv_heads %d", d.num_q_heads,
                d.num_kv_heads);
  if (d.head_dim != 64 && d.head_dim != 128 && d.head_dim != 256)
    return fail(PDA_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128, 256)", d.head_dim);
  if (d.batch > pda::kMaxGemvBatchAnyRows &&
      (static_cast<int64_t>(d.num_q_heads + 2 * d.num_kv_heads) * d.head_dim) % 128)
    return fail(PDA_ERR_UNSUPPORTED, "prelude batch %d above %d needs (num_q_heads + 2 num_kv_heads) * head_dim "
                "a multiple of 128", d.batch, pda::kMaxGemvBatchAnyRows);
  if (d.num_kv_heads > PDA_MAX_KV_HEADS || d.num_q_heads > 8 * PDA_MAX_KV_HEADS)
    return fail(PDA_ERR_UNSUPPORTED, "too many heads (q %d, kv %d)", d.num_q_heads, d.num_kv_heads);
  if (d.rotary_dim < 0 || d.rotary_dim > d.head_dim || (d.rotary_dim & 1))
    return fail(PDA_ERR_SHAPE, "rotary_dim %d (0, or even up to head_dim %d)", d.rotary_dim, d.head_dim);
  if (d.interleaved != 0 && d.interleaved != 1) return fail(PDA_ERR_SHAPE, "interleaved must be 0 or 1");
  if (!std::isfinite(d.rope_theta) || !(d.rope_theta > 0.f))
    return fail(PDA_ERR_SCALE, "rope_theta must be finite and > 0");
  if (!std::isfinite(d.eps) || d.eps < 0.f) return fail(PDA_ERR_SCALE, "eps must be finite and >= 0");
  return PDA_OK;
}

pda::Fusable prelude_fusable(bool qk_norm, bool interleaved, int rotary_dim) {
  return pda::prelude_fusable(qk_norm, interleaved, rotary_dim) ? pda::Fusable::kPairs : pda::Fusable::kNo;
}

int64_t prelude_rows(const pda_prelude_dims& d) {
  return static_cast<int64_t>(d.num_q_heads + 2 * d.num_kv_heads) * d.head_dim;
}

bool overlaps(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + static_cast<uintptr_t>(b_bytes) && y < x + static_cast<uintptr_t>(a_bytes);
}

// An output that is not one of the arrays it may replace lies apart from all
// that is read.
struct Extent {
  const char* name;
  const void* p;
  int64_t bytes;
};
int check_apart(const Extent& out, std::initializer_list<Extent> others) {
  for (const Extent& o : others)
    if (overlaps(out.p, out.bytes, o.p, o.bytes)) return fail(PDA_ERR_LAYOUT, "%s overlaps %s", out.name, o.name);
  return PDA_OK;
}

// ------------------------------------------------------------ feed-forward
int check_linear(const pda_linear_dims* dm) {
  if (!dm) return fail(PDA_ERR_NULL, "dims is NULL");
  const pda_linear_dims& d = *dm;
  if (d.batch < 0) return fail(PDA_ERR_SHAPE, "batch must be >= 0 (got %d)", d.batch);
  if (d.batch > pda::kMaxGemvBatch) return fail(PDA_ERR_UNSUPPORTED, "batch %d exceeds %d", d.batch, pda::kMaxGemvBatch);
  if (d.in_features <= 0 || d.out_features <= 0) return fail(PDA_ERR_SHAPE, "in_features and out_features must be positive");
  if (d.in_features % pda::kTileK || d.in_features > 65536)
    return fail(PDA_ERR_UNSUPPORTED, "in_features %d (supported: multiples of 32 up to 65536)", d.in_features);
  if (d.out_features % pda::kTileRows || d.out_features > pda::kMaxLinearFeatures)
    return fail(PDA_ERR_UNSUPPORTED, "out_features %d (supported: multiples of 16 up to %d)", d.out_features,
                pda::kMaxLinearFeatures);
  if (d.activation < PDA_ACT_NONE || d.activation > PDA_ACT_RELU)
    return fail(PDA_ERR_UNSUPPORTED, "activation %d is not a pda_activation", d.activation);
  if ((d.gated != 0 && d.gated != 1) || (d.out_f32 != 0 && d.out_f32 != 1))
    return fail(PDA_ERR_SHAPE, "gated and out_f32 must be 0 or 1");
  if (d.gated && static_cast<int64_t>(d.in_features) * d.out_features > pda::kMaxGatedElements)
    return fail(PDA_ERR_UNSUPPORTED, "a gated product takes in_features * out_features up to %lld",
                static_cast<long long>(pda::kMaxGatedElements));
  return PDA_OK;
}

int linear_rows(const pda_linear_dims& d) { return d.gated ? 2 * d.out_features : d.out_features; }

pda::RowsPlan linear_plan(const pda_linear_dims& d, int cus) {
  return pda::plan_linear(d.batch, linear_rows(d), d.in_features, cus, d.gated != 0);
}

int64_t linear_ws_bytes(const pda_linear_dims& d, int cus) {
  return align256(pda::linear_most_floats(d.batch, linear_rows(d), cus) * 4);
}

int check_moe(const pda_moe_dims* dm) {
  if (!dm) return fail(PDA_ERR_NULL, "dims is NULL");
  const pda_moe_dims& d = *dm;
  if (d.tokens < 0) return fail(PDA_ERR_SHAPE, "tokens must be >= 0 (got %d)", d.tokens);
  if (d.tokens > pda::kMaxMoeTokens) return fail(PDA_ERR_UNSUPPORTED, "tokens %d exceeds %d", d.tokens, pda::kMaxMoeTokens);
  if (d.hidden <= 0 || d.inter <= 0 || d.num_experts <= 0 || d.top_k <= 0)
    return fail(PDA_ERR_SHAPE, "hidden, inter, num_experts and top_k must be positive");
  if (d.hidden % pda::kTileK || d.hidden > 32768)
    return fail(PDA_ERR_UNSUPPORTED, "hidden %d (supported: multiples of 32 up to 32768)", d.hidden);
  if (d.inter % pda::kTileK || d.inter > 65536)
    return fail(PDA_ERR_UNSUPPORTED, "inter %d (supported: multiples of 32 up to 65536)", d.inter);
  if (d.num_experts > pda::kMaxExperts || d.top_k > pda::kMaxTopK)
    return fail(PDA_ERR_UNSUPPORTED, "num_experts %d, top_k %d (supported: up to %d and %d)", d.num_experts, d.top_k,
                pda::kMaxExperts, pda::kMaxTopK);
  if (static_cast<int64_t>(d.num_experts) * std::max(2 * d.inter, d.hidden) >= (int64_t{1} << 31))
    return fail(PDA_ERR_UNSUPPORTED, "num_experts * 2 inter and num_experts * hidden must be below 2^31");
  if (d.activation < PDA_ACT_NONE || d.activation > PDA_ACT_RELU)
    return fail(PDA_ERR_UNSUPPORTED, "activation %d is not a pda_activation", d.activation);
  return PDA_OK;
}

pda::ExpertsPlan moe_plan(const pda_moe_dims& d, int cus) {
  return pda::plan_experts(d.tokens, d.hidden, d.inter, d.num_experts, d.top_k, cus);
}

// h [pairs, inter] in bf16, then y [splits, pairs, hidden] in fp32: what a call
// writes, and what covers every call of fewer tokens or choices.
int64_t moe_h_bytes(const pda_moe_dims& d) { return align256(int64_t{2} * d.tokens * d.top_k * d.inter); }
int64_t moe_call_bytes(const pda_moe_dims& d, const pda::ExpertsPlan& p) { return moe_h_bytes(d) + align256(4 * p.y_floats); }
int64_t moe_ws_bytes(const pda_moe_dims& d, int cus) {
  return moe_h_bytes(d) + align256(4 * pda::moe_most_floats(d.tokens * d.top_k, d.hidden, cus));
}

// k splits of an output projection: only where the kernel that adds them
// holds a row of z.
int oproj_splits(int hidden) { return hidden <= pda::kSumFeatures ? pda::kMaxRowsSplits : 1; }

// Workspace of a prelude whose epilogue is a kernel of its own: the fp32
// projection, one per k split.  Like that of the output projection it covers
// every smaller batch of the same rows, so that a workspace grown or reserved
// for one batch serves (also under capture) all below it, and it is asked for
// by every prelude, whether this one's epilogue needs it or not: which do
// depends on the batch, the norm weights and the outputs' places.
int64_t prelude_ws_bytes(const pda_prelude_dims& d, int cus) {
  return align256(pda::rows_most_floats(d.batch, static_cast<int>(prelude_rows(d)), cus, pda::kMaxRowsSplits) * 4);
}

pda::RowsPlan oproj_plan(int batch, int in_features, int hidden, int cus) {
  return pda::plan_rows(batch, hidden, in_features, cus, pda::Fusable::kNo, oproj_splits(hidden));
}

// o_proj workspace: z [splits, batch, hidden] in fp32, then the partial sums
// of z^2.
int64_t oproj_ss_offset(const pda::RowsPlan& plan, int batch, int hidden) {
  return align256(static_cast<int64_t>(plan.splits) * batch * hidden * 4);
}

int64_t oproj_ss_bytes(int batch, int hidden, int parts) {
  return align256(static_cast<int64_t>(batch) * (hidden / pda::kTileRows) * parts * 4);
}

int64_t oproj_ws_bytes(int batch, int hidden, int cus) {
  return align256(pda::rows_most_floats(batch, hidden, cus, oproj_splits(hidden)) * 4) +
         oproj_ss_bytes(batch, hidden, pda::kMaxSsParts);
}

bool oproj_in_range(int32_t batch, int32_t in_features, int32_t hidden) {
  return batch >= 0 && batch <= pda::kMaxGemvBatch && in_features > 0 && in_features % pda::kTileK == 0 && hidden > 0 &&
         hidden % pda::kTileRows == 0 && hidden <= pda::kMaxOProjHidden &&
         (batch <= pda::kMaxGemvBatchAnyRows || hidden % 128 == 0);
}

pda_projection projection(const pda::RowsPlan& p, int64_t workspace_bytes) {
  pda_projection o;
  o.row_tiles = p.rt;
  o.col_tiles = p.bt;
  o.wide = p.wide ? 1 : 0;
  o.col_groups = p.col_groups;
  o.k_splits = p.splits;
  o.fused = p.fused ? 1 : 0;
  o.workgroups = p.row_groups * p.col_groups * p.splits;
  o.ss_parts = p.ss_parts;
  o.workspace_bytes = workspace_bytes;
  return o;
}

// Shared by both prelude entry points once their own arguments are checked.
int run_prelude(const void* x, const void* w_packed, const void* bias, const void* q_norm, const void* k_norm,
                const int32_t* context_lens, void* q_out, pda::PreludeArgs ep, const pda_prelude_dims& d,
                void* stream) {
  if (!x || !w_packed || !context_lens || !q_out) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if ((q_norm == nullptr) != (k_norm == nullptr))
    return fail(PDA_ERR_NULL, "q_norm and k_norm must both be given or both be NULL");
  if (misaligned(x, 16) || misaligned(w_packed, 16) || misaligned(q_out, 16))
    return fail(PDA_ERR_ALIGN, "x, w_packed and the outputs must be 16-byte aligned");
  if (misaligned(bias, 2) || misaligned(q_norm, 2) || misaligned(k_norm, 2) || misaligned(context_lens, 4))
    return fail(PDA_ERR_ALIGN, "bias / norm weights must be 2-byte and context_lens 4-byte aligned");
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  int rc = device_cus(dev, &cus);
  if (rc) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  pda::RowsArgs g;
  g.x = static_cast<const uint16_t*>(x);
  g.wp = static_cast<const uint16_t*>(w_packed);
  g.y = nullptr;
  g.batch = d.batch;
  g.n = static_cast<int>(prelude_rows(d));
  g.k = d.hidden;
  ep.y = nullptr;
  ep.bias = static_cast<const uint16_t*>(bias);
  ep.q_norm = static_cast<const uint16_t*>(q_norm);
  ep.k_norm = static_cast<const uint16_t*>(k_norm);
  ep.lens = context_lens;
  ep.q_out = static_cast<uint16_t*>(q_out);
  ep.batch = d.batch;
  ep.hq = d.num_q_heads;
  ep.hkv = d.num_kv_heads;
  ep.d = d.head_dim;
  ep.rotary_dim = d.rotary_dim;
  ep.interleaved = d.interleaved;
  {
    const double log2_theta = std::log2(static_cast<double>(d.rope_theta));
    for (int k = 0; k < 8; ++k)
      ep.freq_pow2[k] = d.rotary_dim > 0 ? std::exp2(-(2.0 * (1 << k) / d.rotary_dim) * log2_theta) : 0.0;
  }
  ep.eps = d.eps;
  // The epilogue runs in the projection kernel where it can, unless an
  // output lies over something that kernel still reads for other outputs:
  // then the projection goes through the workspace.
  bool fusable = pda::prelude_fusable(ep.q_norm != nullptr, ep.interleaved != 0, ep.rotary_dim);
  if (fusable) {
    const int64_t kv_bytes = static_cast<int64_t>(d.batch) * d.num_kv_heads * d.head_dim * 2;
    const int64_t cache_bytes =
        ep.k_cache ? (static_cast<int64_t>(ep.num_pages) << ep.page_shift) * d.num_kv_heads * d.head_dim * 2 : 0;
    const struct { const void* p; int64_t bytes; } outs[] = {
        {q_out, static_cast<int64_t>(d.batch) * d.num_q_heads * d.head_dim * 2},
        {ep.k_out, kv_bytes}, {ep.v_out, kv_bytes}, {ep.k_cache, cache_bytes}, {ep.v_cache, cache_bytes}};
    for (const auto& o : outs)
      fusable = fusable && !overlaps(o.p, o.bytes, x, static_cast<int64_t>(d.batch) * d.hidden * 2) &&
              !overlaps(o.p, o.bytes, w_packed, static_cast<int64_t>(g.n) * g.k * 2);
  }
  const pda::RowsPlan plan = pda::plan_rows(g.batch, g.n, g.k, cus, fusable ? pda::Fusable::kPairs : pda::Fusable::kNo,
                                            pda::kMaxRowsSplits);
  const bool fused = plan.fused;
  void* ws = nullptr;
  const int64_t least = fused ? 0 : align256(static_cast<int64_t>(plan.splits) * g.batch * g.n * 4);
  if ((rc = workspace_for(dev, st, least, prelude_ws_bytes(d, cus), &ws))) return rc;
  if (!fused) {
    g.y = static_cast<float*>(ws);
    ep.y = g.y;
    ep.splits = plan.splits;
  }
  const Rec rec = prof_begin(1);
  const bool prof = rec.a != nullptr;
  if (prof && (e = hipEventRecord(rec.a, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
  e = fused ? pda::launch_rows_prelude(g, plan, ep, st) : pda::launch_rows(g, plan, st);
  if (e != hipSuccess) return hip_fail(e, "GEMV kernel launch");
  if (prof && (e = hipEventRecord(rec.b, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
  if (!fused && (e = pda::launch_prelude_epilogue(ep, st)) != hipSuccess)
    return hip_fail(e, "prelude epilogue launch");
  if (prof) {
    if ((e = hipEventRecord(rec.c, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
    prof_push(rec);
  }
  return PDA_OK;
}

int check_kv4_page(int32_t p) {
  if (p < 16) return fail(PDA_ERR_UNSUPPORTED, "page_size %d (a 4-bit cache: powers of two from 16 to %d)", p, PDA_MAX_PAGE_SIZE);
  return PDA_OK;
}

// The checks of an append to a 4-bit cache and of a read from it (k, v: the
// bf16 side), and the arguments of their kernels.
int check_kv4_tokens(pda::Kv4Args* c, const void* k, const void* v, const void* k_codes, const void* k_scales,
                     const void* v_codes, const void* v_scales, const int32_t* block_table, const int32_t* context_lens,
                     int32_t batch, int32_t num_tokens, int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                     int32_t num_pages, int32_t max_pages_per_seq, void* stream) {
  g_err.clear();
  int rc = check_shape(batch, num_kv_heads, num_kv_heads, head_dim, page_size, max_pages_per_seq);
  if (rc || (rc = check_kv4_page(page_size))) return rc;
  if (num_tokens < 1 || num_tokens > pda::kKv4MaxTokens)
    return fail(PDA_ERR_SHAPE, "num_tokens must be in [1, %d] (got %d)", pda::kKv4MaxTokens, num_tokens);
  if (static_cast<int64_t>(num_tokens) * num_kv_heads * head_dim > (int64_t{1} << 30))
    return fail(PDA_ERR_UNSUPPORTED, "num_tokens * num_kv_heads * head_dim exceeds 2^30");
  if (num_pages <= 0) return fail(PDA_ERR_SHAPE, "num_pages must be positive (got %d)", num_pages);
  if (batch == 0) return PDA_OK;
  if (!k || !v || !k_codes || !k_scales || !v_codes || !v_scales || !block_table || !context_lens)
    return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (misaligned(k, 16) || misaligned(v, 16) || misaligned(k_codes, 16) || misaligned(v_codes, 16))
    return fail(PDA_ERR_ALIGN, "keys, values and codes must be 16-byte aligned");
  if (misaligned(block_table, 4) || misaligned(context_lens, 4))
    return fail(PDA_ERR_ALIGN, "block_table and context_lens must be 4-byte aligned");
  if ((rc = maybe_validate(block_table, context_lens, batch, max_pages_per_seq, page_size, num_pages, last_tokens(num_tokens),
                           static_cast<hipStream_t>(stream))))
    return rc;
  c->k = static_cast<uint8_t*>(const_cast<void*>(k_codes));
  c->ks = static_cast<uint8_t*>(const_cast<void*>(k_scales));
  c->v = static_cast<uint8_t*>(const_cast<void*>(v_codes));
  c->vs = static_cast<uint8_t*>(const_cast<void*>(v_scales));
  c->bt = block_table;
  c->lens = context_lens;
  c->batch = batch;
  c->tokens = num_tokens;
  c->hkv = num_kv_heads;
  c->head_dim = head_dim;
  c->page_shift = log2i(page_size);
  c->num_pages = num_pages;
  c->maxp = max_pages_per_seq;
  return PDA_OK;
}

// The attention entry points: argument checks, plan, workspace, launches.
// kv4: the caches are its 4-bit ones (k_cache, v_cache: the codes).
// noalloc: the workspace is the library's fixed per-device scratch (no
// allocation, no paging validation, no profiling events) instead of the
// (device, stream) workspace, and shapes whose plan needs more than it
// holds are rejected.
int attention_call(const void* q, const void* k_cache, const void* v_cache, const int32_t* block_table,
                   const int32_t* context_lens, void* out, int32_t batch, int32_t num_q_heads,
                   int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t num_pages,
                   int32_t max_pages_per_seq, int32_t num_queries, int32_t window, float scale, void* stream,
                   bool noalloc, int32_t sinks = 0, const pda::Kv4Args* kv4 = nullptr) {
  g_err.clear();
  int rc = check_attention(batch, num_q_heads, num_kv_heads, head_dim, page_size, max_pages_per_seq);
  if (rc) return rc;
  if (kv4 && (rc = check_kv4_page(page_size))) return rc;
  if (num_pages <= 0) return fail(PDA_ERR_SHAPE, "num_pages must be positive (got %d)", num_pages);
  if (num_queries < 1) return fail(PDA_ERR_SHAPE, "num_queries must be >= 1 (got %d)", num_queries);
  if (window < 0) return fail(PDA_ERR_SHAPE, "window must be >= 0 (got %d)", window);
  if (sinks < 0) return fail(PDA_ERR_SHAPE, "num_sinks must be >= 0 (got %d)", sinks);
  // Every key is visible without a window; with several queries the kernel for sinks still is the one that keeps what
  // is not finite from those that do not see it.
  if (window == 0 && num_queries == 1) sinks = 0;
  // A window as long as the table hides nothing and no query sees more sinks than it holds; the kernels subtract a
  // window from positions that go down to 1 - num_queries, in 32 bits.
  const int32_t most_tokens = max_pages_per_seq * page_size;  // at most 2^30 (check_shape)
  window = std::min(window, most_tokens);
  sinks = std::min(sinks, most_tokens);
  if (num_queries > pda::kMaxCols || num_queries * (num_q_heads / num_kv_heads) > pda::kMaxCols)
    return fail(PDA_ERR_UNSUPPORTED, "num_queries %d x query group %d exceeds %d", num_queries,
                num_q_heads / num_kv_heads, pda::kMaxCols);
  if (!std::isfinite(scale)) return fail(PDA_ERR_SCALE, "scale is not finite");
  const int cols = num_queries * (num_q_heads / num_kv_heads);
  int valu_cols = 0;
  if (!kv4 && !sinks && (rc = check_compute_path(head_dim, page_size, cols, batch, &valu_cols))) return rc;
  if (batch == 0) return PDA_OK;
  if (!q || !k_cache || !v_cache || !block_table || !context_lens || !out || (kv4 && (!kv4->ks || !kv4->vs)))
    return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  auto misaligned = [](const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; };
  if (misaligned(q, 16) || misaligned(k_cache, 16) || misaligned(v_cache, 16) || misaligned(out, 16))
    return fail(PDA_ERR_ALIGN, "q, %s and out must be 16-byte aligned", kv4 ? "k_codes, v_codes" : "k_cache, v_cache");
  if (misaligned(block_table, 4) || misaligned(context_lens, 4))
    return fail(PDA_ERR_ALIGN, "block_table and context_lens must be 4-byte aligned");
  if (!noalloc && (rc = maybe_validate(block_table, context_lens, batch, max_pages_per_seq, page_size, num_pages,
                                       Touched{num_queries, window, sinks, 0}, static_cast<hipStream_t>(stream))))
    return rc;

  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  if ((rc = device_cus(dev, &cus))) return rc;
  const Form form = kv4 ? kv4_form(head_dim, batch) : bf16_form(head_dim, sinks > 0);
  const Plan pl = make_plan(form, batch, num_kv_heads, head_dim,
                            most_steps(page_size, max_pages_per_seq, num_queries, window, sinks), cus, cols);
  const size_t lds = kv4 ? pda::kv4_attn_lds_bytes(head_dim, batch, pl.waves)
                         : pda::attn_lds_bytes(head_dim, batch, pl.waves, valu_cols > 0);
  if (lds > static_cast<size_t>(pda::kMaxLdsBytes))
    return fail(PDA_ERR_UNSUPPORTED, "batch %d needs more LDS than a workgroup has", batch);
  hipStream_t st = static_cast<hipStream_t>(stream);
  void* ws = nullptr;
  int32_t* cnt = nullptr;
  if (noalloc) {
    // the partials from the start of the scratch, the merge counters at its end
    const int64_t counter_bytes = static_cast<int64_t>(pda::kMaxFusedGrid) * 4;
    if (pl.bytes > PDA_NOALLOC_SCRATCH_BYTES - counter_bytes)
      return fail(PDA_ERR_UNSUPPORTED,
                  "this shape needs %lld bytes of workspace; the no-allocation entry point holds %lld",
                  static_cast<long long>(pl.bytes), static_cast<long long>(PDA_NOALLOC_SCRATCH_BYTES - counter_bytes));
    if ((e = pda::noalloc_scratch(dev, &ws)) != hipSuccess) return hip_fail(e, "hipGetSymbolAddress(scratch)");
    cnt = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + PDA_NOALLOC_SCRATCH_BYTES - counter_bytes);
  } else {
    const int64_t most = workspace_bytes(form, batch, num_kv_heads, head_dim, page_size, max_pages_per_seq, cus, cols);
    if ((rc = workspace_for(dev, st, pl.bytes, most, &ws))) return rc;
    if (pl.fused && (rc = counters_for(dev, st, &cnt))) return rc;
  }

  pda::LaunchArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k_cache);
  a.v = static_cast<const uint16_t*>(v_cache);
  a.bt = block_table;
  a.lens = context_lens;
  a.out = static_cast<uint16_t*>(out);
  a.ws_acc = reinterpret_cast<float*>(static_cast<char*>(ws) + pl.off_acc);
  a.ws_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + pl.off_ml);
  a.ws_pref = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + pl.off_pref);
  a.batch = batch;
  a.hq = num_q_heads;
  a.hkv = num_kv_heads;
  a.group = num_q_heads / num_kv_heads;
  a.head_dim = head_dim;
  a.page_shift = log2i(page_size);
  a.num_pages = num_pages;
  a.maxp = max_pages_per_seq;
  a.grid = pl.grid;
  a.waves = pl.waves;
  a.hgs = pl.hgs;
  a.min_steps = pl.min_steps;
  a.scale = scale;
  a.nq = num_queries;
  a.window = window;
  a.sinks = sinks;
  a.valu_cols = valu_cols;
  a.ws_cnt = cnt;
  a.fused = pl.fused;
  a.chunks = pl.chunks;
  a.chunk_steps = pl.chunk_steps;
  // the first-piece stash of stream-K plans, where the LDS holds it
  a.stash = !kv4 && pl.chunks == 0 && !pl.fused && pl.grid > 1 && valu_cols == 0 &&
            pda::attn_stash_lds_bytes(head_dim, batch, pl.waves, pl.hgs, cols, valu_cols > 0) <=
                static_cast<size_t>(pda::kMaxLdsBytes);

  const Rec rec = noalloc ? Rec{nullptr, nullptr, nullptr, 0} : prof_begin(0);
  const bool prof = rec.a != nullptr;
  if (prof && (e = hipEventRecord(rec.a, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
  e = kv4 ? pda::launch_kv4_attn(a, *kv4, st) : pda::launch_attn_kernel(a, st);
  if (e != hipSuccess) return hip_fail(e, "attention kernel launch");
  if (prof && (e = hipEventRecord(rec.b, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
  // with one workgroup, or one fixed-split chunk per sequence, every piece
  // is a whole sequence: nothing to merge; a fused plan merged in the
  // attention kernel
  if (pl.grid > 1 && !pl.fused && pl.chunks != 1 && (e = pda::launch_merge_kernel(a, st)) != hipSuccess)
    return hip_fail(e, "merge kernel launch");
  if (prof) {
    if ((e = hipEventRecord(rec.c, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
    prof_push(rec);
  }
  return PDA_OK;
}

// ---------------------------------------------------------------- pages
// Checks shared by the calls that rewrite a table: its sizes, and that no
// output lies over an input or another output.
int check_pages(int32_t batch, int32_t rows, int32_t page_size, int32_t num_pages, int32_t maxp) {
  int rc = check_shape(batch, 1, 1, 64, page_size, maxp);
  if (rc || (rc = check_shape(rows, 1, 1, 64, page_size, maxp))) return rc;
  if (num_pages <= 0) return fail(PDA_ERR_SHAPE, "num_pages must be positive (got %d)", num_pages);
  if (num_pages > pda::kMaxPoolPages)
    return fail(PDA_ERR_UNSUPPORTED, "num_pages %d exceeds %d", num_pages, pda::kMaxPoolPages);
  if (static_cast<int64_t>(std::max(batch, rows)) * maxp >= (int64_t{1} << 31))
    return fail(PDA_ERR_UNSUPPORTED, "rows * max_pages_per_seq exceeds 2^31");
  return PDA_OK;
}

struct Span {
  const char* name;
  const void* p;
  int64_t words;
};

// All present (but for empty ones), 4-byte aligned, and the outputs, which come
// last from `first_out` on, apart from everything else.
template <size_t kN>
int check_spans(const Span (&s)[kN], size_t first_out) {
  for (const Span& x : s) {
    if (x.words > 0 && !x.p) return fail(PDA_ERR_NULL, "%s is NULL", x.name);
    if (misaligned(x.p, 4)) return fail(PDA_ERR_ALIGN, "%s must be 4-byte aligned", x.name);
  }
  for (size_t i = first_out; i < kN; ++i)
    for (size_t j = 0; j < i; ++j)
      if (overlaps(s[i].p, 4 * s[i].words, s[j].p, 4 * s[j].words))
        return fail(PDA_ERR_LAYOUT, "%s overlaps %s", s[i].name, s[j].name);
  return PDA_OK;
}

int64_t update_ws_bytes(int32_t rows, int32_t num_pages) {
  return align256((3 * static_cast<int64_t>(num_pages) + 3 * static_cast<int64_t>(rows)) * 4);
}
int64_t compact_ws_bytes(int32_t num_pages) {
  return align256((2 * static_cast<int64_t>(num_pages) + num_pages / pda::kCompactPages + 1) * 4);
}

// A workspace for every call of these sizes, for the most (query token, head)
// columns, so any num_queries fits.
int reserve_attention(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                      int32_t max_pages_per_seq, bool kv4, void* stream) {
  g_err.clear();
  int rc = check_attention(batch, num_q_heads, num_kv_heads, head_dim, page_size, max_pages_per_seq);
  if (rc) return rc;
  if (kv4 && (rc = check_kv4_page(page_size))) return rc;
  if (batch == 0) return PDA_OK;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  if ((rc = device_cus(dev, &cus))) return rc;
  void* ptr = nullptr;
  const int64_t need = workspace_bytes(kv4 ? kv4_form(head_dim, batch) : bf16_form(head_dim), batch, num_kv_heads, head_dim,
                                       page_size, max_pages_per_seq, cus, pda::kMaxCols);
  if ((rc = workspace_for(dev, static_cast<hipStream_t>(stream), need, need, &ptr))) return rc;
  if (kv4) return PDA_OK;  // (no fused merge, so no counters)
  int32_t* cnt = nullptr;
  return counters_for(dev, static_cast<hipStream_t>(stream), &cnt);
}

}  // namespace

extern "C" {

const char* pda_last_error(void) { return g_err.c_str(); }

int32_t pda_version(void) { return PDA_VERSION; }

int pda_plan(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
             int32_t page_size, int32_t max_pages_per_seq, int32_t num_cus, int32_t* grid_blocks,
             int32_t* waves, int64_t* workspace_size) {
  g_err.clear();
  if (!grid_blocks || !waves || !workspace_size) return fail(PDA_ERR_NULL, "pda_plan: NULL output pointer");
  int rc = check_attention(batch, num_q_heads, num_kv_heads, head_dim, page_size, max_pages_per_seq);
  if (rc) return rc;
  if (num_cus <= 0) return fail(PDA_ERR_SHAPE, "num_cus must be positive");
  const Form form = bf16_form(head_dim);
  Plan pl = make_plan(form, batch, num_kv_heads, head_dim, most_steps(page_size, max_pages_per_seq, 1, 0), num_cus,
                      num_q_heads / num_kv_heads);
  *grid_blocks = batch ? pl.grid : 0;
  *waves = batch ? pl.grid * pl.waves : 0;
  *workspace_size =
      batch ? workspace_bytes(form, batch, num_kv_heads, head_dim, page_size, max_pages_per_seq, num_cus, pda::kMaxCols) : 0;
  return PDA_OK;
}

int pda_workspace_reserve(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                          int32_t page_size, int32_t max_pages_per_seq, void* stream) {
  return reserve_attention(batch, num_q_heads, num_kv_heads, head_dim, page_size, max_pages_per_seq, false, stream);
}

int pda_kv4_workspace_reserve(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                              int32_t page_size, int32_t max_pages_per_seq, void* stream) {
  return reserve_attention(batch, num_q_heads, num_kv_heads, head_dim, page_size, max_pages_per_seq, true, stream);
}

int pda_release_workspaces(void) {
  g_err.clear();
  std::lock_guard<std::mutex> lock(g_ws_mu);
  int rc = PDA_OK;
  for (auto& kv : g_ws) {
    if (!kv.second.ptr && !kv.second.cnt) continue;  // (outgrown buffers have a successor in ptr)
    int cur = 0;
    hipError_t e = hipGetDevice(&cur);
    if (e == hipSuccess) e = hipSetDevice(kv.first.first);
    if (e == hipSuccess) e = hipStreamSynchronize(kv.first.second);
    if (e == hipSuccess && kv.second.ptr) e = hipFree(kv.second.ptr);
    for (void* p : kv.second.outgrown)
      if (e == hipSuccess) e = hipFree(p);
    if (e == hipSuccess && kv.second.cnt) e = hipFree(kv.second.cnt);
    const hipError_t back = hipSetDevice(cur);
    if (e == hipSuccess) e = back;
    if (e != hipSuccess) rc = hip_fail(e, "releasing a workspace");
  }
  g_ws.clear();
  return rc;
}

int pda_set_option(int32_t option, int32_t value) {
  g_err.clear();
  switch (option) {
    case PDA_OPT_BLOCKS_PER_CU:
      if (value < 1 || value > kMaxBlocksPerCu)
        return fail(PDA_ERR_SHAPE, "blocks per CU must be in [1, %d]", kMaxBlocksPerCu);
      g_blocks_per_cu.store(value);
      return PDA_OK;
    case PDA_OPT_MIN_STEPS:
      if (value < 0) return fail(PDA_ERR_SHAPE, "min steps per wave must be >= 0 (0 = the planner's choice)");
      g_min_steps.store(value);
      return PDA_OK;
    case PDA_OPT_COMPUTE_PATH:
      if (value < 0 || value > 1) return fail(PDA_ERR_SHAPE, "compute path must be 0 or 1");
      g_compute_path.store(value);
      return PDA_OK;
    case PDA_OPT_FUSED_MERGE:
      if (value < 0 || value > 2) return fail(PDA_ERR_SHAPE, "fused merge must be 0, 1 or 2");
      g_fused_merge.store(value);
      return PDA_OK;
    case PDA_OPT_KV_GROUP:
      if (value < 0 || value > pda::kMaxWaves) return fail(PDA_ERR_SHAPE, "kv group must be in [0, %d]", pda::kMaxWaves);
      g_kv_group.store(value);
      return PDA_OK;
    case PDA_OPT_FIXED_SPLIT:
      if (value < 0 || value > 1) return fail(PDA_ERR_SHAPE, "fixed split must be 0 or 1");
      g_fixed_split.store(value);
      return PDA_OK;
    default:
      return fail(PDA_ERR_UNSUPPORTED, "unknown option %d", option);
  }
}

int32_t pda_get_option(int32_t option) {
  switch (option) {
    case PDA_OPT_BLOCKS_PER_CU: return blocks_per_cu();
    case PDA_OPT_MIN_STEPS: return min_steps_option();
    case PDA_OPT_COMPUTE_PATH: return compute_path();
    case PDA_OPT_FUSED_MERGE: return fused_merge();
    case PDA_OPT_KV_GROUP: return kv_group_cap();
    case PDA_OPT_FIXED_SPLIT: return fixed_split();
    default: return -1;
  }
}

int pda_stream_read(const void* buf, int64_t bytes, uint32_t* sink, int32_t unroll, int32_t blocks_per_cu,
                    void* stream) {
  g_err.clear();
  if (bytes <= 0 || bytes % 16) return fail(PDA_ERR_SHAPE, "bytes must be a positive multiple of 16");
  if (unroll == 0) unroll = 16;
  if (blocks_per_cu == 0) blocks_per_cu = 1;
  if (unroll != 4 && unroll != 8 && unroll != 16) return fail(PDA_ERR_UNSUPPORTED, "unroll must be 4, 8 or 16");
  if (blocks_per_cu < 1 || blocks_per_cu > 32) return fail(PDA_ERR_UNSUPPORTED, "blocks_per_cu must be in [1, 32]");
  if (!buf || !sink) return fail(PDA_ERR_NULL, "a pointer is NULL");
  if (reinterpret_cast<uintptr_t>(buf) & 15) return fail(PDA_ERR_ALIGN, "buf must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(sink) & 3) return fail(PDA_ERR_ALIGN, "sink must be 4-byte aligned");
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  int rc = device_cus(dev, &cus);
  if (rc) return rc;
  const int64_t blocks = static_cast<int64_t>(cus) * blocks_per_cu;
  if ((bytes + blocks - 1) / blocks > (int64_t{1} << 31) - 1024)
    return fail(PDA_ERR_SHAPE, "bytes too large for %lld workgroups", static_cast<long long>(blocks));
  e = pda::launch_stream_read(buf, bytes, sink, unroll, static_cast<int>(blocks), static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "stream read kernel launch");
  return PDA_OK;
}

int pda_profile_enable(int32_t on) {
  std::lock_guard<std::mutex> lock(g_prof_mu);
  g_prof_on = on != 0;
  return PDA_OK;
}

int pda_profile_read(double* split_ms, double* merge_ms, int64_t* calls) {
  g_err.clear();
  if (!split_ms || !merge_ms || !calls) return fail(PDA_ERR_NULL, "pda_profile_read: NULL output pointer");
  return prof_read(0, split_ms, merge_ms, calls);
}

int pda_profile_read_prelude(double* gemv_ms, double* epilogue_ms, int64_t* calls) {
  g_err.clear();
  if (!gemv_ms || !epilogue_ms || !calls) return fail(PDA_ERR_NULL, "pda_profile_read_prelude: NULL output pointer");
  return prof_read(1, gemv_ms, epilogue_ms, calls);
}

int pda_kv_append(const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                  const int32_t* block_table, const int32_t* context_lens, int32_t batch, int32_t num_kv_heads,
                  int32_t head_dim, int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq,
                  void* stream) {
  return pda_kv_append_n(k_new, v_new, k_cache, v_cache, block_table, context_lens, batch, 1, num_kv_heads,
                         head_dim, page_size, num_pages, max_pages_per_seq, stream);
}

int pda_kv_append_n(const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                    const int32_t* block_table, const int32_t* context_lens, int32_t batch, int32_t num_tokens,
                    int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t num_pages,
                    int32_t max_pages_per_seq, void* stream) {
  g_err.clear();
  int rc = check_shape(batch, num_kv_heads, num_kv_heads, head_dim, page_size, max_pages_per_seq);
  if (rc) return rc;
  if (num_tokens < 1 || num_tokens > 1024)
    return fail(PDA_ERR_SHAPE, "num_tokens must be in [1, 1024] (got %d)", num_tokens);
  if (num_pages <= 0) return fail(PDA_ERR_SHAPE, "num_pages must be positive (got %d)", num_pages);
  if (batch == 0) return PDA_OK;
  if (!k_new || !v_new || !k_cache || !v_cache || !block_table || !context_lens)
    return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  auto misaligned = [](const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; };
  if (misaligned(k_new, 16) || misaligned(v_new, 16) || misaligned(k_cache, 16) || misaligned(v_cache, 16))
    return fail(PDA_ERR_ALIGN, "k_new, v_new, k_cache and v_cache must be 16-byte aligned");
  if (misaligned(block_table, 4) || misaligned(context_lens, 4))
    return fail(PDA_ERR_ALIGN, "block_table and context_lens must be 4-byte aligned");
  if ((rc = maybe_validate(block_table, context_lens, batch, max_pages_per_seq, page_size, num_pages, last_tokens(num_tokens),
                           static_cast<hipStream_t>(stream))))
    return rc;
  pda::AppendArgs a;
  a.k_new = static_cast<const uint16_t*>(k_new);
  a.v_new = static_cast<const uint16_t*>(v_new);
  a.k = static_cast<uint16_t*>(k_cache);
  a.v = static_cast<uint16_t*>(v_cache);
  a.bt = block_table;
  a.lens = context_lens;
  a.batch = batch;
  a.tokens = num_tokens;
  a.hkv = num_kv_heads;
  a.head_dim = head_dim;
  a.page_shift = log2i(page_size);
  a.num_pages = num_pages;
  a.maxp = max_pages_per_seq;
  hipError_t e = pda::launch_append_kernel(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "append kernel launch");
  return PDA_OK;
}

int paged_decode_attention_append(const void* q, const void* k_new, const void* v_new, void* k_cache,
                                  void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                                  void* out, int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                  int32_t head_dim, int32_t page_size, int32_t num_pages,
                                  int32_t max_pages_per_seq, float scale, void* stream) {
  g_err.clear();
  // validate the attention arguments first so that nothing is written on error
  int rc = check_attention(batch, num_q_heads, num_kv_heads, head_dim, page_size, max_pages_per_seq);
  if (rc) return rc;
  if (!std::isfinite(scale)) return fail(PDA_ERR_SCALE, "scale is not finite");
  int valu_cols = 0;
  if ((rc = check_compute_path(head_dim, page_size, num_q_heads / num_kv_heads, batch, &valu_cols))) return rc;
  if (batch > 0 && (!q || !out)) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if ((reinterpret_cast<uintptr_t>(q) & 15) || (reinterpret_cast<uintptr_t>(out) & 15))
    return fail(PDA_ERR_ALIGN, "q, k_cache, v_cache and out must be 16-byte aligned");
  if ((rc = pda_kv_append(k_new, v_new, k_cache, v_cache, block_table, context_lens, batch, num_kv_heads,
                          head_dim, page_size, num_pages, max_pages_per_seq, stream)))
    return rc;
  return paged_decode_attention(q, k_cache, v_cache, block_table, context_lens, out, batch, num_q_heads,
                                num_kv_heads, head_dim, page_size, num_pages, max_pages_per_seq, scale, stream);
}

int paged_decode_attention(const void* q, const void* k_cache, const void* v_cache,
                           const int32_t* block_table, const int32_t* context_lens, void* out,
                           int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                           int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq, float scale,
                           void* stream) {
  return paged_decode_attention_ext(q, k_cache, v_cache, block_table, context_lens, out, batch, num_q_heads,
                                    num_kv_heads, head_dim, page_size, num_pages, max_pages_per_seq, 1, 0,
                                    scale, stream);
}

int paged_decode_attention_ext(const void* q, const void* k_cache, const void* v_cache,
                               const int32_t* block_table, const int32_t* context_lens, void* out,
                               int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                               int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq,
                               int32_t num_queries, int32_t window, float scale, void* stream) {
  return attention_call(q, k_cache, v_cache, block_table, context_lens, out, batch, num_q_heads, num_kv_heads,
                        head_dim, page_size, num_pages, max_pages_per_seq, num_queries, window, scale, stream,
                        false);
}

int paged_decode_attention_noalloc(const void* q, const void* k_cache, const void* v_cache,
                                   const int32_t* block_table, const int32_t* context_lens, void* out,
                                   int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                   int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq, float scale,
                                   void* stream) {
  return attention_call(q, k_cache, v_cache, block_table, context_lens, out, batch, num_q_heads, num_kv_heads,
                        head_dim, page_size, num_pages, max_pages_per_seq, 1, 0, scale, stream, true);
}

int paged_decode_attention_desc(const pda_tensor* q, const pda_tensor* k_cache, const pda_tensor* v_cache,
                                const pda_tensor* block_table, const pda_tensor* context_lens,
                                const pda_tensor* out, float scale, void* stream) {
  g_err.clear();
  const pda_tensor* ts[6] = {q, k_cache, v_cache, block_table, context_lens, out};
  static const char* const names[6] = {"q", "k_cache", "v_cache", "block_table", "context_lens", "out"};
  static const int32_t dtypes[6] = {PDA_DTYPE_BF16, PDA_DTYPE_BF16, PDA_DTYPE_BF16,
                                    PDA_DTYPE_I32,  PDA_DTYPE_I32,  PDA_DTYPE_BF16};
  static const int32_t ranks[6] = {3, 4, 4, 2, 1, 3};
  for (int i = 0; i < 6; ++i)
    if (!ts[i]) return fail(PDA_ERR_NULL, "%s: descriptor is NULL", names[i]);
  for (int i = 0; i < 6; ++i)
    if (ts[i]->dtype != dtypes[i])
      return fail(PDA_ERR_DTYPE, "%s: dtype %s (%d), expected %s", names[i], dtype_name(ts[i]->dtype),
                  ts[i]->dtype, dtype_name(dtypes[i]));
  int rc;
  for (int i = 0; i < 6; ++i)
    if ((rc = check_rank(*ts[i], names[i], ranks[i]))) return rc;
  const int64_t* qs = q->shape;
  const int64_t* ks = k_cache->shape;
  for (int i = 0; i < 3; ++i)
    if (out->shape[i] != qs[i]) return fail(PDA_ERR_SHAPE, "out must have the shape of q");
  for (int i = 0; i < 4; ++i)
    if (v_cache->shape[i] != ks[i]) return fail(PDA_ERR_SHAPE, "v_cache must have the shape of k_cache");
  if (ks[3] != qs[2])
    return fail(PDA_ERR_SHAPE, "head_dim of q (%lld) and of the caches (%lld) differ", static_cast<long long>(qs[2]),
                static_cast<long long>(ks[3]));
  if (block_table->shape[0] != qs[0] || context_lens->shape[0] != qs[0])
    return fail(PDA_ERR_SHAPE, "block_table and context_lens must have one row per sequence of q (%lld)",
                static_cast<long long>(qs[0]));
  for (int i = 0; i < 6; ++i)
    if ((rc = check_dense(*ts[i], names[i]))) return rc;
  for (int i = 0; i < 6; ++i)
    if (!desc_empty(*ts[i]) && !ts[i]->data) return fail(PDA_ERR_NULL, "%s: data is NULL", names[i]);
  return attention_call(q->data, k_cache->data, v_cache->data, static_cast<const int32_t*>(block_table->data),
                        static_cast<const int32_t*>(context_lens->data), out->data, static_cast<int32_t>(qs[0]),
                        static_cast<int32_t>(qs[1]), static_cast<int32_t>(ks[2]), static_cast<int32_t>(qs[2]),
                        static_cast<int32_t>(ks[1]), static_cast<int32_t>(ks[0]),
                        static_cast<int32_t>(block_table->shape[1]), 1, 0, scale, stream, false);
}

int pda_pack_weights(const void* w, void* w_packed, int32_t rows, int32_t cols, void* stream) {
  g_err.clear();
  if (rows <= 0 || cols <= 0) return fail(PDA_ERR_SHAPE, "rows and cols must be positive");
  if (rows % pda::kTileRows || cols % pda::kTileK)
    return fail(PDA_ERR_SHAPE, "rows must be a multiple of 16 and cols of 32 (got %d x %d)", rows, cols);
  if (static_cast<int64_t>(rows) * cols > (int64_t{1} << 34)) return fail(PDA_ERR_SHAPE, "matrix too large");
  if (!w || !w_packed) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (misaligned(w, 16) || misaligned(w_packed, 16)) return fail(PDA_ERR_ALIGN, "w and w_packed must be 16-byte aligned");
  const uintptr_t a = reinterpret_cast<uintptr_t>(w), b = reinterpret_cast<uintptr_t>(w_packed);
  const uintptr_t bytes = static_cast<uintptr_t>(rows) * cols * 2;
  if (a < b + bytes && b < a + bytes) return fail(PDA_ERR_SHAPE, "w and w_packed overlap");
  hipError_t e = pda::launch_pack(static_cast<const uint16_t*>(w), static_cast<uint16_t*>(w_packed), rows, cols,
                                  static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "pack kernel launch");
  return PDA_OK;
}

int pda_attention_prelude(const void* x, const void* w_packed, const void* bias, const void* q_norm,
                          const void* k_norm, const int32_t* context_lens, void* q_out, void* k_out,
                          void* v_out, const pda_prelude_dims* dims, void* stream) {
  g_err.clear();
  int rc = check_prelude(dims);
  if (rc) return rc;
  if (dims->batch == 0) return PDA_OK;
  if (!k_out || !v_out) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (misaligned(k_out, 16) || misaligned(v_out, 16))
    return fail(PDA_ERR_ALIGN, "x, w_packed and the outputs must be 16-byte aligned");
  pda::PreludeArgs ep{};
  ep.k_out = static_cast<uint16_t*>(k_out);
  ep.v_out = static_cast<uint16_t*>(v_out);
  return run_prelude(x, w_packed, bias, q_norm, k_norm, context_lens, q_out, ep, *dims, stream);
}

int pda_attention_prelude_append(const void* x, const void* w_packed, const void* bias, const void* q_norm,
                                 const void* k_norm, const int32_t* context_lens, void* q_out, void* k_cache,
                                 void* v_cache, const int32_t* block_table, int32_t page_size, int32_t num_pages,
                                 int32_t max_pages_per_seq, const pda_prelude_dims* dims, void* stream) {
  g_err.clear();
  int rc = check_prelude(dims);
  if (rc) return rc;
  if (page_size <= 0 || max_pages_per_seq <= 0)
    return fail(PDA_ERR_SHAPE, "page_size and max_pages_per_seq must be positive");
  if (!is_pow2(page_size) || page_size > PDA_MAX_PAGE_SIZE)
    return fail(PDA_ERR_UNSUPPORTED, "page_size %d (supported: powers of two up to %d)", page_size,
                PDA_MAX_PAGE_SIZE);
  if (static_cast<int64_t>(max_pages_per_seq) * page_size > (int64_t{1} << 30))
    return fail(PDA_ERR_SHAPE, "max_pages_per_seq * page_size too large");
  if (num_pages <= 0) return fail(PDA_ERR_SHAPE, "num_pages must be positive (got %d)", num_pages);
  if (dims->batch == 0) return PDA_OK;
  if (!k_cache || !v_cache || !block_table) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (misaligned(k_cache, 16) || misaligned(v_cache, 16) || misaligned(block_table, 4))
    return fail(PDA_ERR_ALIGN, "caches must be 16-byte and block_table 4-byte aligned");
  pda::PreludeArgs ep{};
  ep.k_cache = static_cast<uint16_t*>(k_cache);
  ep.v_cache = static_cast<uint16_t*>(v_cache);
  ep.bt = block_table;
  ep.page_shift = log2i(page_size);
  ep.num_pages = num_pages;
  ep.maxp = max_pages_per_seq;
  return run_prelude(x, w_packed, bias, q_norm, k_norm, context_lens, q_out, ep, *dims, stream);
}

int pda_o_proj_residual_norm(const void* attn, const void* w_packed, const void* residual, const void* norm_w,
                             void* residual_out, void* normed_out, int32_t batch, int32_t in_features,
                             int32_t hidden, float eps, void* stream) {
  g_err.clear();
  if (batch < 0) return fail(PDA_ERR_SHAPE, "batch must be >= 0 (got %d)", batch);
  if (batch > pda::kMaxGemvBatch) return fail(PDA_ERR_UNSUPPORTED, "batch %d exceeds %d", batch, pda::kMaxGemvBatch);
  if (in_features <= 0 || hidden <= 0) return fail(PDA_ERR_SHAPE, "in_features and hidden must be positive");
  if (in_features % pda::kTileK || in_features > 65536)
    return fail(PDA_ERR_UNSUPPORTED, "in_features %d (supported: multiples of 32 up to 65536)", in_features);
  if (hidden % pda::kTileRows || hidden > pda::kMaxOProjHidden)
    return fail(PDA_ERR_UNSUPPORTED, "hidden %d (supported: multiples of 16 up to %d)", hidden,
                pda::kMaxOProjHidden);
  if (batch > pda::kMaxGemvBatchAnyRows && hidden % 128)
    return fail(PDA_ERR_UNSUPPORTED, "o_proj batch %d above %d needs hidden a multiple of 128", batch,
                pda::kMaxGemvBatchAnyRows);
  if (!std::isfinite(eps) || eps < 0.f) return fail(PDA_ERR_SCALE, "eps must be finite and >= 0");
  if (batch == 0) return PDA_OK;
  if (!attn || !w_packed || !residual || !norm_w || !residual_out || !normed_out)
    return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (misaligned(attn, 16) || misaligned(w_packed, 16))
    return fail(PDA_ERR_ALIGN, "attn and w_packed must be 16-byte aligned");
  if (misaligned(residual, 2) || misaligned(norm_w, 2) || misaligned(residual_out, 2) || misaligned(normed_out, 2))
    return fail(PDA_ERR_ALIGN, "bf16 arrays must be 2-byte aligned");
  if (normed_out == residual_out) return fail(PDA_ERR_SHAPE, "normed_out must not be residual_out");
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  int rc = device_cus(dev, &cus);
  if (rc) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const pda::RowsPlan plan = oproj_plan(batch, in_features, hidden, cus);
  void* ws = nullptr;
  const int64_t least = oproj_ss_offset(plan, batch, hidden) + oproj_ss_bytes(batch, hidden, plan.ss_parts);
  if ((rc = workspace_for(dev, st, least, oproj_ws_bytes(batch, hidden, cus), &ws))) return rc;
  pda::OProjArgs o;
  o.residual = static_cast<const uint16_t*>(residual);
  o.norm_w = static_cast<const uint16_t*>(norm_w);
  o.residual_out = static_cast<uint16_t*>(residual_out);
  o.normed_out = static_cast<uint16_t*>(normed_out);
  o.z = static_cast<float*>(ws);
  o.splits = plan.splits;
  o.ss = reinterpret_cast<float*>(static_cast<char*>(ws) + oproj_ss_offset(plan, batch, hidden));
  o.ss_count = hidden / pda::kTileRows * plan.ss_parts;
  o.batch = batch;
  o.hidden = hidden;
  o.eps = eps;
  pda::RowsArgs g;
  g.x = static_cast<const uint16_t*>(attn);
  g.wp = static_cast<const uint16_t*>(w_packed);
  g.y = o.z;
  g.batch = batch;
  g.n = hidden;
  g.k = in_features;
  const Rec rec = prof_begin(2);
  const bool prof = rec.a != nullptr;
  if (prof && (e = hipEventRecord(rec.a, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
  e = plan.splits > 1 ? pda::launch_rows(g, plan, st) : pda::launch_rows_residual(g, plan, o, st);
  if (e != hipSuccess) return hip_fail(e, "GEMV kernel launch");
  if (prof && (e = hipEventRecord(rec.b, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
  e = plan.splits > 1 ? pda::launch_oproj_sum(o, st) : pda::launch_oproj_norm(o, st);
  if (e != hipSuccess) return hip_fail(e, "o_proj norm launch");
  if (prof) {
    if ((e = hipEventRecord(rec.c, st)) != hipSuccess) return hip_fail(e, "hipEventRecord");
    prof_push(rec);
  }
  return PDA_OK;
}

int pda_o_proj_workspace_reserve(int32_t batch, int32_t in_features, int32_t hidden, void* stream) {
  g_err.clear();
  if (!oproj_in_range(batch, in_features, hidden)) return fail(PDA_ERR_SHAPE, "o_proj shape out of range");
  if (batch == 0) return PDA_OK;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  int rc = device_cus(dev, &cus);
  if (rc) return rc;
  void* ptr = nullptr;
  const int64_t need = oproj_ws_bytes(batch, hidden, cus);
  return workspace_for(dev, static_cast<hipStream_t>(stream), need, need, &ptr);
}

int pda_o_proj_plan(int32_t batch, int32_t in_features, int32_t hidden, int32_t num_cus, pda_projection* out) {
  g_err.clear();
  if (!out) return fail(PDA_ERR_NULL, "pda_o_proj_plan: NULL output pointer");
  if (!oproj_in_range(batch, in_features, hidden)) return fail(PDA_ERR_SHAPE, "o_proj shape out of range");
  if (num_cus <= 0) return fail(PDA_ERR_SHAPE, "num_cus must be positive");
  *out = pda_projection{};
  if (batch == 0) return PDA_OK;
  *out = projection(oproj_plan(batch, in_features, hidden, num_cus), oproj_ws_bytes(batch, hidden, num_cus));
  return PDA_OK;
}

int pda_linear(const void* x, const void* w_packed, const void* bias, const void* residual, void* out,
               const pda_linear_dims* dims, void* stream) {
  g_err.clear();
  int rc = check_linear(dims);
  if (rc) return rc;
  const pda_linear_dims& d = *dims;
  if (d.batch == 0) return PDA_OK;
  if (!x || !w_packed || !out) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (misaligned(x, 16) || misaligned(w_packed, 16)) return fail(PDA_ERR_ALIGN, "x and w_packed must be 16-byte aligned");
  if (misaligned(bias, 2) || misaligned(residual, 2) || misaligned(out, d.out_f32 ? 4 : 2))
    return fail(PDA_ERR_ALIGN, "bf16 arrays must be 2-byte and an fp32 out 4-byte aligned");
  const int rows = linear_rows(d);
  const int64_t features = static_cast<int64_t>(d.batch) * d.out_features;
  const Extent o{"out", out, features * (d.out_f32 ? 4 : 2)};
  const bool in_place = out == residual && !d.out_f32;
  if ((rc = check_apart(o, {{"x", x, int64_t{2} * d.batch * d.in_features},
                            {"w_packed", w_packed, int64_t{2} * rows * d.in_features},
                            {"bias", bias, int64_t{2} * rows},
                            {"residual", in_place ? nullptr : residual, 2 * features}})))
    return rc;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  if ((rc = device_cus(dev, &cus))) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const pda::RowsPlan plan = linear_plan(d, cus);
  void* ws = nullptr;
  const int64_t least = plan.fused ? 0 : align256(int64_t{4} * plan.splits * d.batch * rows);
  if ((rc = workspace_for(dev, st, least, linear_ws_bytes(d, cus), &ws))) return rc;
  pda::RowsArgs g{};
  g.x = static_cast<const uint16_t*>(x);
  g.wp = static_cast<const uint16_t*>(w_packed);
  g.y = plan.fused ? nullptr : static_cast<float*>(ws);
  g.batch = d.batch;
  g.n = rows;
  g.k = d.in_features;
  pda::LinearArgs l;
  l.bias = static_cast<const uint16_t*>(bias);
  l.residual = static_cast<const uint16_t*>(residual);
  l.out = out;
  l.features = d.out_features;
  l.activation = d.activation;
  l.f32 = d.out_f32;
  if ((e = pda::launch_linear(g, plan, l, d.gated != 0, st)) != hipSuccess) return hip_fail(e, "linear kernel launch");
  return PDA_OK;
}

int pda_linear_workspace_reserve(const pda_linear_dims* dims, void* stream) {
  g_err.clear();
  int rc = check_linear(dims);
  if (rc) return rc;
  if (dims->batch == 0) return PDA_OK;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  if ((rc = device_cus(dev, &cus))) return rc;
  void* ptr = nullptr;
  const int64_t need = linear_ws_bytes(*dims, cus);
  return workspace_for(dev, static_cast<hipStream_t>(stream), need, need, &ptr);
}

int pda_linear_plan(const pda_linear_dims* dims, int32_t num_cus, pda_projection* out) {
  g_err.clear();
  if (!out) return fail(PDA_ERR_NULL, "pda_linear_plan: NULL output pointer");
  int rc = check_linear(dims);
  if (rc) return rc;
  if (num_cus <= 0) return fail(PDA_ERR_SHAPE, "num_cus must be positive");
  *out = pda_projection{};
  if (dims->batch == 0) return PDA_OK;
  *out = projection(linear_plan(*dims, num_cus), linear_ws_bytes(*dims, num_cus));
  return PDA_OK;
}

int pda_moe_route(const float* logits, const float* select_bias, int32_t* expert_ids, float* expert_weights,
                  const pda_route_dims* dims, void* stream) {
  g_err.clear();
  if (!dims) return fail(PDA_ERR_NULL, "dims is NULL");
  const pda_route_dims& d = *dims;
  if (d.tokens < 0) return fail(PDA_ERR_SHAPE, "tokens must be >= 0 (got %d)", d.tokens);
  if (d.tokens > pda::kMaxRouteTokens)
    return fail(PDA_ERR_UNSUPPORTED, "tokens %d exceeds %d", d.tokens, pda::kMaxRouteTokens);
  if (d.num_experts <= 0 || d.top_k <= 0) return fail(PDA_ERR_SHAPE, "num_experts and top_k must be positive");
  if (d.num_experts > pda::kMaxExperts || d.top_k > pda::kMaxTopK)
    return fail(PDA_ERR_UNSUPPORTED, "num_experts %d, top_k %d (supported: up to %d and %d)", d.num_experts, d.top_k,
                pda::kMaxExperts, pda::kMaxTopK);
  if (d.top_k > d.num_experts) return fail(PDA_ERR_SHAPE, "top_k %d of %d experts", d.top_k, d.num_experts);
  if (d.logit_stride < d.num_experts)
    return fail(PDA_ERR_LAYOUT, "logit_stride %d is below num_experts %d", d.logit_stride, d.num_experts);
  if ((d.sigmoid != 0 && d.sigmoid != 1) || (d.renormalise != 0 && d.renormalise != 1))
    return fail(PDA_ERR_SHAPE, "sigmoid and renormalise must be 0 or 1");
  if (!std::isfinite(d.scale)) return fail(PDA_ERR_SCALE, "scale must be finite");
  if (d.tokens == 0) return PDA_OK;
  if (!logits || !expert_ids || !expert_weights) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (misaligned(logits, 4) || misaligned(select_bias, 4) || misaligned(expert_ids, 4) || misaligned(expert_weights, 4))
    return fail(PDA_ERR_ALIGN, "logits, select_bias, expert_ids and expert_weights must be 4-byte aligned");
  const int64_t out = int64_t{4} * d.tokens * d.top_k;
  const Extent in{"logits", logits, int64_t{4} * ((d.tokens - 1) * static_cast<int64_t>(d.logit_stride) + d.num_experts)};
  const Extent bias{"select_bias", select_bias, int64_t{4} * d.num_experts};
  int rc = check_apart({"expert_ids", expert_ids, out}, {in, bias, {"expert_weights", expert_weights, out}});
  if (rc || (rc = check_apart({"expert_weights", expert_weights, out}, {in, bias}))) return rc;
  pda::RouteArgs a;
  a.logits = logits;
  a.select_bias = select_bias;
  a.ids = expert_ids;
  a.weights = expert_weights;
  a.stride = d.logit_stride;
  a.tokens = d.tokens;
  a.experts = d.num_experts;
  a.top_k = d.top_k;
  a.sigmoid = d.sigmoid;
  a.renormalise = d.renormalise;
  a.scale = d.scale;
  hipError_t e = pda::launch_route(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "route kernel launch");
  return PDA_OK;
}

int pda_moe_experts(const void* x, const int32_t* expert_ids, const float* expert_weights, const void* w_gate_up,
                    const void* w_down, const void* residual, void* out, const pda_moe_dims* dims, void* stream) {
  g_err.clear();
  int rc = check_moe(dims);
  if (rc) return rc;
  const pda_moe_dims& d = *dims;
  if (d.tokens == 0) return PDA_OK;
  if (!x || !expert_ids || !expert_weights || !w_gate_up || !w_down || !out)
    return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (misaligned(x, 16) || misaligned(w_gate_up, 16) || misaligned(w_down, 16))
    return fail(PDA_ERR_ALIGN, "x, w_gate_up and w_down must be 16-byte aligned");
  if (misaligned(expert_ids, 4) || misaligned(expert_weights, 4) || misaligned(residual, 2) || misaligned(out, 2))
    return fail(PDA_ERR_ALIGN, "expert_ids and expert_weights must be 4-byte, residual and out 2-byte aligned");
  const int64_t rows = int64_t{2} * d.tokens * d.hidden, pairs = static_cast<int64_t>(d.tokens) * d.top_k;
  const int64_t matrix = int64_t{2} * d.num_experts * d.hidden * d.inter;
  if ((rc = check_apart({"out", out, rows}, {{"x", out == x ? nullptr : x, rows},
                                             {"residual", out == residual ? nullptr : residual, rows},
                                             {"expert_ids", expert_ids, 4 * pairs},
                                             {"expert_weights", expert_weights, 4 * pairs},
                                             {"w_gate_up", w_gate_up, 2 * matrix},
                                             {"w_down", w_down, matrix}})))
    return rc;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  if ((rc = device_cus(dev, &cus))) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const pda::ExpertsPlan plan = moe_plan(d, cus);
  void* ws = nullptr;
  if ((rc = workspace_for(dev, st, moe_call_bytes(d, plan), moe_ws_bytes(d, cus), &ws))) return rc;
  pda::ExpertsArgs a{};
  a.x = static_cast<const uint16_t*>(x);
  a.ids = expert_ids;
  a.weights = expert_weights;
  a.w_gate_up = static_cast<const uint16_t*>(w_gate_up);
  a.w_down = static_cast<const uint16_t*>(w_down);
  a.residual = static_cast<const uint16_t*>(residual);
  a.out = static_cast<uint16_t*>(out);
  a.h = static_cast<uint16_t*>(ws);
  a.y = reinterpret_cast<float*>(static_cast<char*>(ws) + moe_h_bytes(d));
  a.tokens = d.tokens;
  a.hidden = d.hidden;
  a.inter = d.inter;
  a.experts = d.num_experts;
  a.top_k = d.top_k;
  a.activation = d.activation;
  if ((e = pda::launch_experts(a, plan, st)) != hipSuccess) return hip_fail(e, "experts kernel launch");
  return PDA_OK;
}

int pda_moe_workspace_reserve(const pda_moe_dims* dims, void* stream) {
  g_err.clear();
  int rc = check_moe(dims);
  if (rc) return rc;
  if (dims->tokens == 0) return PDA_OK;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  if ((rc = device_cus(dev, &cus))) return rc;
  void* ptr = nullptr;
  const int64_t need = moe_ws_bytes(*dims, cus);
  return workspace_for(dev, static_cast<hipStream_t>(stream), need, need, &ptr);
}

int pda_moe_plan(const pda_moe_dims* dims, int32_t num_cus, pda_experts* out) {
  g_err.clear();
  if (!out) return fail(PDA_ERR_NULL, "pda_moe_plan: NULL output pointer");
  int rc = check_moe(dims);
  if (rc) return rc;
  if (num_cus <= 0) return fail(PDA_ERR_SHAPE, "num_cus must be positive");
  *out = pda_experts{};
  if (dims->tokens == 0) return PDA_OK;
  const pda::ExpertsPlan p = moe_plan(*dims, num_cus);
  out->shared_up = p.shared_up;
  out->shared_down = p.shared_down;
  out->joined = p.joined;
  out->k_splits = p.splits;
  out->call_bytes = moe_call_bytes(*dims, p);
  out->workspace_bytes = moe_ws_bytes(*dims, num_cus);
  return PDA_OK;
}

int pda_block_norm(const void* y, const void* residual, const void* post_w, const void* pre_w, const void* gate,
                   void* residual_out, void* normed_out, const pda_block_norm_dims* dims, void* stream) {
  g_err.clear();
  if (!dims) return fail(PDA_ERR_NULL, "dims is NULL");
  const pda_block_norm_dims& d = *dims;
  if (d.rows < 0) return fail(PDA_ERR_SHAPE, "rows must be >= 0 (got %d)", d.rows);
  if (d.rows > pda::kMaxNormRows) return fail(PDA_ERR_UNSUPPORTED, "rows %d exceeds %d", d.rows, pda::kMaxNormRows);
  if (d.hidden <= 0) return fail(PDA_ERR_SHAPE, "hidden must be positive");
  if (d.hidden % 8 || d.hidden > 32768)
    return fail(PDA_ERR_UNSUPPORTED, "hidden %d (supported: multiples of 8 up to 32768)", d.hidden);
  if (d.gate_rows != 0 && d.gate_rows != 1) return fail(PDA_ERR_SHAPE, "gate_rows must be 0 or 1");
  if (!std::isfinite(d.scale) || !std::isfinite(d.weight_offset) || !std::isfinite(d.eps) || d.eps < 0.f)
    return fail(PDA_ERR_SCALE, "scale, weight_offset and eps must be finite and eps >= 0");
  if (d.rows == 0) return PDA_OK;
  if ((pre_w == nullptr) != (normed_out == nullptr))
    return fail(PDA_ERR_NULL, "pre_w and normed_out must both be given or both be NULL");
  if (!y || !residual_out) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  for (const void* p : {y, residual, post_w, pre_w, gate, static_cast<const void*>(residual_out),
                        static_cast<const void*>(normed_out)})
    if (misaligned(p, 2)) return fail(PDA_ERR_ALIGN, "bf16 arrays must be 2-byte aligned");
  const int64_t all = int64_t{2} * d.rows * d.hidden, one = int64_t{2} * d.hidden;
  const Extent post{"post_w", post_w, one}, pre{"pre_w", pre_w, one}, g{"gate", gate, d.gate_rows ? all : one};
  for (const Extent& o : {Extent{"residual_out", residual_out, all}, Extent{"normed_out", normed_out, all}}) {
    const int rc = check_apart(o, {{"y", o.p == y ? nullptr : y, all}, {"residual", o.p == residual ? nullptr : residual, all},
                                   post, pre, g});
    if (rc) return rc;
  }
  if (overlaps(residual_out, all, normed_out, all)) return fail(PDA_ERR_LAYOUT, "normed_out overlaps residual_out");
  pda::BlockNormArgs a;
  a.y = static_cast<const uint16_t*>(y);
  a.residual = static_cast<const uint16_t*>(residual);
  a.post_w = static_cast<const uint16_t*>(post_w);
  a.pre_w = static_cast<const uint16_t*>(pre_w);
  a.gate = static_cast<const uint16_t*>(gate);
  a.z = static_cast<uint16_t*>(residual_out);
  a.h = static_cast<uint16_t*>(normed_out);
  a.gate_stride = d.gate_rows ? d.hidden : 0;
  a.rows = d.rows;
  a.hidden = d.hidden;
  a.scale = d.scale;
  a.weight_offset = d.weight_offset;
  a.eps = d.eps;
  hipError_t e = pda::launch_block_norm(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "block norm kernel launch");
  return PDA_OK;
}

int pda_prelude_plan(const pda_prelude_dims* dims, int32_t qk_norm, int32_t num_cus, pda_projection* out) {
  g_err.clear();
  if (!out) return fail(PDA_ERR_NULL, "pda_prelude_plan: NULL output pointer");
  int rc = check_prelude(dims);
  if (rc) return rc;
  if (num_cus <= 0) return fail(PDA_ERR_SHAPE, "num_cus must be positive");
  *out = pda_projection{};
  if (dims->batch == 0) return PDA_OK;
  const pda_prelude_dims& d = *dims;
  const pda::RowsPlan plan =
      pda::plan_rows(d.batch, static_cast<int>(prelude_rows(d)), d.hidden, num_cus,
                     prelude_fusable(qk_norm != 0, d.interleaved != 0, d.rotary_dim), pda::kMaxRowsSplits);
  *out = projection(plan, prelude_ws_bytes(d, num_cus));
  return PDA_OK;
}

int pda_profile_read_o_proj(double* gemv_ms, double* epilogue_ms, int64_t* calls) {
  g_err.clear();
  if (!gemv_ms || !epilogue_ms || !calls) return fail(PDA_ERR_NULL, "pda_profile_read_o_proj: NULL output pointer");
  return prof_read(2, gemv_ms, epilogue_ms, calls);
}

int pda_validate_paging(const int32_t* block_table, const int32_t* context_lens, int32_t batch,
                        int32_t max_pages_per_seq, int32_t page_size, int32_t num_pages, void* stream) {
  g_err.clear();
  if (batch < 0 || max_pages_per_seq <= 0 || page_size <= 0 || num_pages <= 0)
    return fail(PDA_ERR_SHAPE, "batch, max_pages_per_seq, page_size and num_pages out of range");
  if (batch == 0) return PDA_OK;
  if (!block_table || !context_lens) return fail(PDA_ERR_NULL, "a tensor pointer is NULL");
  if (static_cast<int64_t>(batch) * max_pages_per_seq > (int64_t{1} << 31))
    return fail(PDA_ERR_SHAPE, "block_table too large to validate");
  return validate_paging(block_table, context_lens, batch, max_pages_per_seq, page_size, num_pages, Touched{},
                         static_cast<hipStream_t>(stream));
}

int pda_prelude_workspace_reserve(const pda_prelude_dims* dims, void* stream) {
  g_err.clear();
  int rc = check_prelude(dims);
  if (rc) return rc;
  if (dims->batch == 0) return PDA_OK;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  if ((rc = device_cus(dev, &cus))) return rc;
  void* ptr = nullptr;
  const int64_t need = prelude_ws_bytes(*dims, cus);
  return workspace_for(dev, static_cast<hipStream_t>(stream), need, need, &ptr);
}

int paged_decode_attention_sink(const void* q, const void* k_cache, const void* v_cache, const int32_t* block_table,
                                const int32_t* context_lens, void* out, int32_t batch, int32_t num_q_heads,
                                int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t num_pages,
                                int32_t max_pages_per_seq, int32_t num_queries, int32_t window, int32_t num_sinks,
                                float scale, void* stream) {
  return attention_call(q, k_cache, v_cache, block_table, context_lens, out, batch, num_q_heads, num_kv_heads, head_dim,
                        page_size, num_pages, max_pages_per_seq, num_queries, window, scale, stream, false, num_sinks);
}

int paged_decode_attention_kv4(const void* q, const void* k_codes, const void* k_scales, const void* v_codes,
                               const void* v_scales, const int32_t* block_table, const int32_t* context_lens, void* out,
                               int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                               int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq, int32_t num_queries,
                               int32_t window, int32_t num_sinks, float scale, void* stream) {
  pda::Kv4Args c = {};
  c.k = static_cast<uint8_t*>(const_cast<void*>(k_codes));
  c.ks = static_cast<uint8_t*>(const_cast<void*>(k_scales));
  c.v = static_cast<uint8_t*>(const_cast<void*>(v_codes));
  c.vs = static_cast<uint8_t*>(const_cast<void*>(v_scales));
  return attention_call(q, k_codes, v_codes, block_table, context_lens, out, batch, num_q_heads, num_kv_heads, head_dim,
                        page_size, num_pages, max_pages_per_seq, num_queries, window, scale, stream, false, num_sinks, &c);
}

int pda_pages_update(const int32_t* block_table, const int32_t* context_lens, const int32_t* parents,
                     const int32_t* new_lens, const int32_t* refcount, int32_t* table_out, int32_t* refcount_out,
                     int32_t* copy_src, int32_t* copy_dst, int32_t* info, int32_t batch, int32_t rows, int32_t page_size,
                     int32_t num_pages, int32_t max_pages_per_seq, int32_t num_queries, int32_t window, int32_t num_sinks,
                     void* stream) {
  g_err.clear();
  int rc = check_pages(batch, rows, page_size, num_pages, max_pages_per_seq);
  if (rc) return rc;
  if (num_queries < 1) return fail(PDA_ERR_SHAPE, "num_queries must be >= 1 (got %d)", num_queries);
  if (window < 0 || num_sinks < 0)
    return fail(PDA_ERR_SHAPE, "window and num_sinks must be >= 0 (got %d, %d)", window, num_sinks);
  const int64_t table = static_cast<int64_t>(batch) * max_pages_per_seq;
  const Span spans[] = {{"block_table", block_table, table}, {"context_lens", context_lens, batch},
                        {"parents", parents, parents ? rows : 0}, {"new_lens", new_lens, rows},
                        {"refcount", refcount, num_pages}, {"table_out", table_out, static_cast<int64_t>(rows) * max_pages_per_seq},
                        {"refcount_out", refcount_out, num_pages}, {"copy_src", copy_src, rows},
                        {"copy_dst", copy_dst, rows}, {"info", info, 2}};
  if ((rc = check_spans(spans, 5))) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  void* ws = nullptr;
  const int64_t need = update_ws_bytes(rows, num_pages);
  if ((rc = workspace_for(dev, st, need, need, &ws))) return rc;
  pda::PagesUpdateArgs a;
  a.table = block_table;
  a.lens = context_lens;
  a.parents = parents;
  a.new_lens = new_lens;
  a.refcount = refcount;
  a.table_out = table_out;
  a.refcount_out = refcount_out;
  a.src = copy_src;
  a.dst = copy_dst;
  a.info = info;
  a.writer = static_cast<int32_t*>(ws);
  a.fresh = a.writer + num_pages;
  a.start = a.fresh + num_pages;
  a.written = a.start + rows;
  a.grows = a.written + rows;
  a.cnt = a.grows + rows;
  a.batch = batch;
  a.rows = rows;
  a.page_shift = log2i(page_size);
  a.num_pages = num_pages;
  a.maxp = max_pages_per_seq;
  a.nq = num_queries;
  a.window = window;
  a.sinks = num_sinks;
  if ((e = pda::launch_pages_update(a, st)) != hipSuccess) return hip_fail(e, "page update launch");
  return PDA_OK;
}

int pda_pages_compact(const int32_t* block_table, const int32_t* context_lens, const int32_t* refcount, int32_t* table_out,
                      int32_t* refcount_out, int32_t* page_map, int32_t* copy_src, int32_t* copy_dst, int32_t* info,
                      int32_t batch, int32_t page_size, int32_t num_pages, int32_t max_pages_per_seq, void* stream) {
  g_err.clear();
  int rc = check_pages(batch, batch, page_size, num_pages, max_pages_per_seq);
  if (rc) return rc;
  const int64_t table = static_cast<int64_t>(batch) * max_pages_per_seq;
  const Span spans[] = {{"block_table", block_table, table}, {"context_lens", context_lens, batch},
                        {"refcount", refcount, num_pages}, {"table_out", table_out, table},
                        {"refcount_out", refcount_out, num_pages}, {"page_map", page_map, num_pages},
                        {"copy_src", copy_src, num_pages}, {"copy_dst", copy_dst, num_pages}, {"info", info, 2}};
  if ((rc = check_spans(spans, 3))) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  void* ws = nullptr;
  const int64_t need = compact_ws_bytes(num_pages);
  if ((rc = workspace_for(dev, st, need, need, &ws))) return rc;
  pda::PagesCompactArgs a;
  a.table = block_table;
  a.lens = context_lens;
  a.refcount = refcount;
  a.table_out = table_out;
  a.refcount_out = refcount_out;
  a.map = page_map;
  a.src = copy_src;
  a.dst = copy_dst;
  a.info = info;
  a.place = static_cast<int32_t*>(ws);
  a.ranked = a.place + num_pages;
  a.counts = a.ranked + num_pages;
  a.batch = batch;
  a.page_shift = log2i(page_size);
  a.num_pages = num_pages;
  a.maxp = max_pages_per_seq;
  if ((e = pda::launch_pages_compact(a, st)) != hipSuccess) return hip_fail(e, "page compaction launch");
  return PDA_OK;
}

int pda_pages_copy(const pda_pool* pools, int32_t num_pools, const int32_t* copy_src, const int32_t* copy_dst,
                   const int32_t* count, int32_t max_copies, int32_t num_pages, void* stream) {
  g_err.clear();
  if (num_pools < 0 || max_copies < 0)
    return fail(PDA_ERR_SHAPE, "num_pools and max_copies must be >= 0 (got %d, %d)", num_pools, max_copies);
  if (num_pages <= 0) return fail(PDA_ERR_SHAPE, "num_pages must be positive (got %d)", num_pages);
  if (num_pools == 0 || max_copies == 0) return PDA_OK;
  if (!pools || !copy_src || !copy_dst) return fail(PDA_ERR_NULL, "a pointer is NULL");
  if (misaligned(copy_src, 4) || misaligned(copy_dst, 4) || misaligned(count, 4))
    return fail(PDA_ERR_ALIGN, "copy_src, copy_dst and count must be 4-byte aligned");
  for (int32_t i = 0; i < num_pools; ++i) {
    const pda_pool& p = pools[i];
    if (!p.data) return fail(PDA_ERR_NULL, "pool %d is NULL", i);
    if (p.page_bytes <= 0 || p.page_bytes > (int64_t{1} << 30))
      return fail(PDA_ERR_SHAPE, "pool %d: page_bytes %lld outside [16, 2^30]", i, static_cast<long long>(p.page_bytes));
    if (misaligned(p.data, 16) || p.page_bytes % 16)
      return fail(PDA_ERR_ALIGN, "pool %d must be 16-byte aligned, its pages a multiple of 16 bytes", i);
    if (static_cast<int64_t>(max_copies) * pda::kMaxCopyPools * pda::pages_copy_parts(p.page_bytes) >= (int64_t{1} << 31))
      return fail(PDA_ERR_UNSUPPORTED, "max_copies %d of pages of %lld bytes", max_copies, static_cast<long long>(p.page_bytes));
  }
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  int cus = 0;
  const int rc = device_cus(dev, &cus);
  if (rc) return rc;
  for (int32_t at = 0; at < num_pools; at += pda::kMaxCopyPools) {
    pda::PagesCopyArgs a = {};
    a.pools = std::min(pda::kMaxCopyPools, num_pools - at);
    int64_t most = 0;
    for (int i = 0; i < a.pools; ++i) {
      a.pool[i].data = static_cast<char*>(pools[at + i].data);
      a.pool[i].bytes = pools[at + i].page_bytes;
      most = std::max(most, pools[at + i].page_bytes);
    }
    a.src = copy_src;
    a.dst = copy_dst;
    a.count = count;
    a.most = max_copies;
    a.num_pages = num_pages;
    if ((e = pda::launch_pages_copy(a, most, cus, static_cast<hipStream_t>(stream))) != hipSuccess)
      return hip_fail(e, "page copy launch");
  }
  return PDA_OK;
}

int pda_pages_workspace_reserve(int32_t rows, int32_t num_pages, void* stream) {
  g_err.clear();
  if (rows < 0 || rows > PDA_MAX_BATCH) return fail(PDA_ERR_SHAPE, "rows must be in [0, %d] (got %d)", PDA_MAX_BATCH, rows);
  if (num_pages <= 0 || num_pages > pda::kMaxPoolPages)
    return fail(PDA_ERR_SHAPE, "num_pages must be in [1, %d] (got %d)", pda::kMaxPoolPages, num_pages);
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  void* ptr = nullptr;
  const int64_t need = std::max(update_ws_bytes(rows, num_pages), compact_ws_bytes(num_pages));
  return workspace_for(dev, static_cast<hipStream_t>(stream), need, need, &ptr);
}

int pda_kv4_append(const void* k_new, const void* v_new, void* k_codes, void* k_scales, void* v_codes, void* v_scales,
                   const int32_t* block_table, const int32_t* context_lens, int32_t batch, int32_t num_tokens,
                   int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t num_pages,
                   int32_t max_pages_per_seq, void* stream) {
  pda::Kv4Args c;
  const int rc = check_kv4_tokens(&c, k_new, v_new, k_codes, k_scales, v_codes, v_scales, block_table, context_lens, batch,
                                  num_tokens, num_kv_heads, head_dim, page_size, num_pages, max_pages_per_seq, stream);
  if (rc || batch == 0) return rc;
  const hipError_t e = pda::launch_kv4_append(c, static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new),
                                              static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PDA_OK : hip_fail(e, "append kernel launch");
}

int pda_kv4_read(void* k_out, void* v_out, const void* k_codes, const void* k_scales, const void* v_codes,
                 const void* v_scales, const int32_t* block_table, const int32_t* context_lens, int32_t batch,
                 int32_t num_tokens, int32_t num_kv_heads, int32_t head_dim, int32_t page_size, int32_t num_pages,
                 int32_t max_pages_per_seq, void* stream) {
  pda::Kv4Args c;
  const int rc = check_kv4_tokens(&c, k_out, v_out, k_codes, k_scales, v_codes, v_scales, block_table, context_lens, batch,
                                  num_tokens, num_kv_heads, head_dim, page_size, num_pages, max_pages_per_seq, stream);
  if (rc || batch == 0) return rc;
  const hipError_t e = pda::launch_kv4_read(c, static_cast<uint16_t*>(k_out), static_cast<uint16_t*>(v_out),
                                            static_cast<hipStream_t>(stream));
  return e == hipSuccess ? PDA_OK : hip_fail(e, "read kernel launch");
}

}  // extern "C"
