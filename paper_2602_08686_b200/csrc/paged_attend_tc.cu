// Attention of longer chunks over the pages: bf16 on the tensor cores (tcgen05 + TMA), one persistent CTA per SM.
//
// An item is up to two tiles of 128 query rows of one (unit, KV head): a tile holds whole tokens, row = token * G + head, so one TMA
// box {G heads, 128 / G tokens} of q is a K-major operand.  Keys and values come in tiles of 128 rows, one TMA box per page and
// 64-dimension half, into a ring of five 32 KB stages (K0 V0 K1 V1 ...), and are worked on in steps of 64.  Per step and query
// tile s ("stream"):
//   S = Q_s K^T       M = 128, N = 64, K = 128, into one of the stream's two buffers of 64 TMEM columns
//   P = 2^(x - m)     one thread per row: a row's 64 logits are one thread's registers, so nothing is shuffled; P goes back as
//                     bf16 over the columns S came from (the rounding tensor cores want; the sum l is of the unrounded values)
//   O_s += P V        A = P from TMEM, V as it lies in memory ([keys][dims], MN-major B), into 128 TMEM columns
// With two buffers a stream's logits are a step ahead of its softmax, so that the softmax threads do not wait for the tensor
// cores (512 TMEM columns hold two streams' outputs and four 64-column buffers, or two of 128: with those the two took turns).
// N = 64 costs the first product half as much again (48 clocks for 32 of arithmetic: A and B are read from shared memory at 128
// bytes a clock), 2600 clocks per key tile and pair of query tiles; the exponentials alone take 2050 (16 a clock).
// Bound: those two together, at the clocks the power limit leaves under them (1.4 to 1.6 GHz).  2048 tokens over 32k rows:
// 2.0 us per key tile and 918 us after a rest (1.24 PFLOP/s, 77 % of the measured rate of a plain matrix product), 1030 to 1060 us
// kept up (1.07 to 1.1, 80 % of that product's); at 8192 rows the
// tensor pipe is active 58 % of the time, and as much the exponentials' one.  An item takes 5 us besides its tiles: its last
// product, and its output, whose 32-byte pieces of 128 rows keep the store path busy (gathered to lines by shuffles
// they take 0.5 us less on two query tiles and more on one).
// No maximum is taken per step.  Any reference m gives the same softmax, up to overflow: P, l and O are floating-point, and a
// common factor costs none of their bits.  So a row keeps the reference of its first visible step, and the sums tell
// whether an exponential left the range (2^16: then, or where the reference itself is too far from zero to be exact, the maximum
// is taken, O is rescaled in TMEM and the step is done again).
// Warps 0-3 and 4-7: softmax of stream 0 and 1; warps 8, 9: their MMAs; warp 10: TMA; warp 11 walks the items ahead of the others.
// Every wait is bounded and reports CKV_ERR_TIMEOUT through the status word.
#include "paged_work.cuh"
#include "tc_ptx.cuh"

namespace ckv {
namespace {

using namespace ptx;

constexpr int kThreads = 384;
constexpr int kStages = 5;
constexpr int kTile = 128, kStep = 64;         // keys of a tile, and of a step
constexpr uint32_t kHalf = 128 * 128;          // 128 rows x 64 bf16
constexpr uint32_t kTileBytes = 2 * kHalf;
constexpr int kTcGranule = kBothTiles;         // least cost a CTA takes on (two tiles: 31 us instead of 27 for 40 tokens on 2048 rows)
constexpr int kInfo = 8;                       // ring of per-tile notes from the loader
constexpr int kJobs = 4;                       // ring of items
// A step's sum above it is done again with a new reference.  Sums and outputs of up to 2^24 rows (2^18 steps) then stay below 2^34 and
// 2^34 max|v|, in range for values up to 2^94 (the largest fp32 is 2^128).
constexpr float kOverflow = 65536.0f;
// A logit is off its own rounded product with the scale by up to 2^-24 of it: a factor of two where the reference is this far from zero.
constexpr float kFar = 16777216.0f;
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 4) << 24);   // fp32 += bf16 * bf16, M = 128
constexpr uint32_t kIdescQK = kIdesc | ((64u >> 3) << 17);
constexpr uint32_t kIdescPV = kIdesc | ((128u >> 3) << 17) | (1u << 16);                // B (the values) is MN-major
constexpr uint32_t kNegateA = 1u << 13;
constexpr uint32_t kColS = 0, kColO = 256;     // TMEM columns: two buffers of stream 0, of stream 1, O_0, O_1

struct TcArgs {
  WorkArgs w;
  float x_scale;         // |scale| * log2(e)
  uint32_t idesc_qk;     // with A negated where the scale is negative
  uint32_t q_bytes;      // of one query tile
  int TQ;                // tokens per query tile
  int pages_per_tile;    // 128 / page_size, at least 1
  uint32_t page_bytes;   // of one box: min(page_size, 128) rows of 128 bytes
  unsigned long long wait_ns;
  // the arrays themselves, for the rows that add_row fetches
  const __nv_bfloat16 *q, *k, *v;
  int64_t q_tok, q_head, page_stride, page_row;
  float signed_scale;    // scale * log2(e)
  __nv_bfloat16* out;
  float* lse;
};

// An item, as the roles need it.
struct Job {
  Item it;
  int pair, block;       // where it comes from
  int n;                 // key tiles (0: there are no more items)
  int tiles2;            // whether it has two query tiles
  int steps;             // of each stream
  int see;               // rows that every token of the block sees: those its first token does
  int whole;             // not a part
  int odd;               // some value rows have been zeroed that tokens see
};

struct __align__(1024) Smem {
  uint8_t kv[kStages][kTileBytes];
  uint8_t q[2][kTileBytes];
  uint64_t full[kStages], empty[kStages];
  uint64_t q_full, q_empty;
  uint64_t clean;                               // a value tile has been looked at
  uint64_t s_full[2][2], p_full[2][2], pv_done[2], item_done[2];   // [stream][buffer]
  uint64_t join_full, join_done;                // stream 1's result is there; stream 0 has read it
  uint64_t job_full[kJobs], job_empty[kJobs];
  Job jobs[kJobs];
  float2 other[kTile];                          // stream 1's maximum and sum per row
  uint32_t bad[kInfo];                          // which pages of a key tile are missing (bit per page)
  uint32_t odd[kInfo][4];                       // which rows of a value tile were not finite and have been zeroed
  Plan plan;
  uint32_t tmem_base;
  int abort_flag;
};
static_assert(sizeof(Smem) <= 232448, "shared memory of one CTA");

__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lead) { return ((addr >> 4) & 0x3fffu) | ((lead >> 4) << 16); }
__device__ __forceinline__ uint64_t desc_of(uint32_t lo) {   // 128-byte swizzle, groups of eight rows 1024 bytes apart
  constexpr uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);
  return ((uint64_t)hi << 32) | lo;
}

// All lanes of a warp wait and agree on the outcome (what follows is warp-wide).
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, const Waiter& w, int code) {
  return __all_sync(0xffffffffu, bar_wait(bar, parity, w, code));
}

// How an item is cut up.  Two query tiles: each stream has one, and takes both halves of every key tile.  One query tile (the
// tokens fill no more than half of the block): both streams work on it, each on its half of every key tile, and join at the end.
//
// One warp looks the items up for all (lengths, token counts, divisions: 2000 to 6000 clocks each where every warp did it between
// two items).
__device__ __forceinline__ void job_role(const TcArgs& a, Smem& sm, const Waiter& w, int lane) {
  Walk k;
  k.start(a.w, sm.plan);
  // this wait takes as long as an item does; the others are for one step's work
  const Waiter patient{w.abort_flag, w.status, 64 * w.limit_ns};
  for (uint32_t i = 0;; ++i) {
    if (!wait_warp(smem_u32(&sm.job_empty[i % kJobs]), ((i / kJobs) & 1) ^ 1, patient, 10)) return;
    if (lane == 0) {
      Job& job = sm.jobs[i % kJobs];
      job.n = 0;
      if (k.live) {
        const Item& it = k.it;
        job.it = it, job.pair = k.pair, job.block = k.block;
        job.n = it.t1 - it.t0, job.tiles2 = both_tiles(a.w, it.n, it.block), job.steps = job.tiles2 ? 2 * job.n : job.n;
        job.see = rows_seen(a.w, it.n, it.len, it.block * a.w.tokens + 1);
        job.whole = it.t0 == 0 && it.t1 == it.tiles;
        job.odd = 0;
      }
      bar_arrive(smem_u32(&sm.job_full[i % kJobs]));
    }
    if (!k.live) return;
    k.next(a.w, sm.plan);
  }
}
// The i-th item, for a warp that arrives on its `job_empty` when it is done with it; null: a wait has given up.
__device__ __forceinline__ Job* job_of(Smem& sm, uint32_t i, const Waiter& w) {
  return wait_warp(smem_u32(&sm.job_full[i % kJobs]), (i / kJobs) & 1, w, 11) ? &sm.jobs[i % kJobs] : nullptr;
}
__device__ __forceinline__ void job_done(Smem& sm, uint32_t i, int lane) {
  __syncwarp();
  if (lane == 0) bar_arrive(smem_u32(&sm.job_empty[i % kJobs]));
}

// First row of the item's j-th key tile that the block's first token does not see (128: it sees them all).  Where every
// token sees every row there is none.
__device__ __forceinline__ int late_row(const TcArgs& a, const Job& job, int j) {
  return a.w.causal ? min(max(job.see - (job.it.t0 + j) * kTile, 0), kTile) : kTile;
}

__device__ __forceinline__ void load_role(const TcArgs& a, Smem& sm, const CUtensorMap* qm, const CUtensorMap* km,
                                          const CUtensorMap* vm, const Waiter& w, int lane) {
  uint32_t n_loads = 0, n_tiles = 0;
  const int slot_of_lane = lane >> 1, half = lane & 1;
  const uint64_t first = evict_first();
  const bool copies = slot_of_lane < a.pages_per_tile;
  const int tiles_per_page = a.w.P > kTile ? a.w.P / kTile : 1;
  for (uint32_t n_items = 0;; ++n_items) {
    Job* job = job_of(sm, n_items, w);
    if (!job || job->n == 0) return;
    const Item& it = job->it;
    const int ns = job->tiles2 ? 2 : 1, t0 = it.t0, t1 = it.t1, visible = it.visible;
    // Keys and values that one block alone reads leave L2 first: what every call needs again (code, tables, lengths) is then not
    // streamed out of it, and the next call does not start with misses (49 us instead of 62 for 8 x 5 tokens on 16k).
    const bool once = it.n <= a.w.tokens;
    if (!wait_warp(smem_u32(&sm.q_empty), (n_items & 1) ^ 1, w, 1)) return;
    if (lane == 0) bar_arrive_tx(smem_u32(&sm.q_full), ns * a.q_bytes);
    __syncwarp();
    if (lane < 2 * ns)   // lane: (tile, half)
      tma_load_4d(qm, smem_u32(&sm.q[lane >> 1][(lane & 1) * kHalf]), smem_u32(&sm.q_full), 0, it.g * a.w.G,
                  it.first + it.block * a.w.tokens + (lane >> 1) * a.TQ, lane & 1);
    const int32_t* table = a.w.table + ((int64_t)it.u * a.w.Hkv + it.g) * a.w.max_pages;
    // the pages that hold visible rows of a tile, looked up a tile ahead
    auto row_of = [&](int t) { return t * kTile + slot_of_lane * (a.w.P < kTile ? a.w.P : kTile); };
    auto wants = [&](int t) { return copies && t < t1 && row_of(t) < visible; };
    int next_page = wants(t0) ? table[row_of(t0) >> a.w.log_p] : 0;
    for (int t = t0; t < t1; ++t, ++n_tiles) {
      const bool wanted = wants(t);
      const int page = next_page;
      if (wants(t + 1)) next_page = table[row_of(t + 1) >> a.w.log_p];
      const bool fine = (unsigned)page < (unsigned)a.w.n_pages;
      if (wanted && !fine && half == 0) report_status(a.w.status, kStatusPage);
      const bool copy = wanted && fine;
      const uint32_t bytes = a.page_bytes * __popc(__ballot_sync(0xffffffffu, copy));
      const uint32_t missing = __ballot_sync(0xffffffffu, wanted && !fine && half == 0);
      const int row_in_page = tiles_per_page > 1 ? (t & (tiles_per_page - 1)) * kTile : 0;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv, ++n_loads) {
        const uint32_t s = n_loads % kStages;
        if (!wait_warp(smem_u32(&sm.empty[s]), ((n_loads / kStages) & 1) ^ 1, w, 2)) return;
        if (lane == 0) {
          if (kv == 0) {
            uint32_t m = 0;
            for (uint32_t b = missing; b; b &= b - 1) m |= 1u << ((__ffs(b) - 1) >> 1);
            sm.bad[n_tiles % kInfo] = m;
          }
          bar_arrive_tx(smem_u32(&sm.full[s]), bytes);
        }
        __syncwarp();
        if (copy) {
          const uint32_t dst = smem_u32(&sm.kv[s][half * kHalf + slot_of_lane * a.page_bytes]);
          if (once) tma_load_4d_hint(kv ? vm : km, dst, smem_u32(&sm.full[s]), 0, row_in_page, half, page, first);
          else tma_load_4d(kv ? vm : km, dst, smem_u32(&sm.full[s]), 0, row_in_page, half, page);
        }
      }
    }
    job_done(sm, n_items, lane);
  }
}

// 0 * NaN is not 0: value rows that no query sees are zeroed, and so are rows with an infinity or a NaN that some of the
// block's tokens do not see yet (the softmax threads add those to the tokens that do).  Each MMA warp has half of the tile's
// rows; reads go out eight at a time (one warp, row by row: 3400 clocks, most of them ahead of the item's last product).
__device__ __forceinline__ void clean_values(const TcArgs& a, Smem& sm, Job& job, int j, uint32_t slot, uint32_t n_tiles,
                                             int s, int lane) {
  const int lo = s * kStep, hi = lo + kStep, valid = job.it.visible - (job.it.t0 + j) * kTile;
  const uint32_t bad = *(volatile uint32_t*)&sm.bad[n_tiles % kInfo];
  uint4* v = reinterpret_cast<uint4*>(sm.kv[slot]);
  uint32_t* odd = sm.odd[n_tiles % kInfo];
  if (lane < 2) odd[2 * s + lane] = 0u;
  __syncwarp();
  const int piece = (lane & 8) * kTile + (lane & 7);          // 16-byte piece lane & 15 of a row: its half, its place
  const int end = min(valid, hi);
#pragma unroll 1
  for (int r0 = max(late_row(a, job, j), lo); r0 < end; r0 += 16) {
    uint32_t hit = 0;                                         // bit i: the piece of row r0 + 2 i (+ 1) has an exponent of all ones
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = min(r0 + 2 * i + (lane >> 4), end - 1);
      const uint4 x = v[piece + row * 8];
      const uint32_t e = 0x7f807f80u;
      if (__vcmpeq2(x.x & e, e) | __vcmpeq2(x.y & e, e) | __vcmpeq2(x.z & e, e) | __vcmpeq2(x.w & e, e)) hit |= 1u << i;
    }
    if (!__any_sync(0xffffffffu, hit != 0u)) continue;
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      const int row = min(r0 + 2 * i + (lane >> 4), end - 1);
      const uint32_t any = __ballot_sync(0xffffffffu, hit >> i & 1u);
      if ((any >> (lane & 16)) & 0xffffu) {
        v[piece + row * 8] = make_uint4(0u, 0u, 0u, 0u);
        if ((lane & 15) == 0) atomicOr(&odd[row >> 5], 1u << (row & 31)), job.odd = 1;
      }
    }
  }
  if (valid < hi || bad)
    for (int e = lane; e < 2 * kStep * 8; e += 32) {
      const int row = lo + (e >> 3 & (kStep - 1)), at = (e >> 9) * kTile * 8 + row * 8 + (e & 7);
      if (row >= valid || (bad >> (row >> a.w.log_p) & 1)) v[at] = make_uint4(0u, 0u, 0u, 0u);
    }
  fence_async_smem();
  __syncwarp();
}

// Where the CTA is in the ring of stages.
struct Ring {
  uint32_t slot = 0, parity = 0;
  __device__ __forceinline__ void step() {
    if (++slot == kStages) slot = 0, parity ^= 1;
  }
};

// The products of one stream, by a warp of its own, step by step (64 keys) through two buffers.  A buffer's are issued in the
// order S, O, next S: the tensor pipe runs them in that order, so S may take the columns that O reads P from without
// waiting for it.
__device__ __forceinline__ void mma_role(const TcArgs& a, Smem& sm, uint32_t tmem, const Waiter& w, int s, int lane) {
  uint32_t n_tiles = 0, n_steps = 0, n_clean = 0;
  Ring ring;                              // of the item's first key tile; two stages per tile: K, V
  const uint32_t kv0 = smem_u32(sm.kv[0]), full0 = smem_u32(&sm.full[0]), empty0 = smem_u32(&sm.empty[0]);
  const uint32_t s_cols = tmem + kColS + s * 128, o_cols = tmem + kColO + s * 128;
  const uint32_t bar_s = smem_u32(&sm.s_full[s][0]), bar_p = smem_u32(&sm.p_full[s][0]);
  const uint32_t bar_o = smem_u32(&sm.pv_done[s]), bar_item = smem_u32(&sm.item_done[s]);
  for (uint32_t n_items = 0;; ++n_items) {
    Job* job = job_of(sm, n_items, w);
    if (!job || job->n == 0) return;
    const bool pair = job->tiles2;
    const int steps = job->steps;
    const uint32_t q_lo = desc_lo(smem_u32(sm.q[pair ? s : 0]), 16);
    const int j_clean = max(job->see / kTile - job->it.t0, 0);   // first tile whose values have to be looked at
    if (!wait_warp(smem_u32(&sm.q_full), n_items & 1, w, 4)) return;
    Ring kr = ring, vr = ring;
    vr.step();
    auto qk = [&](int g) {   // S = Q K^T of step g
      const int h = pair ? g & 1 : s;                          // which half of the tile's keys
      if ((!pair || h == 0) && !wait_warp(full0 + kr.slot * 8, kr.parity, w, 3)) return false;
      tc_fence_after();
      const uint32_t buf = (n_steps + g) & 1;
      if (elect()) {
        const uint32_t b = desc_lo(kv0 + kr.slot * kTileBytes + h * (kStep * 128), 16);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {   // 16 dimensions = 32 bytes of a 128-byte swizzled row; the second half is 16 KB on
          const uint32_t off = (kk & 3) * 2 + (kk >> 2) * (kHalf >> 4);
          mma_ss(s_cols + buf * kStep, desc_of(q_lo + off), desc_of(b + off), a.idesc_qk, kk > 0);
        }
        tc_commit(bar_s + buf * 8);
        if (!pair || h == 1) tc_commit(empty0 + kr.slot * 8);
        if (g == steps - 1) tc_commit(smem_u32(&sm.q_empty));
      }
      if (!pair || h == 1) kr.step(), kr.step();
      return true;
    };
    if (!qk(0) || (steps > 1 && !qk(1))) return;
    for (int g = 0; g < steps; ++g) {
      const int h = pair ? g & 1 : s, j = pair ? g >> 1 : g;
      if (!pair || h == 0) {   // a new tile of values
        if (!wait_warp(full0 + vr.slot * 8, vr.parity, w, 3)) return;
        if (j >= j_clean || *(volatile uint32_t*)&sm.bad[n_tiles % kInfo]) {
          clean_values(a, sm, *job, j, vr.slot, n_tiles, s, lane);
          if (lane == 0) bar_arrive(smem_u32(&sm.clean));
          if (!wait_warp(smem_u32(&sm.clean), n_clean & 1, w, 9)) return;
          ++n_clean;
        }
        ++n_tiles;
      }
      const uint32_t step = n_steps + g, buf = step & 1;
      if (!wait_warp(bar_p + buf * 8, (step >> 1) & 1, w, 5)) return;
      tc_fence_after();
      if (elect()) {           // O += P V
        const uint32_t b = desc_lo(kv0 + vr.slot * kTileBytes, kHalf) + h * 4 * (2048 >> 4);   // 64-dimension halves 16 KB apart
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)     // 16 keys = 16 rows of 128 bytes = 8 columns
          mma_ts(o_cols, s_cols + buf * kStep + kk * 8, desc_of(b + kk * (2048 >> 4)), kIdescPV, g > 0 || kk > 0);
        tc_commit(bar_o);
        if (!pair || h == 1) tc_commit(empty0 + vr.slot * 8);
        if (g == steps - 1) tc_commit(bar_item);
      }
      if (!pair || h == 1) vr.step(), vr.step();
      if (g + 2 < steps && !qk(g + 2)) return;
    }
    if (lane == 0) bar_arrive(bar_item);   // releases what clean_values wrote
    n_steps += steps;
    ring = kr;
    job_done(sm, n_items, lane);
  }
}

// The exponentials of a row's 64 logits, to TMEM as bf16; returns their sum.
__device__ __forceinline__ float softmax_step(const uint32_t (&s)[kStep], float scale, float ref, uint32_t p_addr) {
  uint64_t sum[2] = {0, 0};
  const uint64_t sc = pack2(scale, scale), mr = pack2(-ref, -ref);
  uint32_t p[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    float a, b;
    unpack2(fma2(pack2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), sc, mr), a, b);
    a = ex2(a), b = ex2(b);
    sum[i & 1] = add2(sum[i & 1], pack2(a, b));
    p[i] = bf16x2(a, b);
  }
  tmem_st32(p_addr, p);
  float a, b;
  unpack2(add2(sum[0], sum[1]), a, b);
  return a + b;
}
__device__ __forceinline__ float row_max(const uint32_t (&s)[kStep]) {
  float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < kStep; i += 8) {
#pragma unroll
    for (int c = 0; c < 4; ++c) mx[c] = max3(mx[c], __uint_as_float(s[i + 2 * c]), __uint_as_float(s[i + 2 * c + 1]));
  }
  return fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
}
__device__ __forceinline__ void scale_output(uint32_t o_addr, float f) {
#pragma unroll 1
  for (int c = 0; c < 8; ++c) {
    uint32_t o[16];
    tmem_ld16(o_addr + c * 16, o);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
    tmem_st16(o_addr + c * 16, o);
  }
  tmem_wait_st();
}

// O += 2^(x - m) v for one cache row, with the logit from the rows as they lie in memory; rows of the tile that do
// not see it (limit) are left as they are.
__device__ __noinline__ void add_row(const TcArgs& a, const Item& it, uint32_t o_addr, int key, int limit, int token, int head,
                                     float m) {
  const int page = a.w.table[((int64_t)it.u * a.w.Hkv + it.g) * a.w.max_pages + (key >> a.w.log_p)];
  if ((unsigned)page >= (unsigned)a.w.n_pages) return;
  const int64_t at = page * a.page_stride + (key & (a.w.P - 1)) * a.page_row;
  const bool sees = key < limit;
  float x = 0.f;
  if (sees) {
    const __nv_bfloat16* q = a.q + (it.first + token) * a.q_tok + (it.g * a.w.G + head) * a.q_head;
    for (int d = 0; d < kHeadDim; ++d) x = fmaf(__bfloat162float(q[d]), __bfloat162float(a.k[at + d]), x);
  }
  const float p = ex2(x * a.signed_scale - m);
  for (int c = 0; c < 4; ++c) {
    uint32_t o[32];
    tmem_ld32(o_addr + c * 32, o);
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (sees) o[i] = __float_as_uint(fmaf(p, __bfloat162float(a.v[at + c * 32 + i]), __uint_as_float(o[i])));
    tmem_st32(o_addr + c * 32, o);
  }
  tmem_wait_st();
}

__device__ __forceinline__ void softmax_role(const TcArgs& a, Smem& sm, uint32_t tmem, const Waiter& w, int stream, int quarter,
                                             int lane) {
  uint32_t n_steps = 0, n_all = 0, n_join = 0;              // steps of this stream so far; tiles; joins of the streams
  const int r = quarter * 32 + lane;                        // row of the query tile: token, head
  const int r_tok = r / a.w.G, r_head = r - r_tok * a.w.G;
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  const uint32_t s_addr = tmem + lanes + kColS + stream * 128, o_addr = tmem + lanes + kColO + stream * 128;
  const uint32_t bar_s = smem_u32(&sm.s_full[stream][0]), bar_p = smem_u32(&sm.p_full[stream][0]), bar_o = smem_u32(&sm.pv_done[stream]);
  for (uint32_t n_items = 0;; ++n_items) {
    Job* job = job_of(sm, n_items, w);
    if (!job || job->n == 0) return;
    const Item& it = job->it;
    const int n = job->n, t0 = it.t0;
    const bool pair = job->tiles2;
    const int steps = job->steps, q_tile = pair ? stream : 0;
    const int tok0 = it.block * a.w.tokens + q_tile * a.TQ;   // first token of the tile
    const int token = tok0 + r_tok;
    const bool live = r < a.TQ * a.w.G && token < it.n;
    auto limit_of = [&](int tk) { return rows_seen(a.w, it.n, it.len, tk + 1); };
    const int limit = live ? limit_of(token) : 0, least = limit_of(tok0);
    // rows of no token hold what shared memory held, or another unit's queries: above everything, they ask for no step again
    float m = live ? -INFINITY : INFINITY, l = 0.f;
    bool open = true;                                         // some row of the warp has no reference yet
    bool far = false;                                         // some row's reference is further from zero than its rounding allows
#pragma unroll 1
    for (int g = 0; g < steps; ++g, ++n_steps) {
      const int j = pair ? g >> 1 : g, h = pair ? g & 1 : stream;
      const int key0 = (t0 + j) * kTile + h * kStep;
      const uint32_t buf = n_steps & 1, s_buf = s_addr + buf * kStep;
      if (!wait_warp(bar_s + buf * 8, (n_steps >> 1) & 1, w, 6)) return;
      tc_fence_after();
      uint32_t s[kStep];
      tmem_ld64(s_buf, s);
      const uint32_t bad = *(volatile uint32_t*)&sm.bad[(n_all + j) % kInfo];
      if (key0 + kStep > least || bad) {
#pragma unroll
        for (int i = 0; i < kStep; ++i)
          if (key0 + i >= limit || (bad >> ((h * kStep + i) >> a.w.log_p) & 1)) s[i] = 0xff800000u;
      }
      // Rows that have seen nothing yet take their reference here; what O holds for them is zero.
      if (open) {
        const float top = row_max(s) * a.x_scale;
        if (m == -INFINITY) m = top;
        open = __any_sync(0xffffffffu, m == -INFINITY);
        far = __any_sync(0xffffffffu, live && m > -INFINITY && fabsf(m) > kFar);
      }
      float sum = softmax_step(s, a.x_scale, m == -INFINITY ? 0.f : m, s_buf);
      // Done again with the row's maximum as the reference where the sum has left the range, and with products rounded as the
      // reference is where that is far from zero.
      if (far || __any_sync(0xffffffffu, sum > kOverflow)) {
#pragma unroll
        for (int i = 0; i < kStep; ++i) s[i] = __float_as_uint(__uint_as_float(s[i]) * a.x_scale);
        const float top = fmaxf(m, row_max(s));
        const float f = top == -INFINITY ? 1.0f : ex2(m - top);
        m = top, l *= f;
        far = __any_sync(0xffffffffu, live && m > -INFINITY && fabsf(m) > kFar);
        if (g > 0) {   // the product of the step before; the one before that is done, or S would not be here
          if (!wait_warp(bar_o, (n_steps - 1) & 1, w, 7)) return;
          tc_fence_after();
          scale_output(o_addr, f);
        }
        sum = softmax_step(s, 1.0f, m == -INFINITY ? 0.f : m, s_buf);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bar_p + buf * 8);
      l += sum;
    }
    // the item's output: normalised, or a partial result for the join
    const bool whole = job->whole;
    const int which = t0 > 0 ? 0 : 1;
    const int64_t slot = ((int64_t)blockIdx.x * 2 + which) * a.w.slot_rows + q_tile * a.TQ * a.w.G + r;   // its row of the block
    const int64_t at = (int64_t)(it.first + token) * a.w.H + it.g * a.w.G + r_head;
    __nv_bfloat16* out = a.out + at * kHeadDim;
    float* part = a.w.o + slot * kHeadDim;
    if (!wait_warp(smem_u32(&sm.item_done[stream]), n_items & 1, w, 7)) return;
    tc_fence_after();
    // value rows that were left out because they are not finite, for the tokens that see them
    for (int j = n - 1; job->odd && j >= 0 && late_row(a, *job, j) < kTile; --j) {
      for (int x = pair ? 0 : 2 * stream; x < (pair ? 4 : 2 * stream + 2); ++x) {   // the stream's keys
        uint32_t odd = sm.odd[(n_all + j) % kInfo][x];
        for (; odd; odd &= odd - 1) add_row(a, it, o_addr, (t0 + j) * kTile + x * 32 + __ffs(odd) - 1, limit, token, r_head, m);
      }
    }
    n_all += n;
    // one query tile: stream 1 leaves its maximum and sum, stream 0 takes its output from TMEM (the same lanes, other columns)
    float f0 = 1.0f, f1 = 0.f;
    if (!pair) {
      if (stream == 1) {
        sm.other[r] = make_float2(m, l);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(smem_u32(&sm.join_full));
        if (!wait_warp(smem_u32(&sm.join_done), n_join & 1, w, 8)) return;
        tc_fence_after();
        ++n_join;
        job_done(sm, n_items, lane);
        continue;
      }
      if (!wait_warp(smem_u32(&sm.join_full), n_join & 1, w, 8)) return;
      tc_fence_after();
      ++n_join;
      const float2 x = sm.other[r];
      const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
      f0 = ex2(m - ref), f1 = ex2(x.x - ref);
      l = l * f0 + x.y * f1, m = top;
    }
    const bool joined = !pair;
    const bool none = l == 0.f;   // nothing seen (a NaN sum is not nothing)
    const float inv = none ? 0.f : 1.0f / l;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uint32_t o[32];
      tmem_ld32(o_addr + c * 32, o);
      if (joined) {
        uint32_t o1[32];
        tmem_ld32(o_addr + 128 + c * 32, o1);
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f0 + __uint_as_float(o1[i]) * f1);
      }
      if (!live) continue;
      if (whole) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e)
            p[e] = none ? 0u : bf16x2(__uint_as_float(o[16 * i + 2 * e]) * inv, __uint_as_float(o[16 * i + 2 * e + 1]) * inv);
          st_global32(out + c * 32 + i * 16, p);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = o[8 * i + e];
          st_global32(part + c * 32 + i * 8, p);
        }
      }
    }
    if (live) {
      if (!whole) a.w.ml[slot] = make_float2(m, l);
      else if (a.lse) a.lse[at] = none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    }
    tc_fence_before();   // O is read before the streams' next P is announced
    if (joined) {
      __syncwarp();
      if (lane == 0) bar_arrive(smem_u32(&sm.join_done));
    }
    if (!whole && r == 0 && stream == 0) {
      int* sp = reinterpret_cast<int*>(a.w.split + blockIdx.x);
      sp[2 * which] = job->pair, sp[2 * which + 1] = job->block;
    }
    job_done(sm, n_items, lane);
  }
}

__global__ void __launch_bounds__(kThreads, 1) attend_tc_kernel(const __grid_constant__ CUtensorMap qm,
                                                                const __grid_constant__ CUtensorMap km,
                                                                const __grid_constant__ CUtensorMap vm,
                                                                const __grid_constant__ TcArgs a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::);
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) bar_init(smem_u32(&sm.full[i]), 1), bar_init(smem_u32(&sm.empty[i]), 2);
    bar_init(smem_u32(&sm.q_full), 1), bar_init(smem_u32(&sm.q_empty), 2), bar_init(smem_u32(&sm.clean), 2);
    for (int s = 0; s < 2; ++s) {
      bar_init(smem_u32(&sm.pv_done[s]), 1), bar_init(smem_u32(&sm.item_done[s]), 2);
      for (int b = 0; b < 2; ++b) bar_init(smem_u32(&sm.s_full[s][b]), 1), bar_init(smem_u32(&sm.p_full[s][b]), 4);
    }
    bar_init(smem_u32(&sm.join_full), 4), bar_init(smem_u32(&sm.join_done), 4);
    for (int i = 0; i < kJobs; ++i) bar_init(smem_u32(&sm.job_full[i]), 1), bar_init(smem_u32(&sm.job_empty[i]), 11);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    sm.abort_flag = 0;
  }
  if (warp == 10 && lane == 0) prefetch_map(&qm), prefetch_map(&km), prefetch_map(&vm);
  tc_fence_before();
  pdl_wait();
  make_plan<kThreads>(a.w, blockIdx.x, gridDim.x, sm.plan);
  pdl_launch_dependents();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  if (threadIdx.x == 0) a.w.split[blockIdx.x] = make_int4(-1, -1, -1, -1);
  __syncthreads();
  const Waiter w{&sm.abort_flag, a.w.status, a.wait_ns};
  if (warp < 8) softmax_role(a, sm, tmem, w, warp >> 2, warp & 3, lane);
  else if (warp < 10) mma_role(a, sm, tmem, w, warp - 8, lane);
  else if (warp == 10) load_role(a, sm, &qm, &km, &vm, w, lane);
  else job_role(a, sm, w, lane);
  tc_fence_before();
  __syncthreads();
  if (sm.abort_flag) {   // a wait gave up: let copies and products in flight land before the memory is given back
    const unsigned long long t0 = now_ns();
    while (now_ns() - t0 < 1000000ull) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
  }
}

// ------------------------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess ||
        qres != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}
// Rank-4 map of rows of 128 bf16 split into two 64-element halves: {64, n1 (stride s1), n2 (stride s2)} and the halves as one
// of the outer dimensions; a dimension of extent one gets a legal stride whatever the caller's is.
bool make_map(CUtensorMap* map, const void* base, cuuint64_t n1, int64_t s1, cuuint64_t n2, int64_t s2, bool half_third,
              cuuint32_t box1, cuuint32_t box2) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t b1 = n1 == 1 ? 256 : (cuuint64_t)s1 * 2, b2 = n2 == 1 ? 256 : (cuuint64_t)s2 * 2;
  const cuuint64_t dims_h[4] = {64, n1, 2, n2}, dims_l[4] = {64, n1, n2, 2};
  const cuuint64_t str_h[3] = {b1, 128, b2}, str_l[3] = {b1, b2, 128};
  const cuuint32_t box_h[4] = {64, box1, 1, box2}, box_l[4] = {64, box1, box2, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), half_third ? dims_h : dims_l,
            half_third ? str_h : str_l, half_third ? box_h : box_l, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_attend_tc(const ckv_paged& pg, const WorkArgs& base, int64_t most, float scale, const void* q, const void* k_pages,
                             const void* v_pages, void* out, float* lse, cudaStream_t st) {
  TcArgs a{};
  a.w = base;
  a.TQ = kTile / base.G;
  set_blocks(a.w, most, 2 * a.TQ * base.G, 2 * a.TQ, kTile, kTcGranule);
  a.x_scale = (scale < 0.f ? -scale : scale) * kLog2e;
  a.idesc_qk = kIdescQK | (scale < 0.f ? kNegateA : 0u);
  a.q_bytes = 2u * (uint32_t)(a.TQ * base.G) * 128u;
  const int rows = base.P < kTile ? base.P : kTile;
  a.pages_per_tile = kTile / rows, a.page_bytes = (uint32_t)rows * 128u;
  a.wait_ns = wait_limit_ns();
  a.q = static_cast<const __nv_bfloat16*>(q), a.k = static_cast<const __nv_bfloat16*>(k_pages);
  a.v = static_cast<const __nv_bfloat16*>(v_pages);
  a.q_tok = pg.q_stride_tok, a.q_head = pg.q_stride_head, a.page_stride = pg.page_stride, a.page_row = pg.page_stride_row;
  a.signed_scale = scale * kLog2e;
  a.out = static_cast<__nv_bfloat16*>(out), a.lse = lse;
  CUtensorMap qm, km, vm;
  if (!make_map(&qm, q, pg.n_q_heads, pg.q_stride_head, pg.n_tokens, pg.q_stride_tok, false, base.G, a.TQ) ||
      !make_map(&km, k_pages, pg.page_size, pg.page_stride_row, pg.n_pages, pg.page_stride, true, rows, 1) ||
      !make_map(&vm, v_pages, pg.page_size, pg.page_stride_row, pg.n_pages, pg.page_stride, true, rows, 1))
    return cudaErrorInvalidValue;
  static PerDevice ready;
  cudaError_t e = ready.once([] {
    return cudaFuncSetAttribute(attend_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(kWorkers), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = sizeof(Smem), cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, attend_tc_kernel, qm, km, vm, a);
  count_launch();
  if (e != cudaSuccess) return e;
  return launch_join<true>(a.w, kWorkers, (int)(most * base.G < a.w.M ? most * base.G : a.w.M), out, lse, st);
}

}  // namespace ckv
