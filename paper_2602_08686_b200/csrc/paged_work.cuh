// Work schedule of the attention over pages, and the join of split results.
//
// An item is one block of query rows of one (unit, KV head): the rows r = token * G + head of the unit's tokens and the
// group's G query heads, `M` of them.  Its cost is the number of key tiles its last token sees (at least one, so that rows
// that see nothing are written too), times what a tile of it takes.  Lengths and token counts
// live on the device, so the split is made there: every worker (CTA) adds up the costs, takes an equal share of the total
// and works through the items in it; a tile belongs to the share its cost begins in.  The first item may have been begun by the
// worker before, the last may be finished by the next: those two
// leave unnormalised partial results in the worker's two slots, and join_kernel adds up what belongs together in worker
// order (the result does not depend on timing).
#pragma once
#include "paged.cuh"

namespace ckv {

struct WorkArgs {
  int Nu, H, Hkv, G, T, causal;
  int M;            // query rows of a block
  int blocks;       // blocks a pair is expected to have (clusters)
  int tokens;       // 0, or the whole tokens a block holds (then M is tokens * G)
  int tile, log_tile;   // keys per tile
  int granule;      // least cost per worker (a tile, where that costs more)
  int rounds;       // whether to hand out whole items first (units may have several blocks, which share keys and values)
  int one_warp;     // few pairs of few blocks each: one warp makes the schedule
  int P, log_p, n_pages, max_pages;
  const int32_t *starts, *lengths, *table;
  int* status;
  int4* split;      // [workers]: (pair, block) in slot 0 (begun by an earlier worker) and slot 1 (not finished), or -1
  float2* ml;       // [workers][2][slot_rows]
  float* o;         // [workers][2][slot_rows][128]
  int slot_rows;
};

// Block and tile sizes of a kernel; units have at most `most` tokens.
constexpr int kWarpPairs = 128, kWarpBlocks = 8;
inline void set_blocks(WorkArgs& a, int64_t most, int M, int tokens, int tile, int granule) {
  a.M = M, a.tokens = tokens, a.tile = tile, a.granule = granule;
  for (a.log_tile = 0; (1 << a.log_tile) < tile;) ++a.log_tile;
  const int64_t blocks = (most * a.G + M - 1) / M;
  a.blocks = (int)(blocks < 1 ? 1 : blocks > 4096 ? 4096 : blocks);
  a.rounds = tokens > 0 && most > tokens;
  a.one_warp = (int64_t)a.Nu * a.Hkv <= kWarpPairs && !a.rounds && most * a.G <= (int64_t)kWarpBlocks * M;
}

struct Item {
  int u, g, block;       // block of rows
  int first, n, len;     // the unit's first token and token count; the head's length
  int rows;              // query rows of the unit (n * G)
  int visible;           // rows the block's last token sees
  int tiles;             // tiles of the whole item
  int weight;            // cost of each
  int t0, t1;            // this worker's part
};

__device__ __forceinline__ int unit_blocks(const WorkArgs& a, int n) {
  const int per = a.tokens ? a.tokens : a.M, units = a.tokens ? n : n * a.G;   // at most 2^30 rows (checked on the host)
  return units <= per ? (units > 0) : (units + per - 1) / per;
}
// The head's length; one that the table has no pages for is reported (the rows without a page are left out, see rows_seen), and so
// is one below zero, which counts as zero.
__device__ __forceinline__ int head_length(const WorkArgs& a, int pair) {
  const int len = a.lengths[pair];
  if (len < 0 || len > a.max_pages << a.log_p) report_status(a.status, kStatusPage);
  return max(len, 0);
}
// Rows of the cache that the unit's first `tokens` tokens see between them: those that the last of them sees.
__device__ __forceinline__ int rows_seen(const WorkArgs& a, int n, int len, int tokens) {
  return min(a.causal ? max(len - n + min(tokens, n), 0) : len, a.max_pages << a.log_p);
}
// rows that the last token of a block sees
__device__ __forceinline__ int block_visible(const WorkArgs& a, int n, int len, int block) {
  return rows_seen(a, n, len, a.tokens ? (block + 1) * a.tokens : ((block + 1) * a.M >= n * a.G ? n : ((block + 1) * a.M + a.G - 1) / a.G));
}
__device__ __forceinline__ int tiles_of(const WorkArgs& a, int visible) { return max((visible + a.tile - 1) >> a.log_tile, 1); }

// Whether a block of two tiles of query rows has rows in both.
__device__ __forceinline__ bool both_tiles(const WorkArgs& a, int n, int block) { return 2 * (n - block * a.tokens) > a.tokens; }
// Cost of one of an item's key tiles: one, where blocks are one tile of query rows.  Where they are two tiles of whole tokens, a key
// tile takes 2.1 us if the tokens fill both and 1.15 us if they fill one: 9 and 5.  What an item takes besides (its last
// product, its output: 4.8 and 2.7 us) is spread over its tiles.
constexpr int kBothTiles = 9, kOneTile = 5, kBothItem = 20, kOneItem = 12;
__device__ __forceinline__ int weight_of(const WorkArgs& a, int n, int block, int tiles) {
  if (!a.tokens) return 1;
  const bool both = both_tiles(a, n, block);
  return (both ? kBothTiles : kOneTile) + (int)((unsigned)(both ? kBothItem : kOneItem) / (unsigned)tiles);
}

// The item at (pair, block) of a unit whose tokens and a head whose length are known: its tiles whose cost begins in [begin, end),
// relative to the cost before the item.
__device__ __forceinline__ Item item_of(const WorkArgs& a, int pair, int block, int first, int n, int len, long long begin,
                                        long long end) {
  Item it;
  it.u = pair / a.Hkv, it.g = pair - it.u * a.Hkv, it.block = block;
  it.first = first, it.n = n, it.len = len;
  it.rows = n * a.G;
  it.visible = block_visible(a, n, len, block);
  it.tiles = tiles_of(a, it.visible);
  it.weight = weight_of(a, n, block, it.tiles);
  const long long cost = (long long)it.tiles * it.weight;
  const int from = (int)(begin < cost ? begin : cost), to = (int)(end < cost ? end : cost);
  it.t0 = (from + it.weight - 1) / it.weight, it.t1 = (to + it.weight - 1) / it.weight;
  return it;
}

constexpr int kMaxRounds = 8;
struct Plan {           // in shared memory
  long long warp_sum[16];
  int warp_items[16];
  int2 warp_most[16];
  long long begin, end; // the worker's share, relative to the cost before the item it starts in
  int pair, block;      // that item
  Item it;              // what is known of the worker's first item
  // Whole items ahead of the share: round k hands worker w the item k * workers + w.
  int n_rounds;
  int2 round[kMaxRounds];                      // (pair, block) of the worker's
  long long before[kMaxRounds + 1];            // cost of the items before round k
  long long mine[kMaxRounds], cost[kMaxRounds]; // cost of the items before the worker's of the round, and its own
};

// Cost of a pair's blocks; `most`: the greatest weight of a tile.
__device__ __forceinline__ long long pair_cost(const WorkArgs& a, int p, int& most) {
  int first, n;
  unit_tokens(a.starts, p / a.Hkv, a.T, first, n);
  const int len = head_length(a, p), nb = unit_blocks(a, n);
  long long c = 0;
  for (int b = 0; b < nb; ++b) {
    const int t = tiles_of(a, block_visible(a, n, len, b)), w = weight_of(a, n, b, t);
    c += t * w, most = max(most, w);
  }
  return c;
}
// 32-bit divisions where they do: the plan is all latency.
__device__ __forceinline__ long long part_of(long long total, int worker, int workers) {
  return total < (1 << 24) ? (long long)((unsigned)total * (unsigned)worker / (unsigned)workers) : total * worker / workers;
}
// The share [begin, end) of a worker.
__device__ __forceinline__ void share_of(long long total, int granule, int worker, int n_workers, long long& begin, long long& end) {
  // rounded down: every share is at least `granule` wide, no less than a tile, so that a tile begins in each (the join follows an item from one
  // worker to the next and stops at the first that has no part in it)
  const long long most = max(total / granule, 1ll);
  const int workers = (int)(most < n_workers ? most : n_workers);
  begin = end = total;
  if (worker < workers) {
    begin = part_of(total, worker, workers), end = part_of(total, worker + 1, workers);
  }
}
// Where in pair p's cost offset `at` falls, for a share of `width`.
__device__ __forceinline__ void settle_plan(const WorkArgs& a, int p, long long at, long long width, Plan& plan) {
  int first, n, b = 0;
  unit_tokens(a.starts, p / a.Hkv, a.T, first, n);
  const int len = head_length(a, p);
  for (;; ++b) {
    const int t = tiles_of(a, block_visible(a, n, len, b)), c = t * weight_of(a, n, b, t);
    if (at < c) break;
    at -= c;
  }
  plan.pair = p, plan.block = b, plan.begin = at, plan.end = at + width;
  plan.it = item_of(a, p, b, first, n, len, at, at + width);
}

// All threads of the CTA.  Returns with the worker's share in `plan`.  Few (unit, KV head) pairs of few blocks one warp does
// alone, without barriers; else every thread has its pairs or, where there are more threads, its blocks of a pair (one thread a
// pair: 22 us for the 32 blocks of 2048 tokens, 4 this way).
//
// With rounds: while the most expensive item costs less than a fair share, the first items go out whole, one to each worker and
// round, and only the rest is split, so that the shares even out.  In a round all workers start at the first key of
// neighbouring blocks: they read the same keys and values at the same time, from L2 (shares cut end to end start all over
// the cache: 2.65 GB from memory instead of 0.17 for four 2048-token chunks on 8192 rows).
template <int NT>
__device__ void make_plan(const WorkArgs& a, int worker, int n_workers, Plan& plan) {
  const int pairs = a.Nu * a.Hkv;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (a.one_warp) {
    if (warp == 0) {
      constexpr int kPer = kWarpPairs / 32;
      const int per = (pairs + 31) / 32;
      long long c[kPer], mine = 0;
      int heaviest = a.granule;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        c[i] = i < per && lane * per + i < pairs ? pair_cost(a, lane * per + i, heaviest) : 0;
        mine += c[i];
      }
      long long incl = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
      }
      long long begin, end;
      share_of(__shfl_sync(0xffffffffu, incl, 31), __reduce_max_sync(0xffffffffu, heaviest), worker, n_workers, begin, end);
      long long at = begin - (incl - mine), off = -1;
      if (lane == 0) plan.n_rounds = 0;
      if (begin >= end) {
        if (lane == 0) plan.begin = plan.end = 0;
      } else if (at >= 0 && at < mine) {
        int p = lane * per;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (off < 0 && at < c[i]) p += i, off = at;
          at -= c[i];
        }
        settle_plan(a, p, off, end - begin, plan);
      }
    }
    __syncthreads();
    return;
  }
  static_assert(NT <= 512, "one entry of warp_sum per warp");
  // the thread's items, in order: all blocks of the pairs p0 to p1, or part of the blocks of pair p0
  int log_group = 0;
  while (log_group < 5 && (pairs << (log_group + 1)) <= NT) ++log_group;
  const int per = (pairs + NT - 1) / NT, sub = threadIdx.x & ((1 << log_group) - 1);
  const int p0 = min(log_group ? (int)threadIdx.x >> log_group : (int)threadIdx.x * per, pairs), p1 = min(p0 + per, pairs);
  auto each = [&](auto&& f) {   // f(pair, block, first, n, len, tiles, weight) until it says stop
    for (int p = p0; p < p1; ++p) {
      int first, n;
      unit_tokens(a.starts, p / a.Hkv, a.T, first, n);
      const int len = head_length(a, p), nb = unit_blocks(a, n);
      const int b1 = (nb * (sub + 1)) >> log_group;
      for (int b = (nb * sub) >> log_group; b < b1; ++b) {
        const int t = tiles_of(a, block_visible(a, n, len, b));
        if (f(p, b, first, n, len, t, weight_of(a, n, b, t))) return;
      }
    }
  };
  long long mine = 0;
  int items = 0, most = 0, heaviest = a.granule;
  each([&](int, int, int, int, int, int t, int w) {
    mine += t * w, most = max(most, t * w), heaviest = max(heaviest, w), ++items;
    return false;
  });
  long long incl = mine;
  int incl_items = items;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long o = __shfl_up_sync(0xffffffffu, incl, d);
    const int i = __shfl_up_sync(0xffffffffu, incl_items, d);
    if (lane >= d) incl += o, incl_items += i;
  }
  most = __reduce_max_sync(0xffffffffu, most), heaviest = __reduce_max_sync(0xffffffffu, heaviest);
  if (lane == 31) plan.warp_sum[warp] = incl, plan.warp_items[warp] = incl_items, plan.warp_most[warp] = make_int2(most, heaviest);
  __syncthreads();
  long long before = incl - mine, total = 0;
  int items_before = incl_items - items, n_items = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    if (w < warp) before += plan.warp_sum[w], items_before += plan.warp_items[w];
    total += plan.warp_sum[w], n_items += plan.warp_items[w];
    most = max(most, plan.warp_most[w].x), heaviest = max(heaviest, plan.warp_most[w].y);
  }
  int rounds = 0;
  if (a.rounds && total / heaviest >= n_workers)   // every worker keeps at least a tile of the rest
    rounds = (int)min(min((total / n_workers - heaviest) / most, (long long)(n_items / n_workers)), (long long)kMaxRounds);
  long long begin, end;
  if (rounds > 0) {
    // the thread that has an item says which it is and what comes before it
    for (int k = 0; k <= rounds; ++k) {
      const int head = k * n_workers - items_before, own = k < rounds ? head + worker : -1;   // of the thread's items
      if ((head < 0 || head >= items) && (own < 0 || own >= items)) continue;
      int i = 0;
      long long c = before;
      each([&](int p, int b, int first, int n, int len, int t, int w) {
        const int cost = t * w;
        if (i == head) plan.before[k] = c;
        if (i == own) {
          plan.mine[k] = c, plan.cost[k] = cost, plan.round[k] = make_int2(p, b);
          if (k == 0) plan.it = item_of(a, p, b, first, n, len, 0, 1ll << 40);
        }
        ++i, c += cost;
        return false;
      });
    }
    if (threadIdx.x == 0 && rounds * n_workers == n_items) plan.before[rounds] = total;
    __syncthreads();
    const long long rest = plan.before[rounds];
    begin = rest + part_of(total, worker, n_workers), end = rest + part_of(total, worker + 1, n_workers);
    for (int k = 0; k < rounds; ++k) {
      const long long handed = plan.mine[k] - plan.before[k];
      begin -= handed, end -= handed + plan.cost[k];
    }
  } else {
    share_of(total, heaviest, worker, n_workers, begin, end);
  }
  if (threadIdx.x == 0) {
    plan.n_rounds = rounds;
    if (begin >= end) plan.begin = plan.end = 0;
  }
  if (end > begin && begin >= before && begin < before + mine) {
    long long at = begin - before;
    each([&](int p, int b, int first, int n, int len, int t, int w) {
      if (at >= t * w) {
        at -= t * w;
        return false;
      }
      plan.pair = p, plan.block = b, plan.begin = at, plan.end = at + (end - begin);
      if (rounds == 0) plan.it = item_of(a, p, b, first, n, len, at, at + (end - begin));
      return true;
    });
  }
  __syncthreads();
}

__device__ __forceinline__ Item make_item(const WorkArgs& a, int pair, int block, long long begin, long long end) {
  int first, n;
  unit_tokens(a.starts, pair / a.Hkv, a.T, first, n);
  return item_of(a, pair, block, first, n, head_length(a, pair), begin, end);
}
// Moves to the next item that has rows; false behind the last one.
__device__ __forceinline__ bool next_item(const WorkArgs& a, int& pair, int& block, int n) {
  if (block + 1 < unit_blocks(a, n)) {
    ++block;
    return true;
  }
  block = 0;
  while (++pair < a.Nu * a.Hkv) {
    int first, m;
    unit_tokens(a.starts, pair / a.Hkv, a.T, first, m);
    if (unit_blocks(a, m) > 0) return true;
    pair = (pair / a.Hkv) * a.Hkv + a.Hkv - 1;   // the unit's other heads have none either
  }
  return false;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ float2 ld_peer(const void* mine, int rank) {   // the same place in another CTA's shared memory
  uint32_t at;
  float2 x;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(at) : "memory");
  return x;
}

// Walks a worker's items: for (Walk k(...); k.more(); k.next()) ... k.it
struct Walk {
  int pair, block, round;
  long long begin, end;
  bool live;
  Item it;
  __device__ __forceinline__ void settle(const WorkArgs& a) {   // to the first item with tiles for this worker
    while (live) {
      it = make_item(a, pair, block, begin, end);
      if (it.t1 > it.t0) return;
      step(a);
    }
  }
  __device__ __forceinline__ void step(const WorkArgs& a) {
    end -= (long long)it.tiles * it.weight, begin = 0;
    live = end > 0 && next_item(a, pair, block, it.n);
  }
  __device__ __forceinline__ void start(const WorkArgs& a, const Plan& p) {
    round = 0, pair = p.pair, block = p.block, begin = p.begin, end = p.end, live = end > begin || p.n_rounds > 0;
    if (!live) return;
    it = p.it;
    if (p.n_rounds > 0) pair = p.round[0].x, block = p.round[0].y;
    if (it.t1 > it.t0) return;
    step(a);
    settle(a);
  }
  // The next item; with rounds, whole ones first.
  __device__ __forceinline__ void next(const WorkArgs& a, const Plan& p) {
    if (round < p.n_rounds) {
      if (++round < p.n_rounds) {
        pair = p.round[round].x, block = p.round[round].y;
        it = make_item(a, pair, block, 0, 1ll << 40);
        return;
      }
      pair = p.pair, block = p.block, live = end > begin;
    } else {
      step(a);
    }
    settle(a);
  }
  // Where an item is one cluster's: the i-th of (pair, expected block), and `more` times as many blocks on where a unit has more
  // than expected.
  __device__ __forceinline__ static int cluster_pair(const WorkArgs& a, int i) { return a.blocks == 1 ? i : i / a.blocks; }
  __device__ __forceinline__ bool cluster_item(const WorkArgs& a, int i, int more) {
    const int p = cluster_pair(a, i), b = i + (more - p) * a.blocks;
    it = make_item(a, p, b, 0, 1ll << 40);
    return live = b < unit_blocks(a, it.n);
  }
  // i and `more` of an item
  __device__ __forceinline__ static int cluster_more(const WorkArgs& a, const Item& it) { return it.block / a.blocks; }
  __device__ __forceinline__ static int cluster_index(const WorkArgs& a, const Item& it) {
    return (it.u * a.Hkv + it.g - cluster_more(a, it)) * a.blocks + it.block;
  }
};
// Rows of the block, and where query row r of it (token, head) lives.
__device__ __forceinline__ int block_rows(const WorkArgs& a, const Item& it) {
  return min(a.M, it.rows - it.block * a.M);
}
__device__ __forceinline__ int64_t out_row(const WorkArgs& a, const Item& it, int r) {
  const int row = it.block * a.M + r;
  const int token = row / a.G;
  return (int64_t)(it.first + token) * a.H + it.g * a.G + (row - token * a.G);
}
// Rows of the cache that query row r of the block sees.
__device__ __forceinline__ int row_limit(const WorkArgs& a, const Item& it, int r) {
  return rows_seen(a, it.n, it.len, (it.block * a.M + r) / a.G + 1);
}
// Pool row (page * page_size + row within) is not formed: the pool's strides are free.  A bad page gives -1.
__device__ __forceinline__ int page_of(const WorkArgs& a, const Item& it, int slot) {
  const int p = a.table[((int64_t)it.u * a.Hkv + it.g) * a.max_pages + slot];
  if ((unsigned)p < (unsigned)a.n_pages) return p;
  report_status(a.status, kStatusPage);
  return -1;
}

constexpr int kWorkers = 148;        // CTAs of every attention kernel, one per SM
constexpr int kTcRows = 256;         // query rows of a block of the tensor-core kernel

// `base`: everything but the block and tile sizes; most: the tokens a unit is expected to have at most; scale not 0.
cudaError_t launch_attend_tc(const ckv_paged& pg, const WorkArgs& base, int64_t most, float scale, const void* q, const void* k_pages,
                             const void* v_pages, void* out, float* lse, cudaStream_t st);
constexpr int kMmaRows = 32;         // most query rows of a block of the bf16 kernel for few rows
constexpr int kMmaTile = 64;         // keys per tile of its schedule
constexpr int kMmaCtaKeys = 128;     // keys a CTA of it takes per step
// When a cache (the room its table has) is short: a CTA of a cluster takes `cta_keys` per step, and reads no more than the given part of the split's even share
// and `rows` more.  (A row takes such a CTA 13 ns with up to 16 query rows, 21 with 32, 32 in fp32; the split's schedule and
// join take 10 us.  With 32 query rows the other side is the tensor-core kernel: 9 ns a row.)
struct ShortRule {
  int cta_keys, share_percent, rows;
};
constexpr ShortRule kShortFew{kMmaCtaKeys, 100, 800}, kShortMore{kMmaCtaKeys, 50, 450};
// CTAs per cluster where the cache is short, else 0.  blocks: of query rows of a pair.
int cluster_size(const ckv_paged& pg, const ShortRule& rule, int64_t blocks);
cudaError_t launch_attend_mma(const ckv_paged& pg, const WorkArgs& base, int64_t most, float scale, const void* q, const void* k_pages,
                              const void* v_pages, void* out, float* lse, cudaStream_t st);
// rows: the most query rows a block has.
template <bool BF16>
cudaError_t launch_join(const WorkArgs& a, int workers, int rows, void* out, float* lse, cudaStream_t st);

}  // namespace ckv
