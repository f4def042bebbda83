// The pages of a cache: rows moved together inside them, pages reserved, given back, and shared with new sequences.
// All of it moves whole rows (256 or 512 bytes, in 16-byte pieces) and counts; what is decided on the device depends on the inputs
// alone: page numbers are handed out by rank, counts change by commutative atomics.
#include "pages.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 256;
constexpr int kKeepThreads = 1024;   // most of a CTA that moves the rows of a list

struct Pool {           // rows of the two pools, in bytes
  char *k, *v;
  int64_t page, row;
  int log_p, P, n_pages, max_pages;
};

// ------------------------------------------------------------------------------------------------ rows kept
// A list names the rows of a span that stay, ascending: row base + i of the pair becomes what row base + list[i] was.  Since
// list[i] >= i, a row is never written before the rows in front of it are read, if entries go in order: a group of threads reads
// `U * R` rows, meets, and writes them; what it reads next lies behind all it has written.  Columns do not meet: a pair's rows
// may be cut into slices of their 16-byte pieces, a group each, where there are few pairs.
// Entries that stay where they are (list[i] == i, a prefix of the list) are not touched.
// Every group of a pair looks its list and pages over first and comes to the same answer: a pair is moved whole or left alone.
// Bound: long lists HBM, as far as one CTA of an SM can keep it busy between two meetings; short ones five dependent reads.  64 heads'
// lists of 2048 to 4096 of 32k rows, 207 MB there and back: 54 us, 3.9 TB/s (0.6 of the measured copy rate; the longest list, a third
// above the average, sets the end: lists of one length 47 us, 4.3 TB/s).  In slices of 64 bytes, four times the CTAs: 64 us, since a random row
// is then four visits of HBM; a cluster a list: 75, its barrier waits for the stores too; the next batch asked for before this one is
// written: 62.  Up to eight rows of 4096 heads (19 MB): 8.2 us.
struct KeepArgs {
  Pool pool;
  Lists lists;
  int pairs, n_rows;
  const int32_t *rows, *begins, *counts, *tails, *refs, *lengths, *table;
  int32_t* new_lengths;
  int* status;
};

// A group is a warp (short lists) or a CTA.  slices: of a row; log_s: log2 of the 16-byte pieces in a slice.
template <bool kWarp>
__global__ void __launch_bounds__(kWarp ? kThreads : kKeepThreads) keep_rows_kernel(KeepArgs a, int slices, int log_s) {
  constexpr int U = kWarp ? 4 : 8;
  const int NT = kWarp ? 32 : blockDim.x;
  __shared__ int s_first;
  pdl_wait();
  pdl_launch_dependents();
  const int group = kWarp ? blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5) : blockIdx.x;
  const int t = kWarp ? threadIdx.x & 31 : threadIdx.x;
  const int pair = group / (2 * slices), which = group - pair * 2 * slices;
  if (pair >= a.pairs) return;
  const int list = a.lists.of(pair), len = a.lengths[pair], count = a.counts[list], begin = a.begins[list];
  const int span = a.tails ? a.tails[list] : len, base = len - span, log_p = a.pool.log_p;
  const int32_t* const rows = a.rows + begin;
  const int32_t* const table = a.table + (int64_t)pair * a.pool.max_pages;
  if (!kWarp) {
    if (threadIdx.x == 0) s_first = 0x7fffffff;
    __syncthreads();
  }
  bool ok = len >= 0 && len <= a.pool.max_pages << log_p && span >= 0 && span <= len && count >= 0 && count <= span &&
            begin >= 0 && count <= a.n_rows && begin <= a.n_rows - count;
  const int n = ok ? count : 0;
  int first = 0x7fffffff;      // the first entry that moves
#pragma unroll 4
  for (int i = t; i < n; i += NT) {
    const int x = rows[i];
    const int before = i ? rows[i - 1] : -1;
    if (x < i || x <= before || x >= span) {   // x < i: a list that ascends from zero on never is; such an x may lie before the table
      ok = false;
    } else if (x != i) {       // from and to pages of the pool, and to none that others hold
      first = min(first, i);
      const int to = table[(base + i) >> log_p];
      if ((unsigned)table[(base + x) >> log_p] >= (unsigned)a.pool.n_pages || (unsigned)to >= (unsigned)a.pool.n_pages) ok = false;
      else if (a.refs && a.refs[to] > 1) ok = false;
    }
  }
  if (kWarp) {
    first = __reduce_min_sync(0xffffffffu, first);
    ok = __all_sync(0xffffffffu, ok);
  } else {
    if (first < 0x7fffffff) atomicMin(&s_first, first);
    ok = __syncthreads_and(ok);
    first = s_first;
  }
  if (which == 0 && t == 0) {
    a.new_lengths[pair] = ok ? base + count : len;
    if (!ok) report_status(a.status, kStatusPage);
  }
  if (!ok || first >= count) return;
  const bool values = which >= slices;
  char* const data = (values ? a.pool.v : a.pool.k) + ((((values ? which - slices : which) << log_s) + (t & ((1 << log_s) - 1))) << 4);
  auto at = [&](int row) {
    return reinterpret_cast<uint4*>(data + table[row >> log_p] * a.pool.page + (row & (a.pool.P - 1)) * a.pool.row);
  };
  const int R = NT >> log_s;
  int src[U];                  // rows to read, looked up a batch ahead
  auto look_up = [&](int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) src[u] = i0 + u * R < count ? base + rows[i0 + u * R] : -1;
  };
  int i0 = first + (t >> log_s);
  look_up(i0);
  for (int left = count - first; left > 0; left -= U * R, i0 += U * R) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (src[u] >= 0) x[u] = __ldcg(at(src[u]));
    if (left > U * R) look_up(i0 + U * R);
    if (kWarp) __syncwarp();
    else __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * R < count) __stcg(at(base + i0 + u * R), x[u]);
  }
}

// ------------------------------------------------------------------------------------------------ pages reserved
// A pair needs pages for rows length .. length + new - 1: growth, the slots from `held` on, and copies, those of the slots it will
// write whose page others hold too (only the first of them, slot length / P, has rows to copy).  Page numbers go by rank: the
// r-th page that is needed (pairs in order, a pair's copies before its growth, slots ascending) is the r-th free one.
// reserve_count_kernel leaves the free and the shared pages as bits, their number per chunk of pages, and what each pair needs; nothing
// is changed yet.  reserve_apply_kernel adds the numbers up (a few thousand, each CTA for itself: no waiting), and if there are enough:
//   a CTA per chunk    hands its free pages out to the pairs that grow: one page a thread, whose pair it looks up by rank;
//   a group per pair   updates `held` and makes the pair's copies, whose pages it looks up by rank.
// Bound: latency (two launches, about five dependent reads each); with many copies HBM.  8192 heads, of which one in 32 needs a
// page: 13 us in all; 131072 pages for 512 heads from a pool of a million of which an eighth is free: 4.4 and 13 under ncu; 8192 copies of
// 31 rows (264 MB there and back): 50 us, 5.3 TB/s.
struct ReserveArgs {
  Pool pool;
  Lists lists;
  int pairs;
  const int32_t *new_rows, *lengths;
  int32_t *held, *table, *refs, *room;
  int* status;
  int chunk, n_chunks, n_blocks;
  uint32_t *free_bits, *shared_bits;
  int32_t *chunk_free, *block_need;
  int2* need;
};

// What a pair wants: its first slot to be written and the number of slots it wants to hold (0: nothing, as a pair whose state is none gets).
struct Want {
  int first, slots, rows;    // rows in the first slot's page
};
__device__ __forceinline__ Want want_of(const ReserveArgs& a, int pair, int held, bool& bad) {
  const int len = a.lengths[pair], more = a.new_rows[a.lists.of(pair)];
  const bool none = len < 0 || held < 0 || held > a.pool.max_pages;
  bad |= none || more < 0;
  if (none || more <= 0) return {0, 0, 0};
  const int64_t slots = ((int64_t)len + more + a.pool.P - 1) >> a.pool.log_p;
  bad |= slots > a.pool.max_pages;
  return {len >> a.pool.log_p, (int)min(slots, (int64_t)a.pool.max_pages), len & (a.pool.P - 1)};
}

__global__ void __launch_bounds__(kThreads) reserve_count_kernel(ReserveArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if ((int)blockIdx.x < a.n_chunks) {
    __shared__ int s_free[kThreads / 32];
    const int64_t begin = (int64_t)blockIdx.x * a.chunk;
    int n = 0;
    for (int w0 = warp * 4; w0 < a.chunk / 32; w0 += kThreads / 32 * 4) {     // four words of 32 pages at a time
      int refs[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t page = begin + (w0 + k) * 32 + lane;
        refs[k] = page < a.pool.n_pages ? a.refs[page] : 1;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t none = __ballot_sync(0xffffffffu, refs[k] == 0), several = __ballot_sync(0xffffffffu, refs[k] > 1);
        n += __popc(none);
        if (lane == 0) a.free_bits[begin / 32 + w0 + k] = none, a.shared_bits[begin / 32 + w0 + k] = several;
      }
    }
    if (lane == 0) s_free[warp] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < kThreads / 32; ++w) n += s_free[w];
      a.chunk_free[blockIdx.x] = n;
    }
    return;
  }
  const int block = ((int)blockIdx.x - a.n_chunks) * (kThreads / 32) + warp, pair = block * kPairBlock + lane;
  if (block >= a.n_blocks) return;
  int need = 0, copies = 0;
  bool bad = false;
  if (pair < a.pairs) {
    const int held = a.held[pair];
    const Want w = want_of(a, pair, held, bad);
    for (int s = w.first; s < min(held, w.slots); ++s) {
      const int page = a.table[(int64_t)pair * a.pool.max_pages + s];
      if ((unsigned)page >= (unsigned)a.pool.n_pages) bad = true;
      else copies += a.refs[page] > 1;
    }
    need = copies + (w.slots ? max(w.slots - held, 0) : 0);
  }
  if (bad) report_status(a.status, kStatusPage);
  int sum = need;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += x;
  }
  if (pair < a.pairs) a.need[pair] = make_int2(sum, copies);
  if (lane == 31) a.block_need[block] = sum;
}

__device__ __forceinline__ int warp_scan(int x, int lane) {   // inclusive
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  return x;
}
// A thread's entries [lo, hi) of an array that the CTA adds up.
struct Part {
  int lo, hi;
  __device__ __forceinline__ Part(int n) {
    const int per = (n + kThreads - 1) / kThreads;
    lo = min((int)threadIdx.x * per, n), hi = min(lo + per, n);
  }
};
// What is needed and what is there; `before`: the sum ahead of entry `at` (of the needs, or of the free pages).
struct Sums {
  long long need, free;
  int before;
  int mine;       // sum ahead of this thread's entries of the other array, the one that ranks are looked up in
};
__device__ __forceinline__ Sums add_up(const ReserveArgs& a, bool pages, int at, int (*s_sum)[4]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Part pb(a.n_blocks), pc(a.n_chunks);
  // a block needs less than 2^26 pages, and where a sum passes 2^31 there are not enough
  long long need = 0;
  int free = 0, before = 0;
  for (int i = pb.lo; i < pb.hi; ++i) {
    const int x = a.block_need[i];
    need += x;
    if (!pages && i < at) before += x;
  }
  for (int i = pc.lo; i < pc.hi; ++i) {
    const int x = a.chunk_free[i];
    free += x;
    if (pages && i < at) before += x;
  }
  const int own = pages ? (int)min(need, 1ll << 30) : free, scan = warp_scan(own, lane);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    need += __shfl_xor_sync(0xffffffffu, need, d), free += __shfl_xor_sync(0xffffffffu, free, d);
    before += __shfl_xor_sync(0xffffffffu, before, d);
  }
  __shared__ long long s_need[kThreads / 32];
  if (lane == 31) s_sum[warp][0] = free, s_sum[warp][1] = before, s_sum[warp][2] = scan, s_need[warp] = need;
  __syncthreads();
  Sums s{0, 0, 0, scan - own};
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    s.need += s_need[w], s.free += s_sum[w][0], s.before += s_sum[w][1];
    if (w < warp) s.mine += s_sum[w][2];
  }
  return s;
}
// The last i with x[i] <= r (x ascending, x[0] <= r).
__device__ __forceinline__ int last_at_most(const int32_t* x, int n, int r) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (x[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}
// The rank-th free page, by a warp; starts: free pages ahead of each chunk.
__device__ __forceinline__ int page_of_rank(const ReserveArgs& a, const int32_t* starts, int rank, int lane) {
  const int c = last_at_most(starts, a.n_chunks, rank);
  const uint32_t* const words = a.free_bits + (int64_t)c * (a.chunk / 32);
  int r = rank - starts[c];
  for (int w0 = 0; w0 < a.chunk / 32; w0 += 32) {
    uint32_t bits = words[w0 + lane];
    const int mine = __popc(bits), sum = warp_scan(mine, lane);
    const uint32_t past = __ballot_sync(0xffffffffu, sum > r);
    if (past) {
      const int from = __ffs(past) - 1;
      for (int k = r - (sum - mine); lane == from && k > 0; --k) bits &= bits - 1u;
      return (int)((int64_t)c * a.chunk + (w0 + from) * 32 + __shfl_sync(0xffffffffu, (int)__ffs(bits), from) - 1);
    }
    r -= __shfl_sync(0xffffffffu, sum, 31);
  }
  return 0;    // not reached: there are enough
}

// kPairs: the pairs of a CTA.  One: it copies with all its threads; else a warp copies a page.
template <int kPairs>
__global__ void __launch_bounds__(kThreads, kPairs > 1 ? 2 : 4) reserve_apply_kernel(ReserveArgs a, int log_row) {
  constexpr bool kWarp = kPairs > 1;
  static_assert(kPairBlock % kPairs == 0, "a CTA's pairs are of one block");
  __shared__ int32_t s_prefix[kMaxChunks];
  __shared__ int s_sum[kThreads / 32][4], s_page, s_held[kPairs];
  __shared__ int2 s_need[kPairs];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool pages = (int)blockIdx.x < a.n_chunks;
  const int pair0 = ((int)blockIdx.x - a.n_chunks) * kPairs, block = pair0 / kPairBlock;
  const int64_t page0 = (int64_t)blockIdx.x * a.chunk;
  // asked for ahead of the sums: a thread's four pages, or its pair
  const int pair = pair0 + (int)threadIdx.x;
  const bool live = !pages && threadIdx.x < kPairs && pair < a.pairs;
  uint32_t word = pages ? a.free_bits[page0 / 32 + (threadIdx.x >> 3)] : 0u;
  int2 need = make_int2(0, 0);
  Want w{0, 0, 0};
  int held = 0;
  bool bad = false;
  if (live) need = a.need[pair], held = a.held[pair], w = want_of(a, pair, held, bad);
  const Sums sum = add_up(a, pages, pages ? (int)blockIdx.x : block, s_sum);
  const bool enough = sum.need <= sum.free;
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.room) {
    a.room[0] = (int)(enough ? sum.free - sum.need : sum.free);
    a.room[1] = (int)min(enough ? 0ll : sum.need - sum.free, 0x7fffffffll);
  }
  if (!enough) return;
  if (pages) {
    if (sum.before >= sum.need) return;
    const Part p(a.n_blocks);
    for (int i = p.lo, x = sum.mine; i < p.hi; ++i) s_prefix[i] = x, x += a.block_need[i];
    int rank0 = sum.before;
    for (int w0 = 0; rank0 < sum.need && w0 < a.chunk / 32; w0 += kThreads / 8) {
      if (w0) word = a.free_bits[page0 / 32 + w0 + (threadIdx.x >> 3)];
      uint32_t bits = word >> (4 * (threadIdx.x & 7)) & 15u;
      const int mine = __popc(bits), scan = warp_scan(mine, lane);
      __syncthreads();
      if (lane == 31) s_sum[warp][3] = scan;
      __syncthreads();
      int rank = rank0 + scan - mine;
      for (int k = 0; k < kThreads / 32; ++k) {
        if (k < warp) rank += s_sum[k][3];
        rank0 += s_sum[k][3];
      }
      for (; bits && rank < sum.need; bits &= bits - 1u, ++rank) {
        const int b = last_at_most(s_prefix, a.n_blocks, rank), r = rank - s_prefix[b], last = a.pairs - 1;
        // the first pair of the block with more than r pages up to it
        int to = b * kPairBlock, some = 0;
#pragma unroll
        for (int k = 7; k < 31; k += 8) some += a.need[min(to + k, last)].x <= r;
        to += 8 * some, some = 0;
#pragma unroll
        for (int k = 0; k < 7; ++k) some += a.need[min(to + k, last)].x <= r;
        to += some;
        const int2 n = a.need[to];
        const int before = to % kPairBlock ? a.need[to - 1].x : 0, which = r - before;
        if (which < n.y) continue;                       // a copy
        const Want x = want_of(a, to, 0, bad);           // (one that needs a page holds a number of them that can be)
        const int page = (int)(page0 + (w0 + (threadIdx.x >> 3)) * 32 + 4 * (threadIdx.x & 7) + __ffs(bits) - 1);
        a.table[(int64_t)to * a.pool.max_pages + x.slots - (n.x - before) + which] = page;
        a.refs[page] = 1;
      }
    }
    return;
  }
  if (live) {
    if (w.slots && w.slots > held) a.held[pair] = w.slots;
    // copies: pages from this rank on
    const int at = pair % kPairBlock;
    s_need[threadIdx.x] = make_int2(sum.before + (at ? a.need[pair - 1].x : 0), need.y);
    s_held[threadIdx.x] = min(held, w.slots);
  } else if (threadIdx.x < kPairs) {
    s_need[threadIdx.x] = make_int2(0, 0);
  }
  if (!__syncthreads_or(need.y > 0)) return;
  const Part p(a.n_chunks);
  for (int i = p.lo, x = sum.mine; i < p.hi; ++i) s_prefix[i] = x, x += a.chunk_free[i];
  __syncthreads();
  constexpr int NT = kWarp ? 32 : kThreads, U = kWarp ? 8 : 4;
  const int t = kWarp ? lane : threadIdx.x;
  for (int i = kWarp ? warp : 0; i < kPairs; i += kThreads / 32) {
    if (s_need[i].y == 0) continue;
    const int its = pair0 + i, end = s_held[i];
    int rank = s_need[i].x;
    const Want x = want_of(a, its, 0, bad);
    int32_t* const table = a.table + (int64_t)its * a.pool.max_pages;
    for (int s = x.first; s < end; ++s) {
      const int old = table[s];
      if ((unsigned)old >= (unsigned)a.pool.n_pages || !(a.shared_bits[old >> 5] >> (old & 31) & 1u)) continue;
      int page = 0;
      if (kWarp) {
        page = page_of_rank(a, s_prefix, rank, lane);
      } else {
        if (warp == 0) {
          page = page_of_rank(a, s_prefix, rank, lane);
          if (lane == 0) s_page = page;
        }
        __syncthreads();
        page = s_page;
      }
      if (s == x.first) {
        const int half = x.rows << log_row;              // 16-byte pieces of the keys; the values' follow
        const int64_t from = old * a.pool.page, to = page * a.pool.page - from;
        auto at = [&](int e) {
          char* const pool = e < half ? a.pool.k : a.pool.v;
          e -= e < half ? 0 : half;
          return pool + from + (e >> log_row) * a.pool.row + ((e & ((1 << log_row) - 1)) << 4);
        };
        for (int e0 = t; e0 < 2 * half; e0 += NT * U) {
          uint4 y[U];
#pragma unroll
          for (int k = 0; k < U; ++k)
            if (e0 + k * NT < 2 * half) y[k] = __ldcg(reinterpret_cast<const uint4*>(at(e0 + k * NT)));
#pragma unroll
          for (int k = 0; k < U; ++k)
            if (e0 + k * NT < 2 * half) __stcg(reinterpret_cast<uint4*>(at(e0 + k * NT) + to), y[k]);
        }
      }
      if (kWarp) __syncwarp();
      else __syncthreads();
      if (t == 0) table[s] = page, a.refs[page] = 1, atomicSub(&a.refs[old], 1);
      ++rank;
    }
  }
}

// ------------------------------------------------------------------------------------------------ pages given back
// 2^log_t threads a pair, four pages each at a time.  Bound: latency, and with many pages the atomics of L2 (a million: 11 us).
__global__ void __launch_bounds__(kThreads) pages_trim_kernel(Pool pool, int pairs, int log_t, const int32_t* lengths, int32_t* held, const int32_t* table,
                                                              int32_t* refs, int* status) {
  pdl_wait();
  pdl_launch_dependents();
  const int pair = (int)(blockIdx.x * (kThreads >> log_t) + (threadIdx.x >> log_t)), t = threadIdx.x & ((1 << log_t) - 1);
  const bool live = pair < pairs;
  const int len = live && lengths ? lengths[pair] : 0, have = live ? held[pair] : 0;
  const bool none = len < 0 || have < 0 || have > pool.max_pages;      // the pair is left as it is
  bool bad = none;
  const int end = none ? 0 : have, keep = none ? 0 : (int)(((int64_t)len + pool.P - 1) >> pool.log_p);
  for (int s0 = keep + t; s0 < end; s0 += 4 << log_t) {
    int page[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) page[i] = s0 + (i << log_t) < end ? table[(int64_t)pair * pool.max_pages + s0 + (i << log_t)] : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (s0 + (i << log_t) >= end) continue;
      if ((unsigned)page[i] >= (unsigned)pool.n_pages) bad = true;
      else if (atomicSub(&refs[page[i]], 1) < 1) atomicAdd(&refs[page[i]], 1), bad = true;   // nobody held it
    }
  }
  __syncthreads();     // all of the pair's threads have read `held`
  if (live && t == 0 && keep < end) held[pair] = keep;
  if (bad) report_status(status, kStatusPage);
}

// ------------------------------------------------------------------------------------------------ pages shared
// A warp per pair: those of the new sequences copy their parents' table rows, those of the old ones count their children in (and
// themselves out, where the old sequences end): one atomic a page whatever the number of children.  1024 heads of 126 pages to eight
// each, 8 MB of table: 7.6 us.
struct ForkArgs {
  Pool pool;
  int Hkv, layers, seqs, new_seqs, keep_old;
  const int32_t *parents, *lengths, *held, *table;
  int32_t *refs, *new_lengths, *new_held, *new_table;
  int* status;
};
__global__ void __launch_bounds__(kThreads) pages_fork_kernel(ForkArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int64_t fresh = (int64_t)a.layers * a.new_seqs * a.Hkv, old = (int64_t)a.layers * a.seqs * a.Hkv;
  bool bad = false;
  if (w < fresh) {
    const int pair = (int)w, unit = pair / a.Hkv, g = pair - unit * a.Hkv, layer = unit / a.new_seqs;
    const int p = a.parents[unit - layer * a.new_seqs];
    int len = 0, held = 0;
    if (p >= 0 && p < a.seqs) {
      const int64_t from = ((int64_t)layer * a.seqs + p) * a.Hkv + g;
      len = a.lengths[from], held = a.held[from];
      bad = len < 0 || held < 0 || held > a.pool.max_pages;
      if (bad) len = held = 0;       // nothing to go on from
      const int32_t* const src = a.table + from * a.pool.max_pages;
      int32_t* const dst = a.new_table + (int64_t)pair * a.pool.max_pages;
#pragma unroll 4
      for (int s = lane; s < held; s += 32) dst[s] = src[s];
    } else {
      bad = p != -1;
    }
    if (lane == 0) a.new_lengths[pair] = len, a.new_held[pair] = held;
  } else if (w - fresh < old) {
    const int pair = (int)(w - fresh), unit = pair / a.Hkv, seq = unit % a.seqs;
    int more = a.keep_old ? 0 : -1;
    for (int i = 0; i < a.new_seqs; i += 32) more += __popc(__ballot_sync(0xffffffffu, i + lane < a.new_seqs && a.parents[i + lane] == seq));
    const int len = a.lengths[pair], have = a.held[pair];
    bad = len < 0 || have < 0 || have > a.pool.max_pages;
    const int held = bad ? 0 : have;
    for (int s = lane; more && s < held; s += 32) {
      const int page = a.table[(int64_t)pair * a.pool.max_pages + s];
      // A page that is held has been counted.  Children of one that is not are counted all the same: an addition that is undone could pass for a
      // holder's in between.
      if ((unsigned)page >= (unsigned)a.pool.n_pages) bad = true;
      else if (atomicAdd(&a.refs[page], more) >= 1) continue;
      else if (bad = true; more < 0) atomicSub(&a.refs[page], more);
    }
  }
  if (bad) report_status(a.status, kStatusPage);
}

Pool pool_of(const ckv_paged& pg, void* k_pages, void* v_pages) {
  const int e = pg.dtype == CKV_BF16 ? 2 : 4;
  Pool p{(char*)k_pages, (char*)v_pages, pg.page_stride * e, pg.page_stride_row * e, 0, pg.page_size, pg.n_pages, pg.max_pages};
  while ((1 << p.log_p) < pg.page_size) ++p.log_p;
  return p;
}
template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), int64_t grid, int threads, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid), cfg.blockDim = dim3(threads), cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// A warp moves lists of up to a few dozen rows, a CTA longer ones (n_rows / n_lists: the room a list has, whatever its length).
cudaError_t launch_keep_rows(const ckv_paged& pg, Lists lists, int n_lists, const int32_t* rows, int n_rows, const int32_t* begins,
                             const int32_t* counts, const int32_t* tails, const int32_t* refs, const int32_t* lengths,
                             const int32_t* table, void* k_pages, void* v_pages, int32_t* new_lengths, int* status, cudaStream_t st) {
  KeepArgs a{pool_of(pg, k_pages, v_pages), lists, pg.n_units * pg.n_kv_heads, n_rows, rows, begins, counts, tails, refs, lengths, table,
             new_lengths, status};
  int64_t groups = (int64_t)a.pairs * 2;
  int slices = 1, log_s = pg.dtype == CKV_BF16 ? 4 : 5;
  if (n_rows / n_lists <= 32) return launch(keep_rows_kernel<true>, (groups + kThreads / 32 - 1) / (kThreads / 32), kThreads, st, a, slices, log_s);
  while (log_s > 2 && groups * slices <= 148 / 2) slices *= 2, --log_s;
  groups *= slices;
  int threads = kKeepThreads;
  while (threads > 128 && (groups * threads > 148 * kKeepThreads || (threads * 4 >> log_s) > n_rows / n_lists)) threads /= 2;
  return launch(keep_rows_kernel<false>, groups, threads, st, a, slices, log_s);
}

cudaError_t launch_pages_reserve(const ckv_paged& pg, Lists lists, const int32_t* new_rows, const int32_t* lengths, int32_t* held,
                                 int32_t* table, int32_t* refs, void* k_pages, void* v_pages, int32_t* room, char* ws,
                                 cudaStream_t st) {
  const int pairs = pg.n_units * pg.n_kv_heads;
  const ReserveWs w = reserve_ws(pairs, pg.n_pages);
  ReserveArgs a{};
  a.pool = pool_of(pg, k_pages, v_pages), a.lists = lists, a.pairs = pairs;
  a.new_rows = new_rows, a.lengths = lengths, a.held = held, a.table = table, a.refs = refs, a.room = room;
  a.status = reinterpret_cast<int*>(ws);
  a.chunk = w.chunk, a.n_chunks = w.n_chunks, a.n_blocks = w.n_blocks;
  a.free_bits = reinterpret_cast<uint32_t*>(ws + w.free_bits), a.shared_bits = reinterpret_cast<uint32_t*>(ws + w.shared_bits);
  a.chunk_free = reinterpret_cast<int32_t*>(ws + w.chunk_free), a.block_need = reinterpret_cast<int32_t*>(ws + w.block_need);
  a.need = reinterpret_cast<int2*>(ws + w.need);
  constexpr int kWarps = kThreads / 32;
  cudaError_t e = launch(reserve_count_kernel, w.n_chunks + (w.n_blocks + kWarps - 1) / kWarps, kThreads, st, a);
  if (e != cudaSuccess) return e;
  const int log_row = pg.dtype == CKV_BF16 ? 4 : 5;
  // Copies want many warps, each of which has few pairs; a call without any wants few CTAs, since each adds the needs up (8192 pairs: 8
  // pairs a CTA 72 us with a copy each and 13.7 with none, 16 pairs 74 and 12.3, 32 pairs 79 and 12.3; 1024 pairs with copies: 25, 33, 47).
  const auto grid = [&](int per) { return w.n_chunks + (pairs + per - 1) / per; };
  return pairs <= 148 * 4    ? launch(reserve_apply_kernel<1>, grid(1), kThreads, st, a, log_row)
         : pairs <= 148 * 32 ? launch(reserve_apply_kernel<8>, grid(8), kThreads, st, a, log_row)
                             : launch(reserve_apply_kernel<16>, grid(16), kThreads, st, a, log_row);
}

cudaError_t launch_pages_trim(const ckv_paged& pg, const int32_t* lengths, int32_t* held, const int32_t* table, int32_t* refs,
                              int* status, cudaStream_t st) {
  const int pairs = pg.n_units * pg.n_kv_heads;
  int log_t = 3;       // until the SMs are full, or a pair's threads have a page each
  while (log_t < 8 && (int64_t)pairs << log_t < 148 * 1024 && (1 << log_t) < pg.max_pages) ++log_t;
  const int per = kThreads >> log_t;
  return launch(pages_trim_kernel, (pairs + per - 1) / per, kThreads, st, pool_of(pg, nullptr, nullptr), pairs, log_t, lengths, held, table, refs, status);
}

cudaError_t launch_pages_fork(const ckv_paged& pg, int layers, int new_seqs, const int32_t* parents, const int32_t* lengths,
                              const int32_t* held, const int32_t* table, int32_t* refs, int keep_old, int32_t* new_lengths,
                              int32_t* new_held, int32_t* new_table, int* status, cudaStream_t st) {
  ForkArgs a{pool_of(pg, nullptr, nullptr), pg.n_kv_heads, layers, pg.n_units / layers, new_seqs, keep_old, parents, lengths, held, table,
             refs, new_lengths, new_held, new_table, status};
  const int64_t warps = (int64_t)layers * (new_seqs + a.seqs) * a.Hkv;
  return launch(pages_fork_kernel, (warps + kThreads / 32 - 1) / (kThreads / 32), kThreads, st, a);
}

}  // namespace ckv
