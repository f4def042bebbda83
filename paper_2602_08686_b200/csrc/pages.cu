// The pages of a cache: rows moved together inside them, pages reserved, given back, and shared with new sequences.
// All of it moves whole rows (256 or 512 bytes, in 16-byte pieces) and counts; what is decided on the device depends on the inputs
// alone: page numbers are handed out by rank, counts change by commutative atomics.
#include "pages.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 256;

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
struct KeepArgs {
  Pool pool;
  Lists lists;
  int pairs, n_rows;
  const int32_t *rows, *begins, *counts, *tails, *refs, *lengths, *table;
  int32_t* new_lengths;
  int* status;
};

template <bool kWarp>
__device__ __forceinline__ bool all_of(bool x) {
  if (kWarp) return __all_sync(0xffffffffu, x);
  return __syncthreads_and(x);
}

// A group is a warp (short lists) or a CTA.  slices: of a row; log_s: log2 of the 16-byte pieces in a slice.
template <bool kWarp>
__global__ void __launch_bounds__(kThreads) keep_rows_kernel(KeepArgs a, int slices, int log_s) {
  constexpr int NT = kWarp ? 32 : kThreads, U = 4;
  __shared__ int s_first;
  pdl_wait();
  pdl_launch_dependents();
  const int group = kWarp ? blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5) : blockIdx.x;
  const int t = kWarp ? threadIdx.x & 31 : threadIdx.x;
  const int pair = group / (2 * slices), which = group - pair * 2 * slices;
  if (pair >= a.pairs) return;
  const int list = a.lists.of(pair), len = a.lengths[pair], count = a.counts[list], begin = a.begins[list];
  const int span = a.tails ? a.tails[list] : len, base = len - span;
  const int32_t* const rows = a.rows + begin;
  const int32_t* const table = a.table + (int64_t)pair * a.pool.max_pages;
  if (!kWarp) {
    if (threadIdx.x == 0) s_first = 0x7fffffff;
    __syncthreads();
  }
  const bool sane = len >= 0 && len <= a.pool.max_pages << a.pool.log_p && span >= 0 && span <= len && count >= 0 && count <= span &&
                    begin >= 0 && count <= a.n_rows && begin <= a.n_rows - count;
  bool ok = sane;
  int first = 0x7fffffff;      // the first entry that moves
  if (sane)
    for (int i = t; i < count; i += NT) {
      const int x = rows[i];
      if (x <= (i ? rows[i - 1] : -1) || x >= span) ok = false;
      if (x != i) first = min(first, i);
    }
  if (kWarp) {
    first = __reduce_min_sync(0xffffffffu, first);
  } else {
    if (first < 0x7fffffff) atomicMin(&s_first, first);
  }
  ok = all_of<kWarp>(ok);
  if (!kWarp) first = s_first;
  if (ok && first < count) {   // the pages of the rows that move; those written are the pair's alone
    const int to = (base + count - 1) >> a.pool.log_p, end = (base + rows[count - 1]) >> a.pool.log_p;
    bool fine = true;
    for (int s = ((base + first) >> a.pool.log_p) + t; s <= end; s += NT) {
      const int page = table[s];
      if ((unsigned)page >= (unsigned)a.pool.n_pages) fine = false;
      else if (a.refs && s <= to && a.refs[page] > 1) fine = false;
    }
    ok = all_of<kWarp>(fine);
  }
  if (which == 0 && t == 0) {
    a.new_lengths[pair] = ok ? base + count : len;
    if (!ok) report_status(a.status, kStatusPage);
  }
  if (!ok) return;
  const bool values = which >= slices;
  char* const data = (values ? a.pool.v : a.pool.k) + ((((values ? which - slices : which) << log_s) + (t & ((1 << log_s) - 1))) << 4);
  auto at = [&](int row) {
    return reinterpret_cast<uint4*>(data + table[row >> a.pool.log_p] * a.pool.page + (row & (a.pool.P - 1)) * a.pool.row);
  };
  const int R = NT >> log_s, r = t >> log_s;
  for (int i0 = first; i0 < count; i0 += U * R) {
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * R + r < count) x[u] = *at(base + rows[i0 + u * R + r]);
    if (kWarp) __syncwarp();
    else __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * R + r < count) *at(base + i0 + u * R + r) = x[u];
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
// Bound: latency (two launches, about five dependent reads each); with many copies HBM.
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

// What a pair wants: its first slot to be written and the number of slots it wants to hold (0: nothing).
struct Want {
  int first, slots, rows;    // rows in the first slot's page
};
__device__ __forceinline__ Want want_of(const ReserveArgs& a, int pair, bool& bad) {
  const int len = a.lengths[pair], more = a.new_rows[a.lists.of(pair)];
  bad |= len < 0 || more < 0;
  if (len < 0 || more <= 0) return {0, 0, 0};
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
    const Want w = want_of(a, pair, bad);
    int held = a.held[pair];
    bad |= held < 0 || held > a.pool.max_pages;
    held = min(max(held, 0), a.pool.max_pages);
    for (int s = w.first; s < min(held, w.slots); ++s) {
      const int page = a.table[(int64_t)pair * a.pool.max_pages + s];
      if ((unsigned)page >= (unsigned)a.pool.n_pages) bad = true;
      else copies += a.refs[page] > 1;
    }
    need = copies + max(w.slots - held, 0);
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

// Sums of ints over the CTA: `before` of those with index < at, `total` of all.
struct Sums {
  long long before, total;
};
__device__ __forceinline__ Sums add_up(const int32_t* x, int n, int at, long long* s_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long b = 0, t = 0;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int v = x[i];
    t += v;
    if (i < at) b += v;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) b += __shfl_xor_sync(0xffffffffu, b, d), t += __shfl_xor_sync(0xffffffffu, t, d);
  if (lane == 0) s_sum[warp * 2] = b, s_sum[warp * 2 + 1] = t;
  __syncthreads();
  Sums s{0, 0};
  for (int w = 0; w < kThreads / 32; ++w) s.before += s_sum[w * 2], s.total += s_sum[w * 2 + 1];
  __syncthreads();
  return s;
}
// Exclusive prefix sums of n ints (at most kMaxChunks; sums below 2^31) in shared memory.
__device__ __forceinline__ void prefix(const int32_t* x, int n, int32_t* out, int* s_part) {
  const int per = (n + kThreads - 1) / kThreads, lo = min((int)threadIdx.x * per, n), hi = min(lo + per, n);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int mine = 0;
  for (int i = lo; i < hi; ++i) mine += x[i];
  int sum = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, sum, d);
    if (lane >= d) sum += y;
  }
  if (lane == 31) s_part[warp] = sum;
  __syncthreads();
  int before = sum - mine;
  for (int w = 0; w < warp; ++w) before += s_part[w];
  for (int i = lo; i < hi; ++i) out[i] = before, before += x[i];
  __syncthreads();
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

// kWarp: a group per pair is a warp, else a CTA (few pairs).
template <bool kWarp>
__global__ void __launch_bounds__(kThreads) reserve_apply_kernel(ReserveArgs a, int row_bytes) {
  __shared__ int32_t s_prefix[kMaxChunks];
  __shared__ long long s_sum[kThreads / 32 * 2];
  __shared__ int s_part[kThreads / 32], s_count[kThreads / 32], s_page[2];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool pages = (int)blockIdx.x < a.n_chunks;
  const Sums need = add_up(a.block_need, a.n_blocks, 0, s_sum), have = add_up(a.chunk_free, a.n_chunks, blockIdx.x, s_sum);
  const bool enough = need.total <= have.total;
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.room) {
    a.room[0] = (int)(enough ? have.total - need.total : have.total);
    a.room[1] = (int)min(enough ? 0ll : need.total - have.total, 0x7fffffffll);
  }
  if (!enough) return;
  if (pages) {
    if (have.before >= need.total) return;
    prefix(a.block_need, a.n_blocks, s_prefix, s_part);
    int rank0 = (int)have.before;
    const int64_t begin = (int64_t)blockIdx.x * a.chunk;
    for (int w0 = 0; w0 < a.chunk / 32; w0 += kThreads / 32) {              // a word of 32 pages a warp
      const uint32_t bits = a.free_bits[begin / 32 + w0 + warp];
      if (lane == 0) s_count[warp] = __popc(bits);
      __syncthreads();
      int rank = rank0 + __popc(bits & ((1u << lane) - 1u));
      for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) rank += s_count[w];
        rank0 += s_count[w];
      }
      if ((bits >> lane & 1u) && rank < need.total) {
        const int block = last_at_most(s_prefix, a.n_blocks, rank), r = rank - s_prefix[block];
        int lo = block * kPairBlock, hi = min(lo + kPairBlock, a.pairs) - 1;   // the first pair of the block with more than r pages up to it
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (a.need[mid].x > r) hi = mid;
          else lo = mid + 1;
        }
        const int2 n = a.need[lo];
        const int before = lo > block * kPairBlock ? a.need[lo - 1].x : 0, mine = r - before;
        if (mine >= n.y) {
          bool bad = false;
          const Want w = want_of(a, lo, bad);
          const int page = (int)(begin + (w0 + warp) * 32 + lane);
          a.table[(int64_t)lo * a.pool.max_pages + w.slots - (n.x - before) + mine] = page;
          a.refs[page] = 1;
        }
      }
      __syncthreads();
      if (rank0 >= need.total) return;
    }
    return;
  }
  // pairs
  constexpr int NT = kWarp ? 32 : kThreads;
  const int group = (int)blockIdx.x - a.n_chunks, t = kWarp ? lane : threadIdx.x;
  const int pair0 = kWarp ? group * (kThreads / 32) : group, n_pairs = kWarp ? min(kThreads / 32, a.pairs - pair0) : 1;
  int any = 0;
  for (int p = 0; p < n_pairs; ++p) any |= a.need[pair0 + p].y;
  const int pair = kWarp ? pair0 + warp : pair0;
  const bool live = pair < a.pairs;
  bool bad = false;
  const Want w = live ? want_of(a, pair, bad) : Want{0, 0, 0};
  const int held = live ? a.held[pair] : 0;
  int2 n = make_int2(0, 0);
  int rank = 0;
  if (any) {                                                                // pages by rank
    if (live) {
      const int block = pair / kPairBlock;
      n = a.need[pair];
      for (int b = t; b < block; b += NT) rank += a.block_need[b];
      if (t == 0 && pair % kPairBlock) rank += a.need[pair - 1].x;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) rank += __shfl_xor_sync(0xffffffffu, rank, d);
    if (!kWarp) {
      if (lane == 0) s_count[warp] = rank;
      __syncthreads();
      rank = 0;
      for (int k = 0; k < kThreads / 32; ++k) rank += s_count[k];
    }
    prefix(a.chunk_free, a.n_chunks, s_prefix, s_part);
  }
  int32_t* const table = a.table + (int64_t)(live ? pair : 0) * a.pool.max_pages;
  for (int s = w.first; n.y > 0 && s < min(held, w.slots); ++s) {
    const int old = table[s];
    if ((unsigned)old >= (unsigned)a.pool.n_pages || !(a.shared_bits[old >> 5] >> (old & 31) & 1u)) continue;
    // the rank-th free page: its chunk, then a word a lane
    if (kWarp || warp == 0) {
      const int c = last_at_most(s_prefix, a.n_chunks, rank);
      int r = rank - s_prefix[c], page = -1;
      const uint32_t* words = a.free_bits + (int64_t)c * (a.chunk / 32);
      for (int w0 = 0; page < 0 && w0 < a.chunk / 32; w0 += 32) {
        const uint32_t bits = words[w0 + lane];
        int sum = __popc(bits);
        const int mine = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, sum, d);
          if (lane >= d) sum += x;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, sum > r);
        const int all = __shfl_sync(0xffffffffu, sum, 31);
        if (past) {
          const int from = __ffs(past) - 1;
          uint32_t b = bits;
          for (int k = r - (sum - mine); lane == from && k > 0; --k) b &= b - 1u;
          page = (int)((int64_t)c * a.chunk + (w0 + from) * 32 + __shfl_sync(0xffffffffu, (int)__ffs(b), from) - 1);
        }
        r -= all;
      }
      if (!kWarp && lane == 0) s_page[0] = page;
      if (kWarp && lane == 0) s_count[warp] = page;
    }
    if (kWarp) __syncwarp();
    else __syncthreads();
    const int page = kWarp ? s_count[warp] : s_page[0];
    if (s == w.first) {
      const int pieces = row_bytes >> 4, log_r = pieces == 16 ? 4 : 5, items = w.rows << log_r;
      for (int which = 0; which < 2; ++which) {
        char* const pool = which ? a.pool.v : a.pool.k;
        const char* const from = pool + old * a.pool.page;
        char* const to = pool + page * a.pool.page;
#pragma unroll 8
        for (int e = t; e < items; e += NT) {
          const int64_t off = (e >> log_r) * a.pool.row + ((e & (pieces - 1)) << 4);
          *reinterpret_cast<uint4*>(to + off) = *reinterpret_cast<const uint4*>(from + off);
        }
      }
    }
    if (kWarp) __syncwarp();
    else __syncthreads();
    if (t == 0) table[s] = page, a.refs[page] = 1, atomicSub(&a.refs[old], 1);
    ++rank;
  }
  if (live && t == 0 && w.slots > held) a.held[pair] = w.slots;
}

// ------------------------------------------------------------------------------------------------ pages given back
// Eight lanes a pair, four pages each at a time.
__global__ void __launch_bounds__(kThreads) pages_trim_kernel(Pool pool, int pairs, const int32_t* __restrict__ lengths, int32_t* __restrict__ held,
                                                              const int32_t* __restrict__ table, int32_t* __restrict__ refs, int* __restrict__ status) {
  pdl_wait();
  pdl_launch_dependents();
  const int pair = blockIdx.x * (kThreads / 8) + (threadIdx.x >> 3), l8 = threadIdx.x & 7;
  const bool live = pair < pairs;
  const int len = live && lengths ? lengths[pair] : 0, have = live ? held[pair] : 0;
  bool bad = len < 0 || have < 0 || have > pool.max_pages;
  const int end = min(have, pool.max_pages), keep = len < 0 ? have : (int)(((int64_t)len + pool.P - 1) >> pool.log_p);
  for (int s0 = keep + l8; s0 < end; s0 += 32) {
    int page[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) page[i] = s0 + 8 * i < end ? table[(int64_t)pair * pool.max_pages + s0 + 8 * i] : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (s0 + 8 * i >= end) continue;
      if ((unsigned)page[i] >= (unsigned)pool.n_pages) bad = true;
      else if (atomicSub(&refs[page[i]], 1) < 1) bad = true;
    }
  }
  __syncwarp();     // all eight have read `held`
  if (live && l8 == 0 && keep < have) held[pair] = keep;
  if (bad) report_status(status, kStatusPage);
}

// ------------------------------------------------------------------------------------------------ pages shared
// A warp per pair: those of the new sequences copy their parents' table rows, those of the old ones count their children in (and
// themselves out, where the old sequences end): one atomic a page whatever the number of children.
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
      bad = held < 0 || held > a.pool.max_pages;
      held = min(max(held, 0), a.pool.max_pages);
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
    const int held = min(a.held[pair], a.pool.max_pages);
    for (int s = lane; more && s < held; s += 32) {
      const int page = a.table[(int64_t)pair * a.pool.max_pages + s];
      if ((unsigned)page >= (unsigned)a.pool.n_pages) bad = true;
      else if (atomicAdd(&a.refs[page], more) < 1) bad = true;    // a page that is held has been counted
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
cudaError_t launch(void (*kernel)(P...), int64_t grid, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)grid), cfg.blockDim = dim3(kThreads), cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// A warp moves lists of up to a few dozen rows, a CTA longer ones: what counts is how long they are on average (n_rows is the room
// they have).  Slices: until there are groups enough to fill the SMs.
cudaError_t launch_keep_rows(const ckv_paged& pg, Lists lists, int n_lists, const int32_t* rows, int n_rows, const int32_t* begins,
                             const int32_t* counts, const int32_t* tails, const int32_t* refs, const int32_t* lengths,
                             const int32_t* table, void* k_pages, void* v_pages, int32_t* new_lengths, int* status, cudaStream_t st) {
  KeepArgs a{pool_of(pg, k_pages, v_pages), lists, pg.n_units * pg.n_kv_heads, n_rows, rows, begins, counts, tails, refs, lengths, table,
             new_lengths, status};
  const bool warp = n_rows / n_lists <= 32;
  int slices = 1, log_s = pg.dtype == CKV_BF16 ? 4 : 5;
  if (warp) return launch(keep_rows_kernel<true>, ((int64_t)a.pairs * 2 + kThreads / 32 - 1) / (kThreads / 32), st, a, slices, log_s);
  while (log_s > 2 && (int64_t)a.pairs * 2 * slices < 148 * 8) slices *= 2, --log_s;
  return launch(keep_rows_kernel<false>, (int64_t)a.pairs * 2 * slices, st, a, slices, log_s);
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
  cudaError_t e = launch(reserve_count_kernel, w.n_chunks + (w.n_blocks + kWarps - 1) / kWarps, st, a);
  if (e != cudaSuccess) return e;
  const int row_bytes = kHeadDim * (pg.dtype == CKV_BF16 ? 2 : 4);
  return pairs <= 148 * 4 ? launch(reserve_apply_kernel<false>, w.n_chunks + pairs, st, a, row_bytes)
                          : launch(reserve_apply_kernel<true>, w.n_chunks + (pairs + kWarps - 1) / kWarps, st, a, row_bytes);
}

cudaError_t launch_pages_trim(const ckv_paged& pg, const int32_t* lengths, int32_t* held, const int32_t* table, int32_t* refs,
                              int* status, cudaStream_t st) {
  const int pairs = pg.n_units * pg.n_kv_heads;
  return launch(pages_trim_kernel, (pairs + kThreads / 8 - 1) / (kThreads / 8), st, pool_of(pg, nullptr, nullptr), pairs, lengths, held,
                table, refs, status);
}

cudaError_t launch_pages_fork(const ckv_paged& pg, int layers, int new_seqs, const int32_t* parents, const int32_t* lengths,
                              const int32_t* held, const int32_t* table, int32_t* refs, int keep_old, int32_t* new_lengths,
                              int32_t* new_held, int32_t* new_table, int* status, cudaStream_t st) {
  ForkArgs a{pool_of(pg, nullptr, nullptr), pg.n_kv_heads, layers, pg.n_units / layers, new_seqs, keep_old, parents, lengths, held, table,
             refs, new_lengths, new_held, new_table, status};
  const int64_t warps = (int64_t)layers * (new_seqs + a.seqs) * a.Hkv;
  return launch(pages_fork_kernel, (warps + kThreads / 32 - 1) / (kThreads / 32), st, a);
}

}  // namespace ckv
