// Attention of longer chunks over the pages: bf16 on the tensor cores (tcgen05 + TMA), one persistent CTA per SM.
//
// An item is up to two tiles of 128 query rows of one (unit, KV head): a tile holds whole tokens, row = token * G + head, so one TMA
// box {G heads, 128 / G tokens} of q is a K-major operand.  Keys and values come in tiles of 128 rows, one TMA box per page and
// 64-dimension half, into a ring of five 32 KB stages (K0 V0 K1 V1 ...).  Per tile of keys and query tile s ("stream"):
//   S_s = Q_s K^T     M = N = K = 128, into 128 TMEM columns
//   P_s = 2^(x - m)   one thread per row: a row's 128 logits are one thread's registers, so maximum and sum need no shuffles;
//                     P goes back as bf16 over the columns S came from (the rounding tensor cores want; the sum l is of the
//                     unrounded values)
//   O_s += P_s V      A = P from TMEM, V as it lies in memory ([keys][dims], MN-major B), into 128 TMEM columns
// The two streams take turns: while the tensor cores run one stream's products the other's softmax runs on the CUDA cores.
// Both sides need about 1024 clocks per tile (4.2 MFMA at 4096 per clock; 16384 exponentials at 16 per clock).
// The running maximum is only raised when a row exceeds it by more than 2^8 (P <= 256 then loses nothing in bf16 and
// the fp32 sums): O is rescaled in TMEM a few times per item instead of at every tile, by the softmax threads themselves.
// Warps 0-3 and 4-7: softmax of stream 0 and 1; warp 8: MMA issue; warp 9: TMA; warps 10, 11 only make the launch a multiple of
// a warpgroup.  Registers are split 208 / 88 by setmaxnreg (256 * 208 + 128 * 88 = 384 * 168, the launch's total).
// Every wait is bounded and reports CKV_ERR_TIMEOUT through the status word.
#include "paged_work.cuh"
#include "tc_ptx.cuh"

namespace ckv {
namespace {

using namespace ptx;

constexpr int kThreads = 384;
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
constexpr int kStages = 5;
constexpr int kTile = 128;
constexpr uint32_t kHalf = 128 * 128;          // 128 rows x 64 bf16
constexpr uint32_t kTileBytes = 2 * kHalf;
constexpr int kInfo = 8;                       // ring of per-tile notes from the loader
constexpr float kRaise = 8.0f;                 // how far (in powers of two) a row may exceed its reference before O is rescaled
constexpr uint32_t kIdescQK = (1u << 4) | (1u << 7) | (1u << 10) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
constexpr uint32_t kIdescPV = kIdescQK | (1u << 16);   // B (the values) is MN-major
constexpr uint32_t kNegateA = 1u << 13;
constexpr uint32_t kColS = 0, kColO = 256;     // TMEM columns: S_0, S_1, O_0, O_1

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

struct __align__(1024) Smem {
  uint8_t kv[kStages][kTileBytes];
  uint8_t q[2][kTileBytes];
  uint64_t full[kStages], empty[kStages];
  uint64_t q_full, q_empty;
  uint64_t s_full[2], p_full[2], pv_done[2];
  uint64_t join_full, join_done;                // stream 1's result is there; stream 0 has read it
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

// How an item is cut up.  Two query tiles: each stream has one, and takes every key tile.  One query tile (the tokens
// fill no more than half of the block): both streams work on it, on every other key tile, and join at the end.
__device__ __forceinline__ bool paired(const Item& it) { return it.weight == 2; }

// First row of the item's j-th key tile that the block's first token does not see (128: it sees them all).  Where every
// token sees every row there is none.
__device__ __forceinline__ int late_row(const TcArgs& a, const Item& it, int j) {
  if (!a.w.causal) return kTile;
  const int sees = min(max(it.len - it.n + it.block * a.w.tokens + 1, 0), it.len);
  return min(max(sees - (it.t0 + j) * kTile, 0), kTile);
}

__device__ __forceinline__ void load_role(const TcArgs& a, Smem& sm, const CUtensorMap* qm, const CUtensorMap* km,
                                          const CUtensorMap* vm, const Waiter& w, int lane) {
  Walk k;
  k.start(a.w, sm.plan);
  uint32_t n_loads = 0, n_items = 0, n_tiles = 0;
  const int slot_of_lane = lane >> 1, half = lane & 1;
  const bool copies = slot_of_lane < a.pages_per_tile;
  const int tiles_per_page = a.w.P > kTile ? a.w.P / kTile : 1;
  for (; k.live; k.next(a.w)) {
    const Item& it = k.it;
    const int ns = it.weight;
    if (!wait_warp(smem_u32(&sm.q_empty), (n_items & 1) ^ 1, w, 1)) return;
    if (lane == 0) bar_arrive_tx(smem_u32(&sm.q_full), ns * a.q_bytes);
    __syncwarp();
    if (lane < 2 * ns)   // lane: (tile, half)
      tma_load_4d(qm, smem_u32(&sm.q[lane >> 1][(lane & 1) * kHalf]), smem_u32(&sm.q_full), 0, it.g * a.w.G,
                  it.first + it.block * a.w.tokens + (lane >> 1) * a.TQ, lane & 1);
    const int32_t* table = a.w.table + ((int64_t)it.u * a.w.Hkv + it.g) * a.w.max_pages;
    for (int t = it.t0; t < it.t1; ++t, ++n_tiles) {
      // the pages of this tile that hold visible rows
      const int first_row = t * kTile + slot_of_lane * (a.w.P < kTile ? a.w.P : kTile);
      const bool wanted = copies && first_row < it.visible;
      const int page = wanted ? table[first_row >> a.w.log_p] : 0;
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
        if (copy)
          tma_load_4d(kv ? vm : km, smem_u32(&sm.kv[s][half * kHalf + slot_of_lane * a.page_bytes]), smem_u32(&sm.full[s]), 0,
                      row_in_page, half, page);
      }
    }
    ++n_items;
  }
}

// 0 * NaN is not 0: value rows that no query sees are zeroed, and so are rows with an infinity or a NaN that some of the
// block's tokens do not see yet (the softmax threads add those to the tokens that do).
__device__ __forceinline__ void clean_values(const TcArgs& a, Smem& sm, const Item& it, int j, uint32_t nv, uint32_t n_tiles, int lane) {
  const int valid = it.visible - (it.t0 + j) * kTile, late = late_row(a, it, j);
  const uint32_t bad = *(volatile uint32_t*)&sm.bad[n_tiles % kInfo];
  if (valid < kTile || bad || late < kTile) {
    uint4* v = reinterpret_cast<uint4*>(sm.kv[nv % kStages]);
    if (lane < 4) sm.odd[n_tiles % kInfo][lane] = 0u;
    __syncwarp();
    const int piece = (lane & 8) * (kTile) + (lane & 7);      // 16-byte piece lane & 15 of a row: its half, its place
#pragma unroll 4
    for (int r0 = late; r0 < min(valid, kTile); r0 += 2) {
      const int row = min(r0 + (lane >> 4), kTile - 1);
      const uint4 x = v[piece + row * 8];
      const uint32_t e = 0x7f807f80u;
      const uint32_t hit = __vcmpeq2(x.x & e, e) | __vcmpeq2(x.y & e, e) | __vcmpeq2(x.z & e, e) | __vcmpeq2(x.w & e, e);
      const uint32_t any = __ballot_sync(0xffffffffu, hit != 0u && row < valid);
      if (any) {
        if ((any >> (lane & 16)) & 0xffffu) v[piece + row * 8] = make_uint4(0u, 0u, 0u, 0u);
        if ((lane & 15) == 0 && ((any >> lane) & 0xffffu)) atomicOr(&sm.odd[n_tiles % kInfo][row >> 5], 1u << (row & 31));
      }
    }
    if (valid < kTile || bad)
      for (int e = lane; e < 2 * kTile * 8; e += 32) {
        const int row = (e >> 3) & (kTile - 1);
        if (row >= valid || (bad >> (row >> a.w.log_p) & 1)) v[e] = make_uint4(0u, 0u, 0u, 0u);
      }
    fence_async_smem();
    __syncwarp();
  }
}

__device__ __forceinline__ void mma_role(const TcArgs& a, Smem& sm, uint32_t tmem, const Waiter& w, int lane) {
  Walk k;
  k.start(a.w, sm.plan);
  uint32_t n_use = 0, n_items = 0, n_tiles = 0, n_p[2] = {0, 0};
  const uint32_t q_lo[2] = {desc_lo(smem_u32(sm.q[0]), 16), desc_lo(smem_u32(sm.q[1]), 16)};
  const uint32_t kv0 = smem_u32(sm.kv[0]);
  auto full = [&](uint32_t n) { return wait_warp(smem_u32(&sm.full[n % kStages]), (n / kStages) & 1, w, 3); };
  auto release = [&](uint32_t n) {
    if (elect()) tc_commit(smem_u32(&sm.empty[n % kStages]));
  };
  auto qk = [&](int s, int q_tile, uint32_t n) {   // S_s = Q K^T
    if (elect()) {
      const uint32_t b = desc_lo(kv0 + (n % kStages) * kTileBytes, 16);
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {   // 16 dimensions = 32 bytes of a 128-byte swizzled row; the second half is 16 KB on
        const uint32_t off = (kk & 3) * 2 + (kk >> 2) * (kHalf >> 4);
        mma_ss(tmem + kColS + s * 128, desc_of(q_lo[q_tile] + off), desc_of(b + off), a.idesc_qk, kk > 0);
      }
      tc_commit(smem_u32(&sm.s_full[s]));
    }
  };
  auto pv = [&](int s, uint32_t n, bool accumulate) {   // O_s += P_s V, once P_s is there
    if (!wait_warp(smem_u32(&sm.p_full[s]), n_p[s] & 1, w, 5)) return false;
    ++n_p[s];
    tc_fence_after();
    if (elect()) {
      const uint32_t b = desc_lo(kv0 + (n % kStages) * kTileBytes, kHalf);   // 64-dimension halves 16 KB apart
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)     // 16 keys = 16 rows of 128 bytes
        mma_ts(tmem + kColO + s * 128, tmem + kColS + s * 128 + kk * 8, desc_of(b + kk * (2048 >> 4)), kIdescPV,
               accumulate || kk > 0);
      tc_commit(smem_u32(&sm.pv_done[s]));
    }
    return true;
  };
  // The products of one stream are issued in the order S(j), O(j), S(j + 1): the tensor pipe runs them in that order, so S(j + 1)
  // may take the columns that O(j) reads P from without waiting for it.
  for (; k.live; k.next(a.w)) {
    const Item& it = k.it;
    const int n = it.t1 - it.t0;
    const bool pair = paired(it);
    const int ahead = pair ? 1 : 2;      // a stream's next key tile
    if (!wait_warp(smem_u32(&sm.q_full), n_items & 1, w, 4)) return;
    for (int j = 0; j < min(ahead, n); ++j) {
      if (!full(n_use + 2 * j)) return;
      tc_fence_after();
      qk(j, 0, n_use + 2 * j);
      if (pair) qk(1, 1, n_use + 2 * j);
      release(n_use + 2 * j);
      if (j == n - 1 && elect()) tc_commit(smem_u32(&sm.q_empty));
    }
    for (int j = 0; j < n; ++j, ++n_tiles) {
      const uint32_t nv = n_use + 2 * j + 1, nk = n_use + 2 * (j + ahead);
      const bool more = j + ahead < n;
      if (!full(nv)) return;
      clean_values(a, sm, it, j, nv, n_tiles, lane);
      const int s = pair ? 0 : j & 1;
      if (!pv(s, nv, j >= ahead)) return;
      if (!pair) release(nv);
      if (more) {
        if (!full(nk)) return;
        tc_fence_after();
        qk(s, 0, nk);
        if (!pair) release(nk);
      }
      if (pair) {
        if (!pv(1, nv, j > 0)) return;
        release(nv);
        if (more) {
          qk(1, 1, nk);
          release(nk);
        }
      }
      if (more && j + ahead == n - 1 && elect()) tc_commit(smem_u32(&sm.q_empty));
    }
    n_use += 2 * n;
    ++n_items;
  }
}

// The exponentials of one tile of one row, to TMEM as bf16; returns their sum.
__device__ __forceinline__ float softmax_tile(float (&s)[kTile], float scale, float ref, uint32_t p_addr) {
  uint64_t sum[4] = {0, 0, 0, 0};
  const uint64_t sc = pack2(scale, scale), mr = pack2(-ref, -ref);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    uint32_t p[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      float a, b;
      unpack2(fma2(pack2(s[c * 64 + 2 * i], s[c * 64 + 2 * i + 1]), sc, mr), a, b);
      a = ex2(a), b = ex2(b);
      sum[i & 3] = add2(sum[i & 3], pack2(a, b));
      p[i] = bf16x2(a, b);
    }
    tmem_st32(p_addr + c * 32, p);
  }
  float a, b;
  unpack2(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), a, b);
  return a + b;
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
  Walk k;
  k.start(a.w, sm.plan);
  uint32_t n_s = 0, n_all = 0, n_join = 0;   // tiles of this stream so far; key tiles of the CTA; joins of the streams
  const int r = quarter * 32 + lane;                        // row of the query tile
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  const uint32_t s_addr = tmem + lanes + kColS + stream * 128, o_addr = tmem + lanes + kColO + stream * 128;
  const uint32_t bar_s = smem_u32(&sm.s_full[stream]), bar_p = smem_u32(&sm.p_full[stream]), bar_o = smem_u32(&sm.pv_done[stream]);
  for (; k.live; k.next(a.w)) {
    const Item& it = k.it;
    const int n = it.t1 - it.t0;
    const bool pair = paired(it);
    const int j0 = pair ? 0 : stream, step = pair ? 1 : 2, q_tile = pair ? stream : 0;
    const int tok0 = it.block * a.w.tokens + q_tile * a.TQ;   // first token of the tile
    const int token = tok0 + r / a.w.G;
    const bool live = r < a.TQ * a.w.G && token < it.n;
    auto limit_of = [&](int tk) { return a.w.causal ? min(max(it.len - it.n + tk + 1, 0), it.len) : it.len; };
    const int limit = live ? limit_of(token) : 0, least = limit_of(tok0);
    float m = -INFINITY, l = 0.f;
    for (int j = j0; j < n; j += step, ++n_s) {
      const int key0 = (it.t0 + j) * kTile;
      if (!wait_warp(bar_s, n_s & 1, w, 6)) return;
      tc_fence_after();
      uint32_t raw[kTile];
      tmem_ld128(s_addr, raw);
      float s[kTile];
#pragma unroll
      for (int i = 0; i < kTile; ++i) s[i] = __uint_as_float(raw[i]);
      const uint32_t bad = *(volatile uint32_t*)&sm.bad[(n_all + j) % kInfo];
      if (key0 + kTile > least || bad) {
#pragma unroll
        for (int i = 0; i < kTile; ++i)
          if (key0 + i >= limit || (bad >> (i >> a.w.log_p) & 1)) s[i] = -INFINITY;
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < kTile; i += 8) {
#pragma unroll
        for (int c = 0; c < 4; ++c) mx[c] = max3(mx[c], s[i + 2 * c], s[i + 2 * c + 1]);
      }
      const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * a.x_scale;
      const bool raise = top > m + kRaise;                    // the first visible key: m is -infinity
      if (__any_sync(0xffffffffu, raise)) {
        const float f = raise ? ex2(m - top) : 1.0f;
        if (raise) m = top;
        l *= f;
        if (j > j0) {
          if (!wait_warp(bar_o, (n_s - 1) & 1, w, 7)) return;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t o[32];
            tmem_ld32(o_addr + c * 32, o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st32(o_addr + c * 32, o);
          }
        }
      }
      l += softmax_tile(s, a.x_scale, m == -INFINITY ? 0.f : m, s_addr);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bar_p);
    }
    // the item's output: normalised, or a partial result for the join
    if (j0 < n) {
      if (!wait_warp(bar_o, (n_s - 1) & 1, w, 7)) return;
      tc_fence_after();
    }
    // value rows that were left out because they are not finite, for the tokens that see them
    for (int j = n - 1; j >= 0 && late_row(a, it, j) < kTile; --j) {
      if (!pair && (j & 1) != stream) continue;
      for (int x = 0; x < 4; ++x) {
        uint32_t odd = *(volatile uint32_t*)&sm.odd[(n_all + j) % kInfo][x];
        for (; odd; odd &= odd - 1) add_row(a, it, o_addr, (it.t0 + j) * kTile + x * 32 + __ffs(odd) - 1, limit, token, r % a.w.G, m);
      }
    }
    n_all += n;
    // one query tile: stream 1 leaves its maximum and sum, stream 0 takes its output from TMEM (the same lanes, other columns)
    float f0 = 1.0f, f1 = 0.f;
    if (!pair && n > 1) {
      if (stream == 1) {
        sm.other[r] = make_float2(m, l);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(smem_u32(&sm.join_full));
        if (!wait_warp(smem_u32(&sm.join_done), n_join & 1, w, 8)) return;
        tc_fence_after();
        ++n_join;
        continue;
      }
      if (!wait_warp(smem_u32(&sm.join_full), n_join & 1, w, 8)) return;
      tc_fence_after();
      ++n_join;
      const float2 x = sm.other[r];
      const float top = fmaxf(m, x.x), ref = top == -INFINITY ? 0.f : top;
      f0 = ex2(m - ref), f1 = ex2(x.x - ref);
      l = l * f0 + x.y * f1, m = top;
    } else if (!pair && stream == 1) {
      continue;
    }
    const bool joined = !pair && n > 1;
    const bool whole = it.t0 == 0 && it.t1 == it.tiles;
    const int which = it.t0 > 0 ? 0 : 1;
    const int br = q_tile * a.TQ * a.w.G + r;                // row of the block
    const bool none = m == -INFINITY;
    const float inv = none ? 0.f : 1.0f / l;
    const int64_t slot = ((int64_t)blockIdx.x * 2 + which) * a.w.slot_rows + br;
    const int64_t at = (int64_t)(it.first + token) * a.w.H + it.g * a.w.G + r % a.w.G;
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
        uint4* dst = reinterpret_cast<uint4*>(a.out + at * kHeadDim + c * 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t p[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            p[e] = bf16x2(none ? 0.f : __uint_as_float(o[8 * i + 2 * e]) * inv, none ? 0.f : __uint_as_float(o[8 * i + 2 * e + 1]) * inv);
          dst[i] = make_uint4(p[0], p[1], p[2], p[3]);
        }
      } else {
        uint4* dst = reinterpret_cast<uint4*>(a.w.o + slot * kHeadDim + c * 32);
#pragma unroll
        for (int i = 0; i < 8; ++i) dst[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
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
      sp[2 * which] = k.pair, sp[2 * which + 1] = k.block;
    }
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
    for (int i = 0; i < kStages; ++i) bar_init(smem_u32(&sm.full[i]), 1), bar_init(smem_u32(&sm.empty[i]), 1);
    bar_init(smem_u32(&sm.q_full), 1), bar_init(smem_u32(&sm.q_empty), 1);
    for (int s = 0; s < 2; ++s)
      bar_init(smem_u32(&sm.s_full[s]), 1), bar_init(smem_u32(&sm.p_full[s]), 4), bar_init(smem_u32(&sm.pv_done[s]), 1);
    bar_init(smem_u32(&sm.join_full), 4), bar_init(smem_u32(&sm.join_done), 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
    sm.abort_flag = 0;
  }
  tc_fence_before();
  pdl_wait();
  make_plan<kThreads>(a.w, blockIdx.x, gridDim.x, sm.plan);
  pdl_launch_dependents();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  if (threadIdx.x == 0) a.w.split[blockIdx.x] = make_int4(-1, -1, -1, -1);
  __syncthreads();
  const Waiter w{&sm.abort_flag, a.w.status, a.wait_ns};
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    softmax_role(a, sm, tmem, w, warp >> 2, warp & 3, lane);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 8) mma_role(a, sm, tmem, w, lane);
    if (warp == 9) load_role(a, sm, &qm, &km, &vm, w, lane);
  }
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

cudaError_t launch_attend_tc(const ckv_paged& pg, const WorkArgs& base, float scale, const void* q, const void* k_pages,
                             const void* v_pages, void* out, float* lse, cudaStream_t st) {
  TcArgs a{};
  a.w = base;
  a.TQ = kTile / base.G;
  a.w.tokens = 2 * a.TQ, a.w.M = a.w.tokens * base.G, a.w.tile = kTile, a.w.granule = 2;
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
    cudaError_t r = cudaFuncSetAttribute(attend_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
    // setmaxnreg hands out what the launch holds: a build with fewer registers would wait for ever
    cudaFuncAttributes attrs;
    if (r == cudaSuccess) r = cudaFuncGetAttributes(&attrs, attend_tc_kernel);
    if (r == cudaSuccess && attrs.numRegs * kThreads < kSoftmaxRegs * 256 + kOtherRegs * 128) r = cudaErrorLaunchOutOfResources;
    return r;
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(kWorkers), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = sizeof(Smem), cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, attend_tc_kernel, qm, km, vm, a);
  count_launch();
  return e != cudaSuccess ? e : launch_join<true>(a.w, kWorkers, out, lse, st);
}

}  // namespace ckv
