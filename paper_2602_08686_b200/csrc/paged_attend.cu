// Attention of new tokens over a paged cache: o = softmax(scale q k^T) v, causal inside the chunk, one pass over the
// keys with a running maximum m and sum l per query row,
//   m' = max(m, x),  l' = l 2^(m - m') + 2^(x - m'),  o' = o 2^(m - m') + 2^(x - m') v,   x = scale log2(e) q.k,
// which can be cut anywhere along the keys: partial (m, l, o) of any two ranges join by the same rule.
// A row that saw nothing is one whose sum is exactly zero: the largest logit adds one to it, and a NaN, which no maximum notices, a
// NaN, which goes on to the output and the lse.
//
// This file has the kernel for fp32 inputs, the join of split items and the choice of kernels.
//
// attend_rows_kernel: fp32 arithmetic on the CUDA cores, blocks of four query rows.  A warp takes eight keys at a
// time, eight lanes per key with 16 dimensions each: queries, keys, values and the output all stay in registers, nothing
// is staged, and each of the four groups of eight lanes keeps its own running (m, l, o); they join when the item ends.
// Bound: the latency of a step at eight warps an SM (255 registers a thread), for single tokens close to HBM: 8 sequences of
// 8192 rows in 110 us, 0.75 of the measured copy rate.
#include <cuda_bf16.h>

#include "paged_work.cuh"

namespace ckv {
namespace {

constexpr int kRowsM = 4;            // query rows of a block
constexpr int kRowsThreads = 256;
constexpr int kRowsWarps = kRowsThreads / 32;
constexpr int kRowsTile = kRowsWarps * 8;   // keys a CTA takes per step
constexpr ShortRule kShortRows{kRowsTile, 100, 300};

// the 16 dimensions of lane l8 of 8: 16-byte pieces l8, l8 + 8, ... of the row (coalesced over the eight lanes)
__device__ __forceinline__ void load16(const char* row, int l8, float (&x)[16]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float4 r = *reinterpret_cast<const float4*>(row + (c * 8 + l8) * 16);
    x[c * 4] = r.x, x[c * 4 + 1] = r.y, x[c * 4 + 2] = r.z, x[c * 4 + 3] = r.w;
  }
}
__device__ __forceinline__ int dim16(int l8, int i) { return ((i >> 2) * 8 + l8) * 4 + (i & 3); }   // dimension in x[i]

struct RowsSmem {
  Plan plan;
  float2 ml[kRowsWarps][kRowsM];
  float o[kRowsWarps][kRowsM][kHeadDim];
  float2 cta_ml[kRowsM];                       // the CTA's result, for the others of its cluster
  float cta_o[kRowsM][kHeadDim];
  Item it;                                     // of the cluster
};

// kCluster: every item is one cluster's, as in the bf16 kernel for few rows.  kTree: a tree's rows are seen by the bits of its tokens.
template <bool kCluster, bool kTree>
__global__ void __launch_bounds__(kRowsThreads, 1) attend_rows_kernel(WorkArgs a, ckv_paged pg, float x_scale,
                                                                      const char* __restrict__ q,
                                                                      const char* __restrict__ kp,
                                                                      const char* __restrict__ vp, float* __restrict__ out,
                                                                      float* __restrict__ lse, int n_cta) {
  constexpr int E = 4;
  __shared__ RowsSmem sm;
  pdl_wait();
  Walk walk;
  const int rank = kCluster ? (int)blockIdx.x % n_cta : 0, n_ranks = kCluster ? n_cta : 1;
  int index = kCluster ? (int)blockIdx.x / n_cta : 0, more = 0;   // of the cluster's item
  if (!kCluster) {
    make_plan<kRowsThreads>(a, blockIdx.x, gridDim.x, sm.plan);
    pdl_launch_dependents();
    if (threadIdx.x == 0) a.split[blockIdx.x] = make_int4(-1, -1, -1, -1);
    walk.start(a, sm.plan);
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l8 = lane & 7, grp = lane >> 3;
  for (;;) {
    if (kCluster) {   // the next item that has rows
      walk.live = false;
      for (; index < a.Nu * a.Hkv * a.blocks && !walk.cluster_item(a, index, more); more = 0) index += gridDim.x / n_cta;
    }
    if (!walk.live) break;
    const Item& now = walk.it;
    if (kCluster && threadIdx.x == 0) sm.it = now;
    const int rows = block_rows(a, now);
    float qr[kRowsM][16], acc[kRowsM][16], m[kRowsM], l[kRowsM];
    int limit[kRowsM];
#pragma unroll
    for (int r = 0; r < kRowsM; ++r) {
      m[r] = -INFINITY, l[r] = 0.f, limit[r] = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[r][i] = 0.f, qr[r][i] = 0.f;
      if (r < rows) {
        const int row = now.block * a.M + r, token = row / a.G, h = now.g * a.G + (row - token * a.G);
        load16(q + ((now.first + token) * pg.q_stride_tok + h * pg.q_stride_head) * E, l8, qr[r]);
        limit[r] = row_limit(a, now, r);
      }
    }
    const int end = min(now.t1 * a.tile, now.visible), step = n_ranks * a.tile;
    const int least = kTree ? rows_before_tree(now) : 0;
    // a warp's eight keys are in one page
    auto page_at = [&](int j) { return j + warp * 8 < end ? page_of(a, now, (j + warp * 8) >> a.log_p) : -1; };
    auto key_at = [&](int j, int s) { return j + warp * 8 + s * 4 + grp; };
    auto load = [&](const char* pool, int j, int page, float (&x)[2][16]) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const int key = key_at(j, s);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[s][i] = 0.f;
        if (page >= 0 && key < end) load16(pool + (page * pg.page_stride + (key & (a.P - 1)) * pg.page_stride_row) * E, l8, x[s]);
      }
    };
    int j0 = now.t0 * a.tile + rank * a.tile;
    int page = page_at(j0), next = page_at(j0 + step);
    float kv[2][16], vv[2][16];
    load(kp, j0, page, kv);
    load(vp, j0, page, vv);
    // The next keys are asked for when the logits are done, the next values when the output is.
    for (; j0 < end; j0 += step) {
      float x[2][kRowsM];
      int key[2] = {0x7fffffff, 0x7fffffff};
      bool raise = false;
      uint32_t hidden = 0;                     // kTree: bit (s, r): a key of the tree that is no ancestor of the row's token
      auto sees = [&](int s, int r) { return key[s] < limit[r] && (!kTree || !(hidden >> (s * kRowsM + r) & 1u)); };
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        key[s] = page >= 0 && key_at(j0, s) < end ? key_at(j0, s) : 0x7fffffff;   // hidden from every row
        if (kTree && key[s] >= least && key[s] < now.visible) {
#pragma unroll
          for (int r = 0; r < kRowsM; ++r)
            if (r < rows && !(tree_bits(tree_words_of(a, now, (now.block * a.M + r) / a.G), a.tree_words, key[s] - (now.len - now.n)) & 1u))
              hidden |= 1u << (s * kRowsM + r);
        }
#pragma unroll
        for (int r = 0; r < kRowsM; ++r) {
          float d = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) d = fmaf(qr[r][i], kv[s][i], d);
#pragma unroll
          for (int b = 1; b < 8; b <<= 1) d += __shfl_xor_sync(0xffffffffu, d, b);
          x[s][r] = sees(s, r) ? d * x_scale : -INFINITY;
          raise |= x[s][r] > m[r];
        }
      }
      load(kp, j0 + step, next, kv);
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int r = 0; r < kRowsM; ++r) {
          const float top = fmaxf(m[r], fmaxf(x[0][r], x[1][r]));
          const float c = exp2f(m[r] - (top == -INFINITY ? 0.f : top));
          m[r] = top, l[r] *= c;
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[r][i] *= c;
        }
      }
#pragma unroll
      for (int r = 0; r < kRowsM; ++r) {
        const float ref = m[r] == -INFINITY ? 0.f : m[r];
        const float p0 = exp2f(x[0][r] - ref), p1 = exp2f(x[1][r] - ref);
        l[r] += p0 + p1;
        // a hidden key's value may be anything: its row is skipped, not multiplied by zero
        const bool s0 = sees(0, r), s1 = sees(1, r);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float o = acc[r][i];
          if (s0) o = fmaf(p0, vv[0][i], o);
          if (s1) o = fmaf(p1, vv[1][i], o);
          acc[r][i] = o;
        }
      }
      page = next;
      load(vp, j0 + step, page, vv);
      next = page_at(j0 + 2 * step);
    }
    // join the four groups of the warp, then the warps
#pragma unroll
    for (int r = 0; r < kRowsM; ++r) {
      float top = m[r];
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
      const float c = exp2f(m[r] - (top == -INFINITY ? 0.f : top));
      float sum = l[r] * c;
      sum += __shfl_xor_sync(0xffffffffu, sum, 8);
      sum += __shfl_xor_sync(0xffffffffu, sum, 16);
      if (lane == 0) sm.ml[warp][r] = make_float2(top, sum);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float o = acc[r][i] * c;
        o += __shfl_xor_sync(0xffffffffu, o, 8);
        o += __shfl_xor_sync(0xffffffffu, o, 16);
        if (grp == 0) sm.o[warp][r][dim16(l8, i)] = o;
      }
    }
    __syncthreads();
    const Item& it = kCluster ? sm.it : walk.it;   // out of registers, which the loop over the keys has no more of
    const bool whole = it.t0 == 0 && it.t1 == it.tiles;
    const int which = it.t0 > 0 ? 0 : 1;
    const int64_t slot = ((int64_t)blockIdx.x * 2 + which) * a.slot_rows;
    auto finish = [&](int r, int d, float top, float sum, float o) {
      const int64_t at = out_row(a, it, r);
      out[at * kHeadDim + d] = sum == 0.f ? 0.f : o / sum;
      if (lse && d == 0) lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    };
    for (int e = threadIdx.x; e < rows * kHeadDim; e += kRowsThreads) {
      const int r = e / kHeadDim, d = e - r * kHeadDim;
      float top = -INFINITY;
      for (int w = 0; w < kRowsWarps; ++w) top = fmaxf(top, sm.ml[w][r].x);
      float sum = 0.f, o = 0.f;
      for (int w = 0; w < kRowsWarps; ++w) {
        const float c = exp2f(sm.ml[w][r].x - (top == -INFINITY ? 0.f : top));
        sum = fmaf(sm.ml[w][r].y, c, sum);
        o = fmaf(sm.o[w][r][d], c, o);
      }
      if (kCluster && n_cta > 1) {
        sm.cta_o[r][d] = o;
        if (d == 0) sm.cta_ml[r] = make_float2(top, sum);
      } else if (kCluster || whole) {
        finish(r, d, top, sum, o);
      } else {
        a.o[(slot + r) * kHeadDim + d] = o;
        if (d == 0) a.ml[slot + r] = make_float2(top, sum);
      }
    }
    if (kCluster) {
      if (n_cta > 1) {
        cluster_sync();
        for (int e = rank * kRowsThreads + threadIdx.x; e < rows * (kHeadDim / 2); e += n_cta * kRowsThreads) {
          const int r = e / (kHeadDim / 2), d = (e - r * (kHeadDim / 2)) * 2;
          float2 ml[8], y[8], x = make_float2(0.f, 0.f);
          float top = -INFINITY, sum = 0.f;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (k < n_cta) ml[k] = ld_peer(&sm.cta_ml[r], k), y[k] = ld_peer(&sm.cta_o[r][d], k), top = fmaxf(top, ml[k].x);
          const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (k < n_cta) {
              const float f = exp2f(ml[k].x - ref);
              sum = fmaf(ml[k].y, f, sum);
              x.x = fmaf(y[k].x, f, x.x), x.y = fmaf(y[k].y, f, x.y);
            }
          finish(r, d, top, sum, x.x);
          finish(r, d + 1, top, sum, x.y);
        }
        cluster_sync();   // nobody's memory is written again or given back while it is read
      }
      index = Walk::cluster_index(a, it), more = Walk::cluster_more(a, it) + 1;
    } else {
      if (!whole && threadIdx.x == 0) {
        int* sp = reinterpret_cast<int*>(a.split + blockIdx.x);
        sp[2 * which] = walk.pair, sp[2 * which + 1] = walk.block;
      }
      walk.next(a, sm.plan);
    }
    __syncthreads();
  }
}

// Worker w's slot 1 holds the beginning of an item that the workers after it went on with (their slots 0): the parts are
// added up in worker order.  A CTA per worker and share of the rows, a warp per row and round; no more CTAs than run at once.
constexpr int kJoinRows = 8, kJoinCtas = 16;
template <bool BF16>
__global__ void __launch_bounds__(32 * kJoinRows) join_kernel(WorkArgs a, int workers, int rows, void* __restrict__ out,
                                                              float* __restrict__ lse) {
  const int w = blockIdx.x, lane = threadIdx.x & 31, d = lane * 4;
  int r = blockIdx.y * kJoinRows + (threadIdx.x >> 5);
  pdl_wait();
  // Who has a part, the first part and the three after it (which may turn out to be none of ours, but are there to be read): where
  // blocks are small all of it is asked for at once, where they are large only what is used.
  constexpr int kBatch = 4;
  const bool early = rows <= 32;
  const int4 next = w + 1 + lane < workers ? a.split[w + 1 + lane] : make_int4(-1, -1, -1, -1);
  const int4 mine = a.split[w];
  float2 x[kBatch];
  float4 y[kBatch];
  auto fetch = [&](int p0, int last) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int part = min(p0 + b, last);
      const int64_t slot = (int64_t)(part == 0 ? w * 2 + 1 : min(w + part, workers - 1) * 2) * a.slot_rows + r;
      x[b] = a.ml[slot];
      y[b] = *reinterpret_cast<const float4*>(a.o + slot * kHeadDim + d);
    }
  };
  if (early && r < rows) fetch(0, kBatch);
  if (mine.z < 0) return;
  const Item it = make_item(a, mine.z, mine.w, 0, 1ll << 40);
  const int have = block_rows(a, it);
  unsigned no = ~__ballot_sync(0xffffffffu, next.x == mine.z && next.y == mine.w);
  int parts = no ? __ffs(no) - 1 : 32;            // workers after w that have one
  for (int w0 = w + 33; !no; w0 += 32) {
    const int4 s = w0 + lane < workers ? a.split[w0 + lane] : make_int4(-1, -1, -1, -1);
    no = ~__ballot_sync(0xffffffffu, s.x == mine.z && s.y == mine.w);
    parts += no ? __ffs(no) - 1 : 32;
  }
  bool asked = early && r < rows;
  for (; r < have; r += gridDim.y * kJoinRows, asked = false) {
    if (!asked) fetch(0, parts);
    float2 ml = make_float2(-INFINITY, 0.f);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 <= parts; p0 += kBatch) {
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        if (p0 + b > parts) break;
        const float top = fmaxf(ml.x, x[b].x), ref = top == -INFINITY ? 0.f : top;
        const float ca = exp2f(ml.x - ref), cb = exp2f(x[b].x - ref);
        ml = make_float2(top, ml.y * ca + x[b].y * cb);
        o.x = o.x * ca + y[b].x * cb, o.y = o.y * ca + y[b].y * cb, o.z = o.z * ca + y[b].z * cb, o.w = o.w * ca + y[b].w * cb;
      }
      if (p0 + kBatch <= parts) fetch(p0 + kBatch, parts);
    }
    const bool none = ml.y == 0.f;
    const float inv = none ? 0.f : 1.0f / ml.y;
    const int64_t at = out_row(a, it, r);
    if (none) o = make_float4(0.f, 0.f, 0.f, 0.f);   // a part that saw nothing may hold anything times zero
    if (BF16) {
      const __nv_bfloat162 lo = __floats2bfloat162_rn(o.x * inv, o.y * inv), hi = __floats2bfloat162_rn(o.z * inv, o.w * inv);
      const uint2 v = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(out) + at * kHeadDim + d) = v;
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(out) + at * kHeadDim + d) =
          make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    }
    if (lse && d == 0) lse[at] = none ? -INFINITY : (ml.x + log2f(ml.y)) * 0.6931471805599453f;
  }
}

int log2_of(int p) {
  int l = 0;
  while ((1 << l) < p) ++l;
  return l;
}

}  // namespace

template <bool BF16>
cudaError_t launch_join(const WorkArgs& a, int workers, int rows, void* out, float* lse, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  const int shares = (rows + kJoinRows - 1) / kJoinRows;
  cfg.gridDim = dim3(workers, shares < kJoinCtas ? shares : kJoinCtas), cfg.blockDim = dim3(32 * kJoinRows), cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, join_kernel<BF16>, a, workers, rows, out, lse);
  count_launch();
  return e;
}

template cudaError_t launch_join<true>(const WorkArgs&, int, int, void*, float*, cudaStream_t);
template cudaError_t launch_join<false>(const WorkArgs&, int, int, void*, float*, cudaStream_t);

// bf16 calls go to the kernel for few rows while every unit has at most so many query rows per KV head, else to the tensor
// cores (lengths are on the device: a cache is as short as its table is narrow).  With up to 16 rows it is ahead (one sequence on 16k rows 27 us against 33; 16 x 32k are read at the memory's rate by either), with
// 32 on a long cache its matrix instructions take longer than the bytes (8 x 8 tokens on 16k rows 159 us against 101); a
// short cache is all latency, where it stays ahead for longer (8 tokens on 1000 rows 13 us against 20).
constexpr int kFewRows = 16;
static bool wants_tc(const ckv_paged& pg) {
  const int64_t G = pg.n_q_heads / pg.n_kv_heads, most = pg.max_new > 0 ? pg.max_new : pg.n_tokens;
  return pg.dtype == CKV_BF16 && G <= 128 && most * G > kFewRows && (most * G > kMmaRows || !cluster_size(pg, kShortMore, 1));
}

// Short caches - those whose table has room for few rows; the lengths, which may be shorter, are on the device - go to clusters, one
// per block of a head's query rows: as many CTAs as the blocks leave room for, as long as each has a step's keys to read.
// Clusters do not cross the GPCs, so that of eight CTAs 15 run at a time, of four 33, of two 74 (148 SMs, one CTA each; 16 heads
// of 2000 rows in clusters of eight: 18 us, of four: 13).  0: the cache is not short: a cluster's CTA may have more rows to
// read than the split's even share and what the split's schedule and join take besides.  A table far wider than the rows held costs the
// cluster form: with room for 131072 rows one sequence of 512 takes 13.6 us on the device (7.9 with its own width), 16 of 1900 36 (27), 8
// tokens on 1000 rows 19.7 (12.8); fp32, 4 sequences of 2048 rows of two heads, 19.8 (12.9).
int cluster_size(const ckv_paged& pg, const ShortRule& rule, int64_t blocks) {
  constexpr int kFit[] = {kWorkers, 74, 33, 15};
  const int64_t items = (int64_t)pg.n_units * pg.n_kv_heads * blocks, capacity = (int64_t)pg.max_pages * pg.page_size;
  int log = 0;
  while (log < 3 && items <= kFit[log + 1] && ((int64_t)rule.cta_keys << log) < capacity) ++log;
  const int64_t rows = (items + kFit[log] - 1) / kFit[log] * capacity >> log, share = items * capacity / kWorkers;
  return rows <= share * rule.share_percent / 100 + rule.rows ? 1 << log : 0;
}

static size_t up256(size_t x) { return (x + 255) / 256 * 256; }
static PagedWs ws_of(const ckv_paged& pg, int f32_rows) {
  PagedWs w{};
  size_t o = 0;
  w.status = o, o += 256;
  const size_t rows = wants_tc(pg) ? kTcRows : (pg.dtype == CKV_BF16 ? kMmaRows : f32_rows);
  w.split = o, o = up256(o + kWorkers * sizeof(int4));
  w.ml = o, o = up256(o + kWorkers * 2 * rows * sizeof(float2));
  w.o = o, o = up256(o + kWorkers * 2 * rows * kHeadDim * sizeof(float));
  w.total = o;
  return w;
}
PagedWs paged_ws(const ckv_paged& pg) { return ws_of(pg, kRowsM); }
PagedWs tree_ws(const ckv_paged& pg) { return ws_of(pg, kTileRows); }

WorkArgs work_args(const ckv_paged& pg, const int32_t* table, const int32_t* lengths, const int32_t* starts, const uint32_t* tree,
                   int tree_words, char* ws) {
  const PagedWs w = tree ? tree_ws(pg) : paged_ws(pg);
  WorkArgs a{};
  a.Nu = pg.n_units, a.H = pg.n_q_heads, a.Hkv = pg.n_kv_heads, a.G = a.H / a.Hkv, a.T = pg.n_tokens, a.causal = tree ? 0 : pg.causal;
  a.tree = tree, a.tree_words = tree_words;
  a.P = pg.page_size, a.log_p = log2_of(pg.page_size), a.n_pages = pg.n_pages, a.max_pages = pg.max_pages;
  a.starts = starts, a.lengths = lengths, a.table = table, a.status = reinterpret_cast<int*>(ws + w.status);
  a.split = reinterpret_cast<int4*>(ws + w.split), a.ml = reinterpret_cast<float2*>(ws + w.ml), a.o = reinterpret_cast<float*>(ws + w.o);
  return a;
}

cudaError_t launch_attend(const ckv_paged& pg, const void* q, const void* k_pages, const void* v_pages, const int32_t* table,
                          const int32_t* lengths, const int32_t* starts, const uint32_t* tree, int tree_words, void* out, float* lse,
                          char* ws, cudaStream_t st) {
  const bool bf16 = pg.dtype == CKV_BF16, tc = wants_tc(pg);
  const int64_t most = most_tokens(pg);
  const float scale = attend_scale(pg);
  WorkArgs a = work_args(pg, table, lengths, starts, tree, tree_words, ws);
  if (tc) {
    a.slot_rows = kTcRows;
    return launch_attend_tc(pg, a, most, scale, q, k_pages, v_pages, out, lse, st);
  }
  if (bf16) {
    a.slot_rows = kMmaRows;
    return launch_attend_mma(pg, a, most, scale, q, k_pages, v_pages, out, lse, st);
  }
  a.slot_rows = kRowsM;
  set_blocks(a, most, kRowsM, 0, kRowsTile, 4);
  const int n_cta = cluster_size(pg, kShortRows, a.blocks);
  const int64_t items = (int64_t)a.Nu * a.Hkv * a.blocks, fit = n_cta ? 2 * kWorkers / n_cta : 0;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(n_cta ? (int)(items < fit ? items : fit) * n_cta : kWorkers), cfg.blockDim = dim3(kRowsThreads), cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0] = pdl_attribute();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = n_cta, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr, cfg.numAttrs = n_cta > 1 ? 2 : 1;
  auto kernel = tree ? (n_cta ? attend_rows_kernel<true, true> : attend_rows_kernel<false, true>)
                     : (n_cta ? attend_rows_kernel<true, false> : attend_rows_kernel<false, false>);
  cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a, pg, scale * kLog2e, (const char*)q, (const char*)k_pages, (const char*)v_pages,
                                     (float*)out, lse, n_cta);
  count_launch();
  if (e == cudaSuccess && !n_cta) e = launch_join<false>(a, kWorkers, kRowsM, out, lse, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_paged_attend(const ckv_paged& pg, const void* q, const void* k_pages, const void* v_pages,
                                const int32_t* table, const int32_t* lengths, const int32_t* starts, void* out, float* lse,
                                char* ws, cudaStream_t st) {
  return launch_attend(pg, q, k_pages, v_pages, table, lengths, starts, nullptr, 0, out, lse, ws, st);
}

}  // namespace ckv
