// Attention of few query rows (single tokens, drafted tokens) over the pages: bf16, bound by reading keys and values once.
//
// A block is 16 or 32 query rows of one (unit, KV head).  Its keys are handed out in groups of 16 to the CTA's warps, each
// of which keeps its own running maximum, sum and output; they join when the item ends.  A group never leaves its page
// (pages hold a multiple of 16 rows), so a warp looks up one page per group.  Nothing is staged in shared memory: the
// fragments of mma.m16n8k16 are loaded from global memory as they are needed, 16 bytes at a time.
//   logits  the order of the 128 dimensions in the sum is free, so thread c of a quad takes the 8 consecutive dimensions that a
//           16-byte load gives it as its share of two k-steps, for queries and keys alike;
//   output  thread (p, c) loads 8 consecutive dimensions of the keys 2c, 2c+1, 2c+8, 2c+9 and pairs them up by byte
//           permutations; which dimension a column of the output fragment means is free again.
// The matrix instructions pad 4 to 8 real rows to 16, which costs nothing: a warp spends about 150 issue slots on a group
// whose 8 KB take the SM 340 clocks to fetch.  The next keys are requested when the logits are done and the next values when
// the output is, so a warp has 4 to 8 KB under way at any time.
// 16 sequences of 32k rows, one token: 344 to 369 us by card, 0.89 to 0.95 of the measured copy rate.  With 32 query rows the 255
// registers do not hold everything: 96 bytes a thread spill in the split form, 232 in clusters.
#include <cuda_bf16.h>

#include "paged_work.cuh"

namespace ckv {
namespace {

constexpr int kMmaWarps = 8;
constexpr int kGroup = 16;          // keys per warp and step
static_assert(kMmaCtaKeys == kMmaWarps * kGroup, "keys of a step");
constexpr float kRaise = 8.0f;      // powers of two a row may exceed its reference before the output is rescaled

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 ldg16(const void* p) {
  uint4 r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int MT, int NW>
struct Smem {
  Plan plan;
  uint4 q[MT][2][4][32];                       // query fragments: [tile][rows +0 / +8][piece][lane]
  float2 ml[NW][16 * MT];
  float o[NW][16 * MT][kHeadDim + 4];
  float2 cta_ml[16 * MT];                      // the CTA's result, for the others of its cluster
  float cta_o[16 * MT][kHeadDim];
};

// kCluster: every item is one cluster's (of n_cta CTAs), whose warps share its keys and whose results join through distributed
// shared memory; no schedule, no second kernel.  Otherwise the items are split evenly over the grid.
template <int MT, int NW, bool kCluster>
__global__ void __launch_bounds__(NW * 32, 1) attend_mma_kernel(WorkArgs a, ckv_paged pg, float x_scale,
                                                                const char* __restrict__ q, const char* __restrict__ kp,
                                                                const char* __restrict__ vp, __nv_bfloat16* __restrict__ out,
                                                                float* __restrict__ lse, int n_cta) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Smem<MT, NW>& sm = *reinterpret_cast<Smem<MT, NW>*>(smem_raw);
  constexpr int kThreads = NW * 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, p = lane >> 2, c = lane & 3;
  const int64_t row_bytes = pg.page_stride_row * 2, page_bytes = pg.page_stride * 2;
  pdl_wait();
  Walk walk;
  const int rank = kCluster ? (int)blockIdx.x % n_cta : 0;
  const int stride = (kCluster ? n_cta : 1) * NW * kGroup;     // keys all warps take per step
  int early_page = 0;                                          // table entry of the warp's first group, asked for ahead of the lengths
  auto cluster_item = [&](int i, int more) {                   // the next item of this cluster that has rows
    walk.live = false;
    for (; i < a.Nu * a.Hkv * a.blocks; i += gridDim.x / n_cta, more = 0) {
      const int slot = (rank * NW + warp) * kGroup >> a.log_p;
      if (slot < a.max_pages) early_page = a.table[(int64_t)Walk::cluster_pair(a, i) * a.max_pages + slot];
      if (walk.cluster_item(a, i, more)) return;
    }
  };
  if (kCluster) {
    cluster_item(blockIdx.x / n_cta, 0);
  } else {
    make_plan<kThreads>(a, blockIdx.x, gridDim.x, sm.plan);
    pdl_launch_dependents();
    if (threadIdx.x == 0) a.split[blockIdx.x] = make_int4(-1, -1, -1, -1);
    walk.start(a, sm.plan);
  }
  while (walk.live) {
    const Item& it = walk.it;
    const int rows = block_rows(a, it);
    const int end = min(it.t1 * a.tile, it.visible), begin = it.t0 * a.tile + (rank * NW + warp) * kGroup;
    // The page of the group at key j, or -1 for none.
    auto page_at = [&](int j) { return j < end ? page_of(a, it, j >> a.log_p) : -1; };
    uint4 kr[2][4], vr[4][2];
    auto load_k = [&](int j, int page) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bool have = page >= 0 && j + t * 8 + p < end;
        const char* at = kp + page * page_bytes + ((j & (a.P - 1)) + t * 8 + p) * row_bytes + c * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) kr[t][i] = have ? ldg16(at + i * 64) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    auto load_v = [&](int j, int page) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = (e >> 1) * 8 + 2 * c + (e & 1);
        const bool have = page >= 0 && j + key < end;
        const char* at = vp + page * page_bytes + ((j & (a.P - 1)) + key) * row_bytes + p * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) vr[e][h] = have ? ldg16(at + h * 128) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    int page = kCluster && (unsigned)early_page < (unsigned)a.n_pages && begin < end ? early_page : page_at(begin);
    int next_page = page_at(begin + stride);
    load_k(begin, page);
    load_v(begin, page);
    // query fragments: the same for every warp
    for (int e = threadIdx.x; e < MT * 2 * 4 * 32; e += kThreads) {
      const int ln = e & 31, i = (e >> 5) & 3, hh = (e >> 7) & 1, mt = e >> 8, r = mt * 16 + hh * 8 + (ln >> 2);
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (r < rows) {
        const int row = it.block * a.M + r, token = row / a.G, h = it.g * a.G + (row - token * a.G);
        x = *reinterpret_cast<const uint4*>(q + ((it.first + token) * pg.q_stride_tok + h * pg.q_stride_head) * 2 + i * 64 + (ln & 3) * 16);
      }
      sm.q[mt][hh][i][ln] = x;
    }
    int limit[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int r = mt * 16 + hh * 8 + p;
        limit[mt][hh] = r < rows ? row_limit(a, it, r) : it.visible;   // rows that do not exist mask nothing
      }
    const int least = row_limit(a, it, 0);
    float o[MT][16][4], m[MT][2], l[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m[mt][0] = m[mt][1] = -INFINITY, l[mt][0] = l[mt][1] = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) o[mt][i][0] = o[mt][i][1] = o[mt][i][2] = o[mt][i][3] = 0.f;
    }
    __syncthreads();
    for (int j = begin; j < end; j += stride) {
      float s[MT][2][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int t = 0; t < 2; ++t) s[mt][t][0] = s[mt][t][1] = s[mt][t][2] = s[mt][t][3] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 q0 = sm.q[mt][0][i][lane], q1 = sm.q[mt][1][i][lane];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            mma16816(s[mt][t], q0.x, q1.x, q0.y, q1.y, kr[t][i].x, kr[t][i].y);
            mma16816(s[mt][t], q0.z, q1.z, q0.w, q1.w, kr[t][i].z, kr[t][i].w);
          }
        }
      }
      const int now_page = page;
      page = next_page, next_page = page_at(j + 2 * stride);
      load_k(j + stride, page);
      uint32_t pr[MT][4];
      const bool mask = j + kGroup > least || now_page < 0;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[mt][t][e] *= x_scale;
            if (mask && (now_page < 0 || j + t * 8 + 2 * c + (e & 1) >= limit[mt][e >> 1])) s[mt][t][e] = -INFINITY;
          }
        bool raise = false;
        float top[2];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          top[hh] = fmaxf(fmaxf(s[mt][0][2 * hh], s[mt][0][2 * hh + 1]), fmaxf(s[mt][1][2 * hh], s[mt][1][2 * hh + 1]));
          raise |= top[hh] > m[mt][hh] + kRaise;
        }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {   // the quad shares its rows' reference
            top[hh] = fmaxf(top[hh], __shfl_xor_sync(0xffffffffu, top[hh], 1));
            top[hh] = fmaxf(top[hh], __shfl_xor_sync(0xffffffffu, top[hh], 2));
            const bool up = top[hh] > m[mt][hh] + kRaise;
            const float f = up ? ex2(m[mt][hh] - top[hh]) : 1.0f;
            if (up) m[mt][hh] = top[hh];
            l[mt][hh] *= f;
#pragma unroll
            for (int i = 0; i < 16; ++i) o[mt][i][2 * hh] *= f, o[mt][i][2 * hh + 1] *= f;
          }
        }
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const float ref = m[mt][hh] == -INFINITY ? 0.f : m[mt][hh];
          float w[4];
#pragma unroll
          for (int t = 0; t < 2; ++t) w[2 * t] = ex2(s[mt][t][2 * hh] - ref), w[2 * t + 1] = ex2(s[mt][t][2 * hh + 1] - ref);
          l[mt][hh] += (w[0] + w[1]) + (w[2] + w[3]);
          pr[mt][hh] = bf16x2(w[0], w[1]), pr[mt][2 + hh] = bf16x2(w[2], w[3]);
        }
      }
      // 0 * NaN is not 0: a value row with an infinity or a NaN that some row of the block does not see yet is taken out of
      // the product and added to the rows that see it
      uint32_t odd = 0;
      if (j + kGroup > least) {
        const uint32_t x = 0x7f807f80u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t hit = 0;
#pragma unroll
          for (int h = 0; h < 2; ++h)
            hit |= __vcmpeq2(vr[e][h].x & x, x) | __vcmpeq2(vr[e][h].y & x, x) | __vcmpeq2(vr[e][h].z & x, x) | __vcmpeq2(vr[e][h].w & x, x);
          const uint32_t any = __ballot_sync(0xffffffffu, hit != 0u);   // bit (p, c): key (e >> 1) * 8 + 2 c + (e & 1)
          if (any) {
            uint32_t cols = any | (any >> 16);
            cols |= cols >> 8, cols |= cols >> 4, cols &= 15u;
            if (cols >> c & 1) vr[e][0] = vr[e][1] = make_uint4(0u, 0u, 0u, 0u);
            for (int cc = 0; cc < 4; ++cc)
              if (cols >> cc & 1) odd |= 1u << ((e >> 1) * 8 + 2 * cc + (e & 1));
          }
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          auto word = [&](const uint4& x) { return i < 2 ? x.x : (i < 4 ? x.y : (i < 6 ? x.z : x.w)); };
          const uint32_t sel = (i & 1) ? 0x7632u : 0x5410u;
          const uint32_t b0 = __byte_perm(word(vr[0][h]), word(vr[1][h]), sel), b1 = __byte_perm(word(vr[2][h]), word(vr[3][h]), sel);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) mma16816(o[mt][h * 8 + i], pr[mt][0], pr[mt][1], pr[mt][2], pr[mt][3], b0, b1);
        }
      load_v(j + stride, page);
      for (; odd; odd &= odd - 1) {
        const int key = __ffs(odd) - 1;
        const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(vp + now_page * page_bytes + ((j & (a.P - 1)) + key) * row_bytes);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            // the row's probability sits in the quad's thread (key & 7) / 2
            const uint32_t both = __shfl_sync(0xffffffffu, key < 8 ? pr[mt][hh] : pr[mt][2 + hh], (lane & 28) | ((key & 7) >> 1));
            const float w = __uint_as_float((key & 1) ? both & 0xffff0000u : both << 16);
            if (j + key < limit[mt][hh])
#pragma unroll
              for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  o[mt][i][2 * hh + e] = fmaf(w, __bfloat162float(v[(i >> 3) * 64 + (2 * c + e) * 8 + (i & 7)]), o[mt][i][2 * hh + e]);
          }
      }
    }
    // join the warps
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const int r = mt * 16 + hh * 8 + p;
        float sum = l[mt][hh];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (r < rows) {
          if (c == 0) sm.ml[warp][r] = make_float2(m[mt][hh], sum);
#pragma unroll
          for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) sm.o[warp][r][(i >> 3) * 64 + (2 * c + e) * 8 + (i & 7)] = o[mt][i][2 * hh + e];
        }
      }
    __syncthreads();
    const bool whole = it.t0 == 0 && it.t1 == it.tiles;
    const int which = it.t0 > 0 ? 0 : 1;
    const int64_t slot = ((int64_t)blockIdx.x * 2 + which) * a.slot_rows;
    auto finish = [&](int r, int d, float top, float sum, float2 x) {
      const int64_t at = out_row(a, it, r);
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      *reinterpret_cast<uint32_t*>(out + at * kHeadDim + d) = bf16x2(x.x * inv, x.y * inv);
      if (lse && d == 0) lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
    };
    for (int e = threadIdx.x; e < rows * (kHeadDim / 2); e += kThreads) {
      const int r = e / (kHeadDim / 2), d = (e - r * (kHeadDim / 2)) * 2;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) top = fmaxf(top, sm.ml[w][r].x);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
      float2 x = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float2 ml = sm.ml[w][r];
        const float f = ex2(ml.x - ref);
        const float2 y = *reinterpret_cast<const float2*>(&sm.o[w][r][d]);
        sum = fmaf(ml.y, f, sum);
        x.x = fmaf(y.x, f, x.x), x.y = fmaf(y.y, f, x.y);
      }
      if (kCluster && n_cta > 1) {
        *reinterpret_cast<float2*>(&sm.cta_o[r][d]) = x;
        if (d == 0) sm.cta_ml[r] = make_float2(top, sum);
      } else if (kCluster || whole) {
        finish(r, d, top, sum, x);
      } else {
        *reinterpret_cast<float2*>(a.o + (slot + r) * kHeadDim + d) = x;
        if (d == 0) a.ml[slot + r] = make_float2(top, sum);
      }
    }
    if (kCluster) {
      if (n_cta > 1) {
        cluster_sync();
        // the CTAs share the rows' outputs; parts are added in the order of their ranks
        for (int e = rank * kThreads + threadIdx.x; e < rows * (kHeadDim / 2); e += n_cta * kThreads) {
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
              const float f = ex2(ml[k].x - ref);
              sum = fmaf(ml[k].y, f, sum);
              x.x = fmaf(y[k].x, f, x.x), x.y = fmaf(y[k].y, f, x.y);
            }
          finish(r, d, top, sum, x);
        }
        cluster_sync();   // nobody's memory is written again or given back while it is read
      }
      cluster_item(Walk::cluster_index(a, walk.it), Walk::cluster_more(a, walk.it) + 1);
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

template <int MT, int NW, bool kCluster>
cudaError_t launch(const ckv_paged& pg, const WorkArgs& a, int grid, int n_cta, float x_scale, const void* q, const void* kp,
                   const void* vp, void* out, float* lse, cudaStream_t st) {
  auto kernel = attend_mma_kernel<MT, NW, kCluster>;
  static PerDevice ready;
  cudaError_t e = ready.once([&] {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<MT, NW>));
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid), cfg.blockDim = dim3(NW * 32), cfg.dynamicSmemBytes = sizeof(Smem<MT, NW>), cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0] = pdl_attribute();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = n_cta, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr, cfg.numAttrs = n_cta > 1 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, kernel, a, pg, x_scale, (const char*)q, (const char*)kp, (const char*)vp, (__nv_bfloat16*)out, lse, n_cta);
  count_launch();
  return e;
}

}  // namespace

cudaError_t launch_attend_mma(const ckv_paged& pg, const WorkArgs& base, int64_t most, float scale, const void* q, const void* k_pages,
                              const void* v_pages, void* out, float* lse, cudaStream_t st) {
  WorkArgs a = base;
  const bool few = most * a.G <= 16;
  set_blocks(a, most, few ? 16 : 32, 0, kMmaTile, 2);
  const float x_scale = scale * kLog2e;
  if (const int n_cta = cluster_size(pg, few ? kShortFew : kShortMore, a.blocks)) {
    const int64_t items = (int64_t)a.Nu * a.Hkv * a.blocks, fit = 2 * kWorkers / n_cta;
    const int grid = (int)(items < fit ? items : fit) * n_cta;
    return few ? launch<1, kMmaWarps, true>(pg, a, grid, n_cta, x_scale, q, k_pages, v_pages, out, lse, st)
                      : launch<2, kMmaWarps, true>(pg, a, grid, n_cta, x_scale, q, k_pages, v_pages, out, lse, st);
  }
  const cudaError_t e = few ? launch<1, kMmaWarps, false>(pg, a, kWorkers, 1, x_scale, q, k_pages, v_pages, out, lse, st)
                                   : launch<2, kMmaWarps, false>(pg, a, kWorkers, 1, x_scale, q, k_pages, v_pages, out, lse, st);
  return e != cudaSuccess ? e : launch_join<true>(a, kWorkers, a.M, out, lse, st);
}

}  // namespace ckv
