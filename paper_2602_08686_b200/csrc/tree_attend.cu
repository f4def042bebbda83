// Attention of drafted trees: the choice of kernels, and the one for fp32.
//
// bf16 goes to the kernels of the attention over pages (few rows: mma.sync, more: tcgen05), whose masks look at the tokens' bits
// behind the rows that all tokens see.  So does fp32 where a head's query rows are at most the four of its block.  A tree has more: with 24
// tokens and four heads a group 24 blocks of four rows would read the same keys and values (70 us for 4 sequences of 2048 rows, all of
// it waiting for L2).
//
// attend_split_kernel: fp32 on the tensor cores, blocks of 16 RG query rows.  An fp32 number is the sum of two of tf32's 11 bits, x = h + l
// with h = x rounded and l what is left, of which the unit takes the first 11 bits (off by 2^-21 |x| at most); a product is
//   x y = hx hy + hx ly + lx hy,   lx ly <= 2^-22 |x y| left out,
// three of the unit's for one.  It cuts sums off instead of rounding them (1 + 0.75 ulp gives 1), a bias for each addition, so nothing
// long is summed there: logits run in four chains of four steps and the rest in four more, and what eight keys give the output starts from
// zero and is added to it by the CUDA cores.  Outputs are off by 3 to 4.5e-7 of their 2-norm on 300 to 32000 rows (elementary
// operations in fp32: 6e-7 to 2.4e-6).
// Keys and values come to shared memory in tiles of 64 rows, three deep, by asynchronous copies that fill in zeros for rows that
// are not there.  A warp has 16 of the block's rows, whose queries and output stay in its registers, and every KG-th eight keys of a tile
// (KG = 8 / RG); fragments of m16n8k8 come straight from the tile, 16 bytes at a time:
//   logits  the order of the 128 dimensions is free: thread c of a quad has dimensions 16 i + 4 c .. + 3 of queries and keys;
//   output  thread c's probabilities are those of keys c and c + 4 of eight (column n of the logits is key n / 2 + 4 (n % 2)), as the
//           second product wants them; which dimension a column of the output means is free again.
// Rows of 528 bytes put all of a quarter-warp's pieces in banks of their own.
// Bound: in the limit the matrix instructions (8 clocks each on one of an SM's four units, 48 a key and 32 rows), so far the latency of a
// step's chain of dependent instructions at two warps a unit (255 registers a thread): 8 sequences of 32 tokens on 4000 rows, four heads
// a group, 480 to 490 us (130 clocks a key and 32 rows; blocks of four rows 1300, the same tiles on the FMA units 520 to 650, whose
// operands come from shared memory at 128 bytes a clock); 4 of 24 tokens on 2000 rows, two KV heads, 43 (68).  Not kept: 16 keys a step
// with two chains (445, errors half as large again), 12 warps with split queries in shared memory (426, and 31 instead of 25 us for 4 of
// 8 tokens on 2000 rows).
#include <cfloat>

#include "paged_work.cuh"
#include "tc_ptx.cuh"

namespace ckv {
namespace {

using namespace ptx;

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kKeys = 64, kStages = 3;
constexpr int kRow = kHeadDim + 4;               // floats from one row to the next
constexpr float kRaise = 8.0f;                   // powers of two a row may exceed its reference before the output is rescaled

struct SplitSmem {
  float kv[kStages][2][kKeys][kRow];             // keys, values
  uint8_t there[kStages][kKeys];                 // whether the row is in the item's range and has a page
  float2 ml[kWarps][16];
  Plan plan;
};

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool have) {   // zeros where there is nothing to read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(have ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void mma1688(float (&d)[4], const float (&a)[4], float b0, float b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(__float_as_uint(a[0])), "r"(__float_as_uint(a[1])), "r"(__float_as_uint(a[2])), "r"(__float_as_uint(a[3])),
                 "r"(__float_as_uint(b0)), "r"(__float_as_uint(b1)));
}
// x rounded to tf32's 11 bits (the unit would cut it off).  cvt.rna.tf32 takes several instructions.
__device__ __forceinline__ float high(float x) { return __uint_as_float((__float_as_uint(x) + 0x1000u) & 0xffffe000u); }
__device__ __forceinline__ void here(float4& x) { asm volatile("" : "+f"(x.x), "+f"(x.y), "+f"(x.z), "+f"(x.w)); }
__device__ __forceinline__ float part(const float4& x, int i) { return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w; }

__device__ __noinline__ float plain_logit(const char* q, const float* k) {
  float d = 0.f;
  for (int i = 0; i < kHeadDim; ++i) d = fmaf(reinterpret_cast<const float*>(q)[i], k[i], d);
  return d;
}

template <int RG>
__global__ void __launch_bounds__(kThreads, 1) attend_split_kernel(WorkArgs a, ckv_paged pg, float x_scale, const char* __restrict__ q,
                                                                   const char* __restrict__ kp, const char* __restrict__ vp,
                                                                   float* __restrict__ out, float* __restrict__ lse) {
  constexpr int KG = kWarps / RG;
  constexpr int64_t E = 4;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  SplitSmem& sm = *reinterpret_cast<SplitSmem*>(smem_raw);
  static_assert(sizeof(SplitSmem) <= 232448, "shared memory of one CTA");
  static_assert(kWarps * 16 <= 2 * kKeys, "the warps' results fit a stage, once the tiles are done");
  float(*const results)[16][kHeadDim] = reinterpret_cast<float(*)[16][kHeadDim]>(&sm.kv[0][0][0][0]);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rg = warp % RG, kg = warp / RG, g = lane >> 2, c = lane & 3;
  pdl_wait();
  Walk walk;
  make_plan<kThreads>(a, blockIdx.x, gridDim.x, sm.plan);
  pdl_launch_dependents();
  if (threadIdx.x == 0) a.split[blockIdx.x] = make_int4(-1, -1, -1, -1);
  walk.start(a, sm.plan);
  while (walk.live) {
    const Item& it = walk.it;
    const int rows = block_rows(a, it), end = min(it.t1 * kKeys, it.visible), begin = it.t0 * kKeys;
    const int tiles = end > begin ? (end - begin + kKeys - 1) / kKeys : 0;
    // A warp copies sixteen of a tile's 128 rows, a lane 16 bytes of each; their pages are looked up side by side.
    auto load = [&](int n) {
      if (n < tiles) {
        const int j0 = begin + n * kKeys, mine = j0 + ((warp + kWarps * lane) & (kKeys - 1));
        const int page = lane < kKeys / kWarps && mine < end ? page_of(a, it, mine >> a.log_p) : -1;
        if (lane < kKeys / kWarps) sm.there[n % kStages][warp + kWarps * lane] = page >= 0;
        const uint32_t dst = smem_u32(&sm.kv[n % kStages][0][warp][lane * 4]);
#pragma unroll
        for (int i = 0; i < kKeys / kWarps; ++i) {
          const int from = __shfl_sync(0xffffffffu, page, i);
          const int64_t at = (from < 0 ? 0 : from * pg.page_stride + ((j0 + warp + kWarps * i) & (a.P - 1)) * pg.page_stride_row) * E + lane * 16;
          copy16(dst + i * kWarps * kRow * 4, kp + at, from >= 0);
          copy16(dst + (kKeys + i * kWarps) * kRow * 4, vp + at, from >= 0);
        }
      }
      copies_end();
    };
    load(0);
    load(1);
    // the thread's two rows, g and g + 8 of the warp's
    float4 qr[2][8];
    const uint32_t* words[2];
    const char* q_at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = rg * 16 + h * 8 + g;
      words[h] = nullptr, q_at[h] = q;
      if (r < rows) {
        const int row = it.block * a.M + r, token = row / a.G, head = it.g * a.G + (row - token * a.G);
        q_at[h] = q + ((it.first + token) * pg.q_stride_tok + head * pg.q_stride_head) * E;
        words[h] = tree_words_of(a, it, token);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        qr[h][i] = r < rows ? *reinterpret_cast<const float4*>(q_at[h] + i * 64 + c * 16) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const int least = rows_before_tree(it), base = it.len - it.n;
    float o[16][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    for (int n = 0; n < tiles; ++n) {
      copies_wait<1>();
      __syncthreads();
      load(n + 2);
      const int j0 = begin + n * kKeys;
#pragma unroll 1
      for (int s = kg * 8; s < kKeys && j0 + s < end && rg * 16 < rows; s += KG * 8) {
        const float(*const keys)[kRow] = &sm.kv[n % kStages][0][s];
        const float(*const values)[kRow] = &sm.kv[n % kStages][1][s];
        // Split queries would not fit the registers: they are split here, and not ahead of the loop.
#pragma unroll
        for (int i = 0; i < 8; ++i) here(qr[0][i]), here(qr[1][i]);
        float chain[4][4], rest[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) chain[i][e] = rest[i][e] = 0.f;
        const float* const key = keys[(g >> 1) + 4 * (g & 1)] + c * 4;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float4 k = *reinterpret_cast<const float4*>(key + i * 16);
#pragma unroll
          for (int t = 0; t < 4; t += 2) {
            const float x[4] = {part(qr[0][i], t), part(qr[1][i], t), part(qr[0][i], t + 1), part(qr[1][i], t + 1)};
            const float k0 = part(k, t), k1 = part(k, t + 1), h0 = high(k0), h1 = high(k1);
            float hx[4], lx[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) hx[e] = high(x[e]), lx[e] = x[e] - hx[e];
            mma1688(rest[t], lx, h0, h1);
            mma1688(rest[t + 1], hx, k0 - h0, k1 - h1);
            mma1688(chain[(2 * i + t / 2) & 3], hx, h0, h1);
          }
        }
        float x[4];        // row g: keys c, c + 4; row g + 8: the same
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = ((chain[0][e] + chain[1][e]) + (chain[2][e] + chain[3][e])) + ((rest[0][e] + rest[1][e]) + (rest[2][e] + rest[3][e]));
        // An infinity splits into one and a NaN: where there is a NaN the logit is taken from the numbers themselves.
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= x[e] != x[e];
        if (__any_sync(0xffffffffu, odd)) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = words[e >> 1] ? plain_logit(q_at[e >> 1], keys[c + 4 * (e & 1)]) : 0.f;
        }
        const bool tree = j0 + s + 8 > least;      // some of the keys are hidden from some rows
        uint32_t see[2] = {0xffu, 0xffu};
        if (tree) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (words[h]) see[h] = tree_bits(words[h], a.tree_words, j0 + s - base);
        }
        bool raise = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int at = c + 4 * (e & 1);
          const bool sees = sm.there[n % kStages][s + at] && (!tree || (see[e >> 1] >> at & 1u));
          x[e] = sees ? x[e] * x_scale : -INFINITY;
          raise |= x[e] > m[e >> 1] + kRaise;
        }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {            // the quad shares its rows' reference
            float top = fmaxf(x[2 * h], x[2 * h + 1]);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const bool up = top > m[h] + kRaise;
            const float f = up ? exp2f(m[h] - top) : 1.0f;
            if (up) m[h] = top;
            l[h] *= f;
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i][2 * h] *= f, o[i][2 * h + 1] *= f;
          }
        }
        float p[4], hp[4], lp[4];                  // as the second product's fragment: rows g, g + 8 of key c, then of key c + 4
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int h = e & 1;
          p[e] = exp2f(x[2 * h + (e >> 1)] - (m[h] == -INFINITY ? 0.f : m[h]));
          l[h] += p[e];
          hp[e] = high(p[e]), lp[e] = p[e] - hp[e];
        }
        // output.  0 * NaN is not 0, and an infinity splits into one and a NaN, the largest finite numbers (whose first part is rounded up)
        // into two infinities: values whose parts are not finite are left out of the products and added, element by element, to the
        // rows that see them.
        const int piece = ((g >> 1) + 4 * (g & 1)) * 4;
#pragma unroll
        for (int b = 0; b < 4; ++b) {              // 32 dimensions at a time
          float4 v0 = *reinterpret_cast<const float4*>(&values[c][b * 32 + piece]), v1 = *reinterpret_cast<const float4*>(&values[c + 4][b * 32 + piece]);
          float l0[4], l1[4], sum = 0.f;
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            l0[t] = part(v0, t) - high(part(v0, t)), l1[t] = part(v1, t) - high(part(v1, t));
            sum += l0[t] + l1[t];
          }
          if (__any_sync(0xffffffffu, !(fabsf(sum) <= FLT_MAX))) {
            uint32_t mine = 0;                     // bit (t, key): element t of the thread's four
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              if (!(fabsf(l0[t]) <= FLT_MAX)) mine |= 1u << (2 * t), l0[t] = 0.f, (t == 0 ? v0.x : t == 1 ? v0.y : t == 2 ? v0.z : v0.w) = 0.f;
              if (!(fabsf(l1[t]) <= FLT_MAX)) mine |= 2u << (2 * t), l1[t] = 0.f, (t == 0 ? v1.x : t == 1 ? v1.y : t == 2 ? v1.z : v1.w) = 0.f;
            }
#pragma unroll 1
            for (uint32_t lanes = __ballot_sync(0xffffffffu, mine != 0u); lanes; lanes &= lanes - 1) {
              const int from = __ffs(lanes) - 1, gf = from >> 2, cf = from & 3;
              uint32_t what = __shfl_sync(0xffffffffu, mine, from);
              for (; what; what &= what - 1) {
                const int bit = __ffs(what) - 1, t = bit >> 1, at = cf + 4 * (bit & 1);
                const float v = values[at][b * 32 + ((gf >> 1) + 4 * (gf & 1)) * 4 + t];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  // the row's probability sits in the quad's thread cf
                  const float w0 = __shfl_sync(0xffffffffu, p[h], (lane & 28) | cf), w1 = __shfl_sync(0xffffffffu, p[2 + h], (lane & 28) | cf);
                  const bool sees = sm.there[n % kStages][s + at] && words[h] && (!tree || (see[h] >> at & 1u));
                  const float w = (bit & 1) ? w1 : w0;
                  // the element is column gf of tile 4 b + t
                  if (sees && (gf >> 1) == c) {
#pragma unroll
                    for (int y = 0; y < 4; ++y)
#pragma unroll
                      for (int z = 0; z < 2; ++z)
                        if (y == t && z == (gf & 1)) o[4 * b + y][2 * h + z] = fmaf(w, v, o[4 * b + y][2 * h + z]);
                  }
                }
              }
            }
          }
          float d[4][4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0.f;
            mma1688(d[t], lp, high(part(v0, t)), high(part(v1, t)));
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) mma1688(d[t], hp, l0[t], l1[t]);
#pragma unroll
          for (int t = 0; t < 4; ++t) mma1688(d[t], hp, high(part(v0, t)), high(part(v1, t)));
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[4 * b + t][e] += d[t][e];
        }
      }
    }
    copies_wait<0>();
    __syncthreads();
    // join the warps that share the rows
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float sum = l[h];
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (c == 0) sm.ml[warp][h * 8 + g] = make_float2(m[h], sum);
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<float4*>(&results[warp][h * 8 + g][b * 32 + e * 16 + c * 4]) =
              make_float4(o[4 * b][2 * h + e], o[4 * b + 1][2 * h + e], o[4 * b + 2][2 * h + e], o[4 * b + 3][2 * h + e]);
    }
    __syncthreads();
    const bool whole = it.t0 == 0 && it.t1 == it.tiles;
    const int which = it.t0 > 0 ? 0 : 1;
    const int64_t slot = ((int64_t)blockIdx.x * 2 + which) * a.slot_rows;
    for (int e = threadIdx.x; e < rows * (kHeadDim / 2); e += kThreads) {
      const int r = e / (kHeadDim / 2), d = (e - r * (kHeadDim / 2)) * 2, w0 = r / 16, i = r % 16;
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int k = 0; k < KG; ++k) top = fmaxf(top, sm.ml[w0 + k * RG][i].x);
      const float ref = top == -INFINITY ? 0.f : top;
      float2 x = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < KG; ++k) {
        const float2 ml = sm.ml[w0 + k * RG][i], y = *reinterpret_cast<const float2*>(&results[w0 + k * RG][i][d]);
        const float f = exp2f(ml.x - ref);
        sum = fmaf(ml.y, f, sum);
        x.x = fmaf(y.x, f, x.x), x.y = fmaf(y.y, f, x.y);
      }
      if (whole) {
        const int64_t at = out_row(a, it, r);
        *reinterpret_cast<float2*>(out + at * kHeadDim + d) = sum == 0.f ? make_float2(0.f, 0.f) : make_float2(x.x / sum, x.y / sum);
        if (lse && d == 0) lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
      } else {
        *reinterpret_cast<float2*>(a.o + (slot + r) * kHeadDim + d) = x;
        if (d == 0) a.ml[slot + r] = make_float2(top, sum);
      }
    }
    if (!whole && threadIdx.x == 0) {
      int* sp = reinterpret_cast<int*>(a.split + blockIdx.x);
      sp[2 * which] = walk.pair, sp[2 * which + 1] = walk.block;
    }
    walk.next(a, sm.plan);
    __syncthreads();
  }
}

template <int RG>
cudaError_t launch_split(const ckv_paged& pg, WorkArgs a, int64_t most, const void* q, const void* kp, const void* vp, void* out, float* lse,
                         cudaStream_t st) {
  auto kernel = attend_split_kernel<RG>;
  constexpr size_t bytes = sizeof(SplitSmem);
  static PerDevice ready;
  cudaError_t e = ready.once([&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); });
  if (e != cudaSuccess) return e;
  a.slot_rows = kTileRows;
  set_blocks(a, most, 16 * RG, 0, kKeys, 2);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(kWorkers), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = bytes, cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kernel, a, pg, attend_scale(pg) * kLog2e, (const char*)q, (const char*)kp, (const char*)vp, (float*)out, lse);
  count_launch();
  return e != cudaSuccess ? e : launch_join<false>(a, kWorkers, a.M, out, lse, st);
}

// fp32 stays with the blocks of four rows where there are few of them (16 rows: 4 sequences of 2000 rows 20 us, 21 here), or of which an
// SM has few cache rows to read (32 rows on 300: 12 us, 14 here; on 2000, in four sequences, 29 and 25).
bool wants_split(const ckv_paged& pg, int64_t rows) {
  const int64_t capacity = (int64_t)pg.max_pages * pg.page_size, blocks = (int64_t)pg.n_units * pg.n_kv_heads * ((rows + 3) / 4);
  return pg.dtype == CKV_F32 && rows > 16 && blocks * capacity > 500 * kWorkers;
}

}  // namespace

cudaError_t launch_tree_attend(const ckv_paged& pg, const void* q, const void* k_pages, const void* v_pages,
                               const int32_t* table, const int32_t* lengths, const int32_t* starts, const uint32_t* tree,
                               int tree_words, void* out, float* lse, char* ws, cudaStream_t st) {
  const int64_t most = most_tokens(pg), rows = most * (pg.n_q_heads / pg.n_kv_heads);
  if (!wants_split(pg, rows)) return launch_attend(pg, q, k_pages, v_pages, table, lengths, starts, tree, tree_words, out, lse, ws, st);
  const WorkArgs a = work_args(pg, table, lengths, starts, tree, tree_words, ws);
  // a block of 64 rows takes as long as 1.75 of 32
  const bool large = 7 * ((rows + 63) / 64) < 4 * ((rows + 31) / 32);
  const cudaError_t e = large ? launch_split<4>(pg, a, most, q, k_pages, v_pages, out, lse, st)
                              : launch_split<2>(pg, a, most, q, k_pages, v_pages, out, lse, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ckv
