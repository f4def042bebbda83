// Ancestors of drafted tokens as bits, and their depths, from the trees' parents:
//   mask[t] = {t} + mask[parent t],  depth[t] = depth[parent t] + 1 (roots: 0).
// A CTA per sequence, everything in shared memory, in rounds that double what is known: after round r a token's mask has its
// 2^r nearest ancestors (itself among them) and `up` is the next one above them; or-ing in that one's mask makes it 2^(r+1).
// A chain of 512 takes nine rounds (a walk from token to token would take 512 dependent reads), a usual tree three or four.
// A mask may be or-ed in before, after or between the words of its own step of the round: it then has more of the same ancestors,
// and the rounds end with all of them either way.  `up` and the depths, which add up, are double-buffered.  Parents in any order.
// Bound: latency.  16 trees of 63 tokens 4.1 us on the device; 64 of 512, chains for the most part, 10 (16 before a lane took four words).
#include "paged.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 512;

// most: tokens of a unit that are handled (32 * words at most); log_w: lanes per token, a power of two, four words each.  In shared
// memory a token has `quads` times four words.
__global__ void __launch_bounds__(kThreads) tree_masks_kernel(int T, int words, int quads, int log_w, int most,
                                                              const int32_t* __restrict__ parents, const int32_t* __restrict__ starts,
                                                              const int32_t* first_positions, uint32_t* __restrict__ masks, int32_t* positions,
                                                              int* status) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint4* const mask = reinterpret_cast<uint4*>(smem_raw);                // [most][quads]
  int2* const link = reinterpret_cast<int2*>(mask + most * quads);       // [2][most]: (next ancestor or -1, depth so far)
  pdl_wait();
  pdl_launch_dependents();
  const int u = blockIdx.x;
  int first, n;
  unit_tokens(starts, u, T, first, n);
  const int m = min(n, most);
  bool bad = n > m;
  for (int t = threadIdx.x; t < m; t += blockDim.x) {
    const int p = parents[first + t];
    bad |= p < -1 || p >= n;
    const bool has = p >= 0 && p < m;
    link[t] = make_int2(has ? p : -1, has);
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int quad = lane & ((1 << log_w) - 1), per = 32 >> log_w, step = (blockDim.x >> 5) * per;   // tokens a warp, and the CTA, has at a time
  const int t0 = quad < quads ? warp * per + (lane >> log_w) : m;
  for (int t = t0; t < m; t += step) {
    const uint32_t own = (t >> 7) == quad ? 1u << (t & 31) : 0u;
    const int w = t >> 5 & 3;
    mask[t * quads + quad] = make_uint4(w == 0 ? own : 0u, w == 1 ? own : 0u, w == 2 ? own : 0u, w == 3 ? own : 0u);
  }
  __syncthreads();
  int2 *now = link, *next = link + most;
  bool above = true;
  for (int reach = 1; above && reach < 2 * m; reach *= 2) {
    constexpr int U = 4;
    for (int t = t0; t < m; t += U * step) {
      uint4 x[U], y[U];
      bool has[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int mine = t + i * step, up = mine < m ? now[mine].x : -1;
        has[i] = up >= 0;
        if (has[i]) x[i] = mask[mine * quads + quad], y[i] = mask[up * quads + quad];
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (has[i]) mask[(t + i * step) * quads + quad] = make_uint4(x[i].x | y[i].x, x[i].y | y[i].y, x[i].z | y[i].z, x[i].w | y[i].w);
    }
    bool more = false;
    for (int t = threadIdx.x; t < m; t += blockDim.x) {
      const int2 a = now[t], b = a.x >= 0 ? now[a.x] : make_int2(-1, 0);
      next[t] = make_int2(b.x, a.y + b.y);
      more |= b.x >= 0;
    }
    above = __syncthreads_or(more);
    int2* const was = now;
    now = next, next = was;
  }
  const int begin = first_positions ? first_positions[u] : 0;
  const uint32_t* const flat = reinterpret_cast<const uint32_t*>(smem_raw);
  uint32_t* const out = masks + (int64_t)first * words;
  for (int t = threadIdx.x >> 2; t < n; t += blockDim.x >> 2)
    for (int w = threadIdx.x & 3; w < words; w += 4) out[t * words + w] = t < m ? flat[t * quads * 4 + w] : 0u;
  for (int t = threadIdx.x; t < n; t += blockDim.x) {
    const bool loops = t < m && now[t].x >= 0;                   // its own ancestor, or under one that is
    bad |= loops;
    if (positions) positions[first + t] = begin + (t < m && !loops ? now[t].y : 0);
  }
  if (bad) report_status(status, kStatusPage);
}

}  // namespace

cudaError_t launch_tree_masks(int Nu, int T, int words, const int32_t* parents, const int32_t* starts,
                              const int32_t* first_positions, uint32_t* masks, int32_t* positions, int* status, cudaStream_t st) {
  const int quads = (words + 3) / 4, most = T < 32 * words ? T : 32 * words;
  int log_w = 0, threads = 128;
  while ((1 << log_w) < quads) ++log_w;
  while (threads < kThreads && threads < most << log_w) threads *= 2;
  const size_t bytes = (size_t)most * (quads * sizeof(uint4) + 2 * sizeof(int2));
  static PerDevice ready;
  cudaError_t e = ready.once([] {
    return cudaFuncSetAttribute(tree_masks_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 32 * kMaxTreeWords * (kMaxTreeWords * 4 + 16));
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(Nu), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = bytes, cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, tree_masks_kernel, T, words, quads, log_w, most, parents, starts, first_positions, masks, positions, status);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ckv
