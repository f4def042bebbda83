// Ancestors of drafted tokens as bits, and their depths, from the trees' parents:
//   mask[t] = {t} + mask[parent t],  depth[t] = depth[parent t] + 1 (roots: 0).
// A CTA per sequence, everything in shared memory, in rounds that double what is known: after round r a token's mask has its
// 2^r nearest ancestors (itself among them) and `up` is the next one above them; or-ing in that one's mask makes it 2^(r+1).
// A chain of 512 takes nine rounds (a walk from token to token would take 512 dependent reads), a usual tree three or four.
// A mask may be or-ed in before or after its own step of the round: it then has more of the same ancestors, and the rounds end
// with all of them either way.  `up` and the depths, which add up, are double-buffered.  Parents in any order; latency all over.
#include "paged.cuh"

namespace ckv {
namespace {

// most: tokens of a unit that are handled (32 * words at most); log_w: lanes per token, a power of two of at least `words`.
__global__ void __launch_bounds__(512) tree_masks_kernel(int T, int words, int log_w, int most, const int32_t* __restrict__ parents,
                                                         const int32_t* __restrict__ starts, const int32_t* __restrict__ first_positions,
                                                         uint32_t* __restrict__ masks, int32_t* __restrict__ positions,
                                                         int* __restrict__ status) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  volatile uint32_t* mask = reinterpret_cast<uint32_t*>(smem_raw);   // [most][words]
  int2* link = reinterpret_cast<int2*>(smem_raw + ((most * words + 1) & ~1) * 4);   // [2][most]: (next ancestor or -1, depth so far)
  pdl_wait();
  pdl_launch_dependents();
  const int u = blockIdx.x;
  int first, n;
  unit_tokens(starts, u, T, first, n);
  const int m = min(n, most);
  bool bad = n > m;
  for (int e = threadIdx.x; e < m * words; e += blockDim.x) mask[e] = 0u;
  for (int t = threadIdx.x; t < m; t += blockDim.x) {
    const int p = parents[first + t];
    bad |= p < -1 || p >= n;
    const bool has = p >= 0 && p < m;
    link[t] = make_int2(has ? p : -1, has);
  }
  __syncthreads();
  for (int t = threadIdx.x; t < m; t += blockDim.x) mask[t * words + (t >> 5)] = 1u << (t & 31);
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  const int word = lane & ((1 << log_w) - 1), per = 32 >> log_w;                  // tokens a warp has at a time
  int2 *now = link, *next = link + most;
  bool above = true;
  for (int reach = 1; above && reach < 2 * m; reach *= 2) {
    if (word < words)
      for (int t = warp * per + (lane >> log_w); t < m; t += n_warps * per) {
        const int up = now[t].x;
        if (up >= 0) mask[t * words + word] = mask[t * words + word] | mask[up * words + word];
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
  for (int e = threadIdx.x; e < n * words; e += blockDim.x) masks[(int64_t)first * words + e] = e < m * words ? mask[e] : 0u;
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
  int log_w = 0;
  while ((1 << log_w) < words) ++log_w;
  const int most = T < 32 * words ? T : 32 * words;
  const size_t bytes = ((size_t)most * words + 1) / 2 * 8 + 2 * (size_t)most * sizeof(int2);
  static PerDevice ready;
  cudaError_t e = ready.once([] {
    return cudaFuncSetAttribute(tree_masks_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 32 * kMaxTreeWords * (kMaxTreeWords + 4) * 4);
  });
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(Nu), cfg.blockDim = dim3(most <= 64 ? 128 : 512), cfg.dynamicSmemBytes = bytes, cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, tree_masks_kernel, T, words, log_w, most, parents, starts, first_positions, masks, positions, status);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ckv
