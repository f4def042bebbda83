// The retained K/V rows into the pages of a cache (K~ = K[S], V~ = V[S] of Sec. 3 / Alg. 1 (D), stored row by row through
// the page table): bit copies in 16-byte pieces, consecutive threads moving consecutive pieces of one row, so that
// both sides are coalesced (a page holds whole rows of 256 or 512 bytes).  The threads of a row look its head up together
// (offsets compared side by side) and no index is divided by anything but a power of two: with 64-bit divisions per
// thread the copy was bound by instruction issue.  Bound: HBM, 4 rows' bytes per kept position; the launch and four
// dependent reads (offset, index, page, row) when small (8 layers of 512 rows: 7.2 us, from L2 5.2; one layer: 2).
#include "paged.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 256;

// kVec: 16-byte pieces, and threads, per row.  Grid: (row groups, units).
template <int kVec>
__global__ void __launch_bounds__(kThreads) gather_pages_kernel(ckv_shape s, ckv_paged pg, int log_p, int rows_per_unit,
                                                                const char* __restrict__ k, const char* __restrict__ v,
                                                                const int32_t* __restrict__ indices,
                                                                const int32_t* __restrict__ budgets,
                                                                const int32_t* __restrict__ offsets,
                                                                const int32_t* __restrict__ table, char* __restrict__ k_pages,
                                                                char* __restrict__ v_pages, int32_t* __restrict__ lengths,
                                                                int* __restrict__ status) {
  constexpr int E = kVec == 16 ? 2 : 4, kRows = kThreads / kVec;
  pdl_wait();   // indices and offsets come from the kernels before
  pdl_launch_dependents();
  const int Hkv = s.n_kv_heads, u = blockIdx.y, lane = threadIdx.x & 31, piece = threadIdx.x % kVec;
  const int32_t* off = offsets + (int64_t)u * (Hkv + 1);
  if (blockIdx.x == 0)
    for (int g = threadIdx.x; g < Hkv; g += kThreads) lengths[(int64_t)u * Hkv + g] = budgets[(int64_t)u * Hkv + g];
  const int kept = off[Hkv];   // an elastic selection keeps fewer rows than the unit's share
  const uint32_t mine = kVec == 32 ? 0xffffffffu : 0xffffu << (lane & 16);   // the row's threads in the warp
  for (int r0 = blockIdx.x * kRows; r0 < rows_per_unit; r0 += gridDim.x * kRows) {
    const int r = r0 + threadIdx.x / kVec;
    const bool live = r < rows_per_unit && r < kept;
    const int t = live ? indices[(int64_t)u * rows_per_unit + r] : 0;
    int g = 0;                 // heads that end at or before r
    for (int h = 0; h < Hkv; h += kVec)
      g += __popc(__ballot_sync(0xffffffffu, h + piece < Hkv && r >= off[min(h + piece + 1, Hkv)]) & mine);
    if (!live) continue;
    g = min(g, Hkv - 1);
    const int64_t ug = (int64_t)u * Hkv + g;
    const int j = r - off[g], slot = j >> log_p;
    const int page = j >= 0 && slot < pg.max_pages ? table[ug * pg.max_pages + slot] : -1;
    if ((unsigned)t >= (unsigned)s.seq_len || (unsigned)page >= (unsigned)pg.n_pages) {
      if (piece == 0) report_status(status, kStatusPage);
      continue;
    }
    const int64_t src = ((int64_t)u * s.kv_stride_unit + (int64_t)g * s.kv_stride_head + (int64_t)t * s.kv_stride_tok) * E + piece * 16;
    const int64_t dst = ((int64_t)page * pg.page_stride + (int64_t)(j & (pg.page_size - 1)) * pg.page_stride_row) * E + piece * 16;
    const uint4 a = *reinterpret_cast<const uint4*>(k + src), b = *reinterpret_cast<const uint4*>(v + src);
    *reinterpret_cast<uint4*>(k_pages + dst) = a;
    *reinterpret_cast<uint4*>(v_pages + dst) = b;
  }
}

}  // namespace

cudaError_t launch_gather_pages(const ckv_shape& s, const ckv_params& p, const ckv_paged& pg, const void* k, const void* v,
                                const int32_t* indices, const int32_t* budgets, const int32_t* offsets,
                                const int32_t* table, void* k_pages, void* v_pages, int32_t* lengths, int* status,
                                cudaStream_t st) {
  const int rows = s.n_kv_heads * (p.budget_per_head < s.seq_len ? p.budget_per_head : s.seq_len);
  const bool bf16 = s.dtype == CKV_BF16;
  const int per_cta = kThreads / (bf16 ? 16 : 32);
  int64_t groups = (rows + per_cta - 1) / per_cta;
  const int64_t most = (148 * 16 + s.n_units - 1) / s.n_units;   // CTAs beyond two full waves loop
  if (groups > most) groups = most;
  int log_p = 0;
  while ((1 << log_p) < pg.page_size) ++log_p;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)groups, (unsigned)s.n_units), cfg.blockDim = dim3(kThreads), cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, bf16 ? gather_pages_kernel<16> : gather_pages_kernel<32>, s, pg, log_p, rows,
                                           (const char*)k, (const char*)v, indices, budgets, offsets, table, (char*)k_pages,
                                           (char*)v_pages, lengths, status);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ckv
