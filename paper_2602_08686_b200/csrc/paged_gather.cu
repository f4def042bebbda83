// The retained K/V rows into the pages of a cache (K~ = K[S], V~ = V[S] of Sec. 3 / Alg. 1 (D), stored row by row through
// the page table): bit copies in 16-byte pieces, consecutive threads moving consecutive pieces of one row, so that
// both sides are coalesced (a page holds whole rows of 256 or 512 bytes).  Bound: HBM; 4 rows' bytes per kept position.
#include "paged.cuh"

namespace ckv {
namespace {

__global__ void __launch_bounds__(256) gather_pages_kernel(ckv_shape s, ckv_paged pg, int rows_per_head, int vec_per_row,
                                                           const uint4* __restrict__ k, const uint4* __restrict__ v,
                                                           const int32_t* __restrict__ indices,
                                                           const int32_t* __restrict__ budgets,
                                                           const int32_t* __restrict__ offsets,
                                                           const int32_t* __restrict__ table, uint4* __restrict__ k_pages,
                                                           uint4* __restrict__ v_pages, int32_t* __restrict__ lengths,
                                                           int* __restrict__ status) {
  pdl_wait();   // indices and offsets come from the kernels before
  const int Hkv = s.n_kv_heads;
  const int64_t rows_per_unit = (int64_t)Hkv * rows_per_head;
  const int64_t total = (int64_t)s.n_units * rows_per_unit * vec_per_row;
  const int elems_per_vec = (s.dtype == CKV_BF16) ? 8 : 4;
  const int64_t first = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t e = first; e < (int64_t)s.n_units * Hkv; e += step) lengths[e] = budgets[e];
  for (int64_t i = first; i < total; i += step) {
    const int64_t row = i / vec_per_row;
    const int piece = (int)(i - row * vec_per_row);
    const int u = (int)(row / rows_per_unit);
    const int r = (int)(row - (int64_t)u * rows_per_unit);
    const int32_t* off = offsets + (int64_t)u * (Hkv + 1);
    if (r >= off[Hkv]) continue;   // an elastic selection keeps fewer rows than the unit's share
    int g = 0;
    while (g + 1 < Hkv && r >= off[g + 1]) ++g;
    const int64_t ug = (int64_t)u * Hkv + g;
    const int j = r - off[g];
    const int t = indices[row];
    const int slot = j / pg.page_size;
    const int page = j >= 0 && slot < pg.max_pages ? table[ug * pg.max_pages + slot] : -1;
    if ((unsigned)t >= (unsigned)s.seq_len || (unsigned)page >= (unsigned)pg.n_pages) {
      if (piece == 0) report_status(status, kStatusPage);
      continue;
    }
    const int64_t src =
        ((int64_t)u * s.kv_stride_unit + (int64_t)g * s.kv_stride_head + (int64_t)t * s.kv_stride_tok) / elems_per_vec +
        piece;
    const int64_t dst = ((int64_t)page * pg.page_stride + (int64_t)(j % pg.page_size) * pg.page_stride_row) / elems_per_vec + piece;
    k_pages[dst] = k[src];
    v_pages[dst] = v[src];
  }
}

}  // namespace

cudaError_t launch_gather_pages(const ckv_shape& s, const ckv_params& p, const ckv_paged& pg, const void* k, const void* v,
                                const int32_t* indices, const int32_t* budgets, const int32_t* offsets,
                                const int32_t* table, void* k_pages, void* v_pages, int32_t* lengths, int* status,
                                cudaStream_t st) {
  const int rows_per_head = p.budget_per_head < s.seq_len ? p.budget_per_head : s.seq_len;
  const int esz = s.dtype == CKV_BF16 ? 2 : 4;
  const int vec_per_row = kHeadDim * esz / 16;
  const int64_t total = (int64_t)s.n_units * s.n_kv_heads * rows_per_head * vec_per_row;
  int64_t blocks = (total + 255) / 256;
  if (blocks > 148 * 16) blocks = 148 * 16;
  if (blocks < 1) blocks = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)blocks), cfg.blockDim = dim3(256), cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, gather_pages_kernel, s, pg, rows_per_head, vec_per_row, (const uint4*)k,
                                           (const uint4*)v, indices, budgets, offsets, table, (uint4*)k_pages,
                                           (uint4*)v_pages, lengths, status);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ckv
