// What the calls that manage the pages of a cache share: who has which list, and the work space of ckv_pages_reserve.
#pragma once
#include "paged.cuh"

namespace ckv {

constexpr int kChunkPages = 1024;    // pages of a CTA of the reserve kernels, times a factor where a pool has very many
constexpr int kMaxChunks = 4096;
constexpr int kPairBlock = 32;       // (unit, KV head) pairs whose needs are summed together

// Work space of ckv_pages_reserve (byte offsets): what its first kernel finds out, for the second.
struct ReserveWs {
  int chunk, n_chunks, n_blocks;     // pages per chunk
  size_t free_bits, shared_bits;     // uint32 [chunks * chunk / 32]: pages nobody holds, pages that several hold
  size_t chunk_free;                 // int32 [chunks]: free pages
  size_t need;                       // int2 [pairs]: pages the pairs of a block up to this one need; copies the pair needs
  size_t block_need;                 // int32 [blocks]
  size_t total;
};
inline ReserveWs reserve_ws(int64_t pairs, int64_t n_pages) {
  ReserveWs w{};
  const int64_t per = kChunkPages * ((n_pages + (int64_t)kChunkPages * kMaxChunks - 1) / ((int64_t)kChunkPages * kMaxChunks));
  w.chunk = (int)per, w.n_chunks = (int)((n_pages + per - 1) / per), w.n_blocks = (int)((pairs + kPairBlock - 1) / kPairBlock);
  size_t o = 256;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += (bytes + 255) / 256 * 256;
    return at;
  };
  w.free_bits = take((size_t)w.n_chunks * per / 8), w.shared_bits = take((size_t)w.n_chunks * per / 8);
  w.chunk_free = take((size_t)w.n_chunks * 4), w.need = take((size_t)pairs * 8), w.block_need = take((size_t)w.n_blocks * 4);
  w.total = o;
  return w;
}

// Units come layer by layer: unit = layer * sequences + sequence.  A list is a pair's (n_lists = pairs) or a sequence's.
struct Lists {
  int per_head, Hkv, seqs;
  __device__ __forceinline__ int of(int pair) const { return per_head ? pair : pair / Hkv % seqs; }
};

cudaError_t launch_keep_rows(const ckv_paged& pg, Lists lists, int n_lists, const int32_t* rows, int n_rows, const int32_t* begins,
                             const int32_t* counts, const int32_t* tails, const int32_t* refs, const int32_t* lengths,
                             const int32_t* table, void* k_pages, void* v_pages, int32_t* new_lengths, int* status, cudaStream_t st);
cudaError_t launch_pages_reserve(const ckv_paged& pg, Lists lists, const int32_t* new_rows, const int32_t* lengths, int32_t* held,
                                 int32_t* table, int32_t* refs, void* k_pages, void* v_pages, int32_t* room, char* ws,
                                 cudaStream_t st);
cudaError_t launch_pages_trim(const ckv_paged& pg, const int32_t* lengths, int32_t* held, const int32_t* table, int32_t* refs,
                              int* status, cudaStream_t st);
cudaError_t launch_pages_fork(const ckv_paged& pg, int layers, int new_seqs, const int32_t* parents, const int32_t* lengths,
                              const int32_t* held, const int32_t* table, int32_t* refs, int keep_old, int32_t* new_lengths,
                              int32_t* new_held, int32_t* new_table, int* status, cudaStream_t st);

}  // namespace ckv
