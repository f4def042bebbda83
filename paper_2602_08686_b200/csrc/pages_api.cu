// Host side of the calls on drafted trees and on the pages of a cache: argument validation and work space.
#include "paged_checks.cuh"
#include "pages.cuh"

using namespace ckv;

namespace {

// What is written is apart from what is read, and from one another.
bool all_apart(std::initializer_list<Range> written, std::initializer_list<Range> read) {
  for (const Range* w = written.begin(); w != written.end(); ++w) {
    if (!clear_of(*w, read)) return false;
    for (const Range* x = w + 1; x != written.end(); ++x)
      if (overlap(*w, *x)) return false;
  }
  return true;
}
// The cache of a call that manages pages, its units layer by layer.
ckv_status check_cache(const ckv_paged* pg, int32_t layers) {
  CKV_TRY(check_tokens(pg));
  CKV_TRY(check_pages(pg));
  return layers >= 1 && pg->n_units % layers == 0 ? CKV_OK : CKV_ERR_INVALID_ARG;
}
// A list per sequence, or per (unit, KV head).
bool lists_of(const ckv_paged& pg, int32_t layers, int32_t n_lists, Lists& lists) {
  const int seqs = pg.n_units / layers;
  lists = {n_lists != seqs, pg.n_kv_heads, seqs};
  return n_lists == seqs || n_lists == pg.n_units * pg.n_kv_heads;
}
Range refs_of(const ckv_paged& pg, const void* refs) { return ints_of(refs, pg.n_pages); }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t ckv_paged_workspace_bytes(const ckv_paged* paged) {     // enough for either attention
  if (check_tokens(paged) != CKV_OK || check_pages(paged) != CKV_OK) return 0;
  return tree_ws(*paged).total;
}

ckv_status ckv_tree_masks(int32_t n_units, int32_t n_tokens, int32_t words, const int32_t* parents, const int32_t* token_starts,
                          const int32_t* first_positions_or_null, uint32_t* masks, int32_t* positions_or_null, void* ws, size_t ws_bytes,
                          void* stream) {
  if (n_units < 1 || n_tokens < 0 || words < 1) return CKV_ERR_INVALID_ARG;
  if (n_units > 65536 || n_tokens > (1 << 20) || words > kMaxTreeWords) return CKV_ERR_UNSUPPORTED;
  CKV_TRY(check_paged_ws(kStatusBytes, ws, ws_bytes));
  if (n_tokens == 0) return CKV_OK;
  if (!good({parents, token_starts, masks}, 4)) return CKV_ERR_INVALID_ARG;
  if ((first_positions_or_null && !aligned(first_positions_or_null, 4)) || (positions_or_null && !aligned(positions_or_null, 4)))
    return CKV_ERR_INVALID_ARG;
  if (!all_apart({ints_of(masks, (int64_t)n_tokens * words), ints_of(positions_or_null, n_tokens), bytes_of(ws, kStatusBytes)},
                 {ints_of(parents, n_tokens), ints_of(token_starts, (int64_t)n_units + 1), ints_of(first_positions_or_null, n_units)}))
    return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_tree_masks(n_units, n_tokens, words, parents, token_starts, first_positions_or_null, masks, positions_or_null,
                             static_cast<int*>(ws), (cudaStream_t)stream));
  return CKV_OK;
}

ckv_status ckv_tree_attend(const ckv_paged* paged, const void* q, const void* k_pages, const void* v_pages, const int32_t* page_table,
                           const int32_t* lengths, const int32_t* token_starts, const uint32_t* masks, int32_t words, void* out,
                           float* lse_or_null, void* ws, size_t ws_bytes, void* stream) {
  CKV_TRY(check_tokens(paged));
  CKV_TRY(check_pages(paged));
  if (words < 1) return CKV_ERR_INVALID_ARG;
  if (words > (1 << 15)) return CKV_ERR_UNSUPPORTED;
  CKV_TRY(check_paged_ws(tree_ws(*paged).total, ws, ws_bytes));
  if (paged->n_tokens == 0) return CKV_OK;
  if (!good({q, k_pages, v_pages}, 16) || !good({out}, 32) || !good({page_table, lengths, token_starts, masks}, 4)) return CKV_ERR_INVALID_ARG;
  if (lse_or_null && !aligned(lse_or_null, 4)) return CKV_ERR_INVALID_ARG;
  if (!token_strides(*paged, paged->q_stride_tok, paged->q_stride_head, paged->n_q_heads)) return CKV_ERR_INVALID_ARG;
  const int64_t T = paged->n_tokens, H = paged->n_q_heads, e = esize(*paged);
  if (!all_apart({range_of(out, T, H, H * kHeadDim, kHeadDim, e), ints_of(lse_or_null, T * H), bytes_of(ws, tree_ws(*paged).total)},
                 {range_of(q, T, H, paged->q_stride_tok, paged->q_stride_head, e), pool_of(*paged, k_pages), pool_of(*paged, v_pages),
                  table_of(*paged, page_table), heads_of(*paged, lengths), starts_of(*paged, token_starts), ints_of(masks, T * words)}))
    return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_tree_attend(*paged, q, k_pages, v_pages, page_table, lengths, token_starts, masks, words, out, lse_or_null,
                              static_cast<char*>(ws), (cudaStream_t)stream));
  return CKV_OK;
}

ckv_status ckv_keep_rows(const ckv_paged* paged, int32_t layers, const int32_t* rows, int32_t n_rows, const int32_t* begins,
                         const int32_t* counts, int32_t n_lists, const int32_t* tails_or_null, const int32_t* refs_or_null,
                         const int32_t* lengths, const int32_t* page_table, void* k_pages, void* v_pages, int32_t* new_lengths,
                         void* ws, size_t ws_bytes, void* stream) {
  CKV_TRY(check_cache(paged, layers));
  Lists lists;
  if (n_rows < 0 || !lists_of(*paged, layers, n_lists, lists)) return CKV_ERR_INVALID_ARG;
  CKV_TRY(check_paged_ws(kStatusBytes, ws, ws_bytes));
  if (!good({begins, counts, lengths, page_table, new_lengths}, 4) || (n_rows > 0 && !good({rows}, 4))) return CKV_ERR_INVALID_ARG;
  if ((tails_or_null && !aligned(tails_or_null, 4)) || (refs_or_null && !aligned(refs_or_null, 4))) return CKV_ERR_INVALID_ARG;
  if (!good({k_pages, v_pages}, 16) || !pools_apart(*paged, k_pages, v_pages)) return CKV_ERR_INVALID_ARG;
  const Range work = bytes_of(ws, kStatusBytes), grown = heads_of(*paged, new_lengths);
  for (const Range& o : {pool_of(*paged, k_pages), pool_of(*paged, v_pages), grown, work})
    if (!clear_of(o, {n_rows ? ints_of(rows, n_rows) : Range{}, ints_of(begins, n_lists), ints_of(counts, n_lists), ints_of(tails_or_null, n_lists),
                      refs_of(*paged, refs_or_null), heads_of(*paged, lengths), table_of(*paged, page_table)}))
      return CKV_ERR_INVALID_ARG;
  for (const Range& o : {grown, work})
    if (!clear_of(o, {pool_of(*paged, k_pages), pool_of(*paged, v_pages)})) return CKV_ERR_INVALID_ARG;
  if (overlap(grown, work)) return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_keep_rows(*paged, lists, n_lists, rows, n_rows, begins, counts, tails_or_null, refs_or_null, lengths, page_table, k_pages,
                            v_pages, new_lengths, static_cast<int*>(ws), (cudaStream_t)stream));
  return CKV_OK;
}

size_t ckv_pages_workspace_bytes(const ckv_paged* paged) {
  if (check_cache(paged, 1) != CKV_OK) return 0;
  return reserve_ws((int64_t)paged->n_units * paged->n_kv_heads, paged->n_pages).total;
}

ckv_status ckv_pages_reserve(const ckv_paged* paged, int32_t layers, const int32_t* new_rows, int32_t n_lists, const int32_t* lengths,
                             int32_t* held, int32_t* page_table, int32_t* refs, void* k_pages, void* v_pages, int32_t* room_or_null,
                             void* ws, size_t ws_bytes, void* stream) {
  CKV_TRY(check_cache(paged, layers));
  Lists lists;
  if (!lists_of(*paged, layers, n_lists, lists)) return CKV_ERR_INVALID_ARG;
  const size_t need = ckv_pages_workspace_bytes(paged);
  CKV_TRY(check_paged_ws(need, ws, ws_bytes));
  if (!good({new_rows, lengths, held, page_table, refs}, 4) || (room_or_null && !aligned(room_or_null, 4))) return CKV_ERR_INVALID_ARG;
  if (!good({k_pages, v_pages}, 16) || !pools_apart(*paged, k_pages, v_pages)) return CKV_ERR_INVALID_ARG;
  const Range own[] = {heads_of(*paged, held), table_of(*paged, page_table), refs_of(*paged, refs), ints_of(room_or_null, 2), bytes_of(ws, need)};
  const Range read[] = {ints_of(new_rows, n_lists), heads_of(*paged, lengths)};
  if (!all_apart({own[0], own[1], own[2], own[3], own[4]}, {read[0], read[1]})) return CKV_ERR_INVALID_ARG;
  for (const Range& o : {pool_of(*paged, k_pages), pool_of(*paged, v_pages)})
    if (!clear_of(o, {own[0], own[1], own[2], own[3], own[4], read[0], read[1]})) return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_pages_reserve(*paged, lists, new_rows, lengths, held, page_table, refs, k_pages, v_pages, room_or_null,
                                static_cast<char*>(ws), (cudaStream_t)stream));
  return CKV_OK;
}

ckv_status ckv_pages_trim(const ckv_paged* paged, const int32_t* lengths_or_null, int32_t* held, const int32_t* page_table, int32_t* refs,
                          void* ws, size_t ws_bytes, void* stream) {
  CKV_TRY(check_cache(paged, 1));
  CKV_TRY(check_paged_ws(kStatusBytes, ws, ws_bytes));
  if (!good({held, page_table, refs}, 4) || (lengths_or_null && !aligned(lengths_or_null, 4))) return CKV_ERR_INVALID_ARG;
  if (!all_apart({heads_of(*paged, held), refs_of(*paged, refs), bytes_of(ws, kStatusBytes)},
                 {heads_of(*paged, lengths_or_null), table_of(*paged, page_table)}))
    return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_pages_trim(*paged, lengths_or_null, held, page_table, refs, static_cast<int*>(ws), (cudaStream_t)stream));
  return CKV_OK;
}

ckv_status ckv_pages_fork(const ckv_paged* paged, int32_t layers, int32_t n_new, const int32_t* parents, const int32_t* lengths,
                          const int32_t* held, const int32_t* page_table, int32_t* refs, int32_t keep_old, int32_t* new_lengths,
                          int32_t* new_held, int32_t* new_page_table, void* ws, size_t ws_bytes, void* stream) {
  CKV_TRY(check_cache(paged, layers));
  if (n_new < 0 || (keep_old != 0 && keep_old != 1)) return CKV_ERR_INVALID_ARG;
  const int64_t pairs = (int64_t)layers * n_new * paged->n_kv_heads;
  if (pairs > 65536) return CKV_ERR_UNSUPPORTED;
  CKV_TRY(check_paged_ws(kStatusBytes, ws, ws_bytes));
  if (!good({lengths, held, page_table, refs}, 4)) return CKV_ERR_INVALID_ARG;
  if (n_new > 0 && !good({parents, new_lengths, new_held, new_page_table}, 4)) return CKV_ERR_INVALID_ARG;
  const Range none{};
  const bool any = n_new > 0;
  if (!all_apart({any ? ints_of(new_lengths, pairs) : none, any ? ints_of(new_held, pairs) : none,
                  any ? ints_of(new_page_table, pairs * paged->max_pages) : none, refs_of(*paged, refs), bytes_of(ws, kStatusBytes)},
                 {any ? ints_of(parents, n_new) : none, heads_of(*paged, lengths), heads_of(*paged, held), table_of(*paged, page_table)}))
    return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_pages_fork(*paged, layers, n_new, parents, lengths, held, page_table, refs, keep_old, new_lengths, new_held,
                             new_page_table, static_cast<int*>(ws), (cudaStream_t)stream));
  return CKV_OK;
}

}  // extern "C"
#pragma GCC visibility pop
