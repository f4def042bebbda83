// Host side of the paged-cache entry points: argument validation and work space.
#include "paged_checks.cuh"

using namespace ckv;

#pragma GCC visibility push(default)
extern "C" {

ckv_status ckv_rotate(const ckv_paged* paged, const ckv_rotary* rotary, const void* q, const void* k,
                      const int32_t* positions, const int32_t* token_starts, void* q_out, void* k_out, void* stream) {
  CKV_TRY(check_tokens(paged));
  if (!rotary) return CKV_ERR_INVALID_ARG;
  CKV_TRY(check_rotary(rotary));
  if (paged->n_tokens == 0) return CKV_OK;
  if (!q && !k) return CKV_ERR_INVALID_ARG;
  if (!good({positions, token_starts}, 4)) return CKV_ERR_INVALID_ARG;
  const int H = paged->n_q_heads, Hkv = paged->n_kv_heads;
  if (q && (!aligned(q, 16) || !token_strides(*paged, paged->q_stride_tok, paged->q_stride_head, H))) return CKV_ERR_INVALID_ARG;
  if (k && (!aligned(k, 16) || !token_strides(*paged, paged->kv_stride_tok, paged->kv_stride_head, Hkv)))
    return CKV_ERR_INVALID_ARG;
  const int64_t T = paged->n_tokens, e = esize(*paged);
  const Range qr = range_of(q, T, H, paged->q_stride_tok, paged->q_stride_head, e), kr = range_of(k, T, Hkv, paged->kv_stride_tok, paged->kv_stride_head, e);
  if ((q && !good({q_out}, 16)) || (k && !good({k_out}, 16))) return CKV_ERR_INVALID_ARG;
  const Rows q_rows{q, T, paged->q_stride_tok, H, paged->q_stride_head, e}, k_rows{k, T, paged->kv_stride_tok, Hkv, paged->kv_stride_head, e};
  const bool q_here = q && q_out == q, k_here = k && k_out == k;
  if ((q_here && !in_place_ok(q_rows, {k_rows})) || (k_here && !in_place_ok(k_rows, {q_rows}))) return CKV_ERR_INVALID_ARG;
  const Range qo = q ? out_range(*paged, q_out, q, qr, H) : Range{}, ko = k ? out_range(*paged, k_out, k, kr, Hkv) : Range{};
  if ((!q_here && !clear_of(qo, {qr, kr, ko})) || (!k_here && !clear_of(ko, {qr, kr, qo}))) return CKV_ERR_INVALID_ARG;
  for (const Range& o : {qo, ko})
    if (!clear_of(o, {ints_of(positions, T), starts_of(*paged, token_starts), freq_of(rotary), q_norm_of(rotary), k_norm_of(rotary)}))
      return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_rotate(*paged, rotary, q, k, nullptr, positions, token_starts, q_out, k_out, nullptr, nullptr, nullptr,
                         nullptr, nullptr, nullptr, (cudaStream_t)stream));
  return CKV_OK;
}

ckv_status ckv_append(const ckv_paged* paged, const ckv_rotary* rotary, const void* q_or_null, const void* k,
                      const void* v, const int32_t* positions, const int32_t* token_starts, const int32_t* lengths,
                      const int32_t* page_table, void* q_out, void* k_pages, void* v_pages,
                      int32_t* new_lengths_or_null, void* ws, size_t ws_bytes, void* stream) {
  CKV_TRY(check_tokens(paged));
  CKV_TRY(check_pages(paged));
  if (rotary) CKV_TRY(check_rotary(rotary));
  if (!good({token_starts, lengths, page_table}, 4)) return CKV_ERR_INVALID_ARG;
  if (new_lengths_or_null && !aligned(new_lengths_or_null, 4)) return CKV_ERR_INVALID_ARG;
  CKV_TRY(check_paged_ws(kStatusBytes, ws, ws_bytes));
  if (paged->n_tokens == 0 && !new_lengths_or_null) return CKV_OK;
  const bool any = paged->n_tokens > 0;
  const Range st = starts_of(*paged, token_starts), len = heads_of(*paged, lengths), tab = table_of(*paged, page_table);
  const Range grown = heads_of(*paged, new_lengths_or_null), work = bytes_of(ws, kStatusBytes);
  if (!clear_of(grown, {st, len, tab, work}) || !clear_of(work, {st, len, tab})) return CKV_ERR_INVALID_ARG;
  if (any) {
    const int H = paged->n_q_heads, Hkv = paged->n_kv_heads;
    if (!good({k, v, k_pages, v_pages}, 16) || !pools_apart(*paged, k_pages, v_pages)) return CKV_ERR_INVALID_ARG;
    const bool turns = rotary && rotary->rot_dim;
    if (turns && !good({positions}, 4)) return CKV_ERR_INVALID_ARG;
    if (!token_strides(*paged, paged->kv_stride_tok, paged->kv_stride_head, Hkv)) return CKV_ERR_INVALID_ARG;
    const int64_t T = paged->n_tokens, e = esize(*paged);
    const Rows k_rows{k, T, paged->kv_stride_tok, Hkv, paged->kv_stride_head, e}, v_rows{v, T, paged->kv_stride_tok, Hkv, paged->kv_stride_head, e};
    const Rows q_rows{q_or_null, T, paged->q_stride_tok, H, paged->q_stride_head, e};
    const Range kr = k_rows.range(), vr = v_rows.range(), qr = q_rows.range();
    const bool q_here = q_or_null && q_out == q_or_null;
    if (q_or_null) {
      if (!aligned(q_or_null, 16) || !good({q_out}, 16) || !token_strides(*paged, paged->q_stride_tok, paged->q_stride_head, H))
        return CKV_ERR_INVALID_ARG;
      if (q_here && !in_place_ok(q_rows, {k_rows, v_rows})) return CKV_ERR_INVALID_ARG;
    }
    const Range qo = q_or_null ? out_range(*paged, q_out, q_or_null, qr, H) : Range{};
    if (!q_here && !clear_of(qo, {qr, kr, vr})) return CKV_ERR_INVALID_ARG;
    const Range pos = turns ? ints_of(positions, T) : Range{}, freq = freq_of(rotary), qn = q_norm_of(rotary), kn = k_norm_of(rotary);
    for (const Range& o : {pool_of(*paged, k_pages), pool_of(*paged, v_pages)})
      if (!clear_of(o, {qr, kr, vr, qo})) return CKV_ERR_INVALID_ARG;
    for (const Range& o : {pool_of(*paged, k_pages), pool_of(*paged, v_pages), qo})
      if (!clear_of(o, {pos, freq, qn, kn, st, len, tab, grown, work})) return CKV_ERR_INVALID_ARG;
    for (const Range& o : {grown, work})
      if (!clear_of(o, {qr, kr, vr, pos, freq, qn, kn})) return CKV_ERR_INVALID_ARG;
  }
  CKV_CUDA(launch_rotate(*paged, rotary, any ? q_or_null : nullptr, any ? k : nullptr, any ? v : nullptr, positions,
                         token_starts, q_out, nullptr, lengths, page_table, k_pages, v_pages, new_lengths_or_null,
                         reinterpret_cast<int*>(static_cast<char*>(ws) + paged_ws(*paged).status), (cudaStream_t)stream));
  return CKV_OK;
}

ckv_status ckv_gather_pages(const ckv_shape* shape, const ckv_params* params, const ckv_paged* paged, const void* k,
                            const void* v, const int32_t* indices, const int32_t* budgets, const int32_t* offsets,
                            const int32_t* page_table, void* k_pages, void* v_pages, int32_t* lengths, void* ws,
                            size_t ws_bytes, void* stream) {
  if (ckv_workspace_bytes(shape, params) == 0) return CKV_ERR_INVALID_ARG;   // shape and params as everywhere else
  CKV_TRY(check_tokens(paged));
  CKV_TRY(check_pages(paged));
  if (shape->n_units != paged->n_units || shape->n_kv_heads != paged->n_kv_heads || shape->dtype != paged->dtype)
    return CKV_ERR_INVALID_ARG;
  if (!good({k, v, k_pages, v_pages}, 16) || !pools_apart(*paged, k_pages, v_pages)) return CKV_ERR_INVALID_ARG;
  if (!good({indices, budgets, offsets, page_table, lengths}, 4)) return CKV_ERR_INVALID_ARG;
  CKV_TRY(check_paged_ws(kStatusBytes, ws, ws_bytes));
  const int64_t kept = (int64_t)shape->n_units * shape->n_kv_heads * (params->budget_per_head < shape->seq_len ? params->budget_per_head : shape->seq_len);
  auto dense_kv = [&](const void* x) {   // [Nu, Hkv, L, d]: the last unit's rows end it
    Range r = range_of(x, shape->n_kv_heads, shape->seq_len, shape->kv_stride_head, shape->kv_stride_tok, esize(*paged));
    const __int128 hi = (__int128)r.hi + (__int128)(shape->n_units - 1) * shape->kv_stride_unit * esize(*paged);
    r.hi = hi < (__int128)UINTPTR_MAX ? (uintptr_t)hi : UINTPTR_MAX;
    return r;
  };
  const Range kr = dense_kv(k), vr = dense_kv(v), ind = ints_of(indices, kept), bud = heads_of(*paged, budgets);
  const Range off = ints_of(offsets, (int64_t)shape->n_units * (shape->n_kv_heads + 1)), tab = table_of(*paged, page_table);
  const Range len = heads_of(*paged, lengths), work = bytes_of(ws, kStatusBytes);
  for (const Range& o : {pool_of(*paged, k_pages), pool_of(*paged, v_pages), len, work})
    if (!clear_of(o, {kr, vr, ind, bud, off, tab})) return CKV_ERR_INVALID_ARG;
  for (const Range& o : {pool_of(*paged, k_pages), pool_of(*paged, v_pages)})
    if (!clear_of(o, {len, work})) return CKV_ERR_INVALID_ARG;
  if (overlap(len, work)) return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_gather_pages(*shape, *params, *paged, k, v, indices, budgets, offsets, page_table, k_pages, v_pages, lengths,
                               reinterpret_cast<int*>(static_cast<char*>(ws) + paged_ws(*paged).status),
                               (cudaStream_t)stream));
  return CKV_OK;
}

ckv_status ckv_paged_attend(const ckv_paged* paged, const void* q, const void* k_pages, const void* v_pages,
                            const int32_t* page_table, const int32_t* lengths, const int32_t* token_starts, void* out,
                            float* lse_or_null, void* ws, size_t ws_bytes, void* stream) {
  CKV_TRY(check_tokens(paged));
  CKV_TRY(check_pages(paged));
  CKV_TRY(check_paged_ws(paged_ws(*paged).total, ws, ws_bytes));
  if (paged->n_tokens == 0) return CKV_OK;
  if (!good({q, k_pages, v_pages}, 16) || !good({out}, 32) || !good({page_table, lengths, token_starts}, 4)) return CKV_ERR_INVALID_ARG;
  if (lse_or_null && !aligned(lse_or_null, 4)) return CKV_ERR_INVALID_ARG;
  if (!token_strides(*paged, paged->q_stride_tok, paged->q_stride_head, paged->n_q_heads)) return CKV_ERR_INVALID_ARG;
  const int64_t T = paged->n_tokens, H = paged->n_q_heads, e = esize(*paged);
  const Range o = range_of(out, T, H, H * kHeadDim, kHeadDim, e), l = ints_of(lse_or_null, T * H), work = bytes_of(ws, paged_ws(*paged).total);
  for (const Range& x : {o, l, work})
    if (!clear_of(x, {range_of(q, T, H, paged->q_stride_tok, paged->q_stride_head, e), pool_of(*paged, k_pages), pool_of(*paged, v_pages),
                      table_of(*paged, page_table), heads_of(*paged, lengths), starts_of(*paged, token_starts)}))
      return CKV_ERR_INVALID_ARG;
  if (overlap(o, l) || overlap(o, work) || overlap(l, work)) return CKV_ERR_INVALID_ARG;
  CKV_CUDA(launch_paged_attend(*paged, q, k_pages, v_pages, page_table, lengths, token_starts, out, lse_or_null,
                               static_cast<char*>(ws), (cudaStream_t)stream));
  return CKV_OK;
}

}  // extern "C"
#pragma GCC visibility pop
