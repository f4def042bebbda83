// Host side of the paged-cache entry points: argument validation and work space.
#include <initializer_list>

#include "paged.cuh"

using namespace ckv;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool good(std::initializer_list<const void*> ps, size_t a) {
  for (const void* p : ps)
    if (!p || !aligned(p, a)) return false;
  return true;
}
int64_t esize(const ckv_paged& pg) { return pg.dtype == CKV_BF16 ? 2 : 4; }

// The bytes an array covers (none: {0, 0}).
struct Range {
  uintptr_t lo = 0, hi = 0;
};
Range bytes_of(const void* p, int64_t bytes) {
  if (!p) return {};
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return {lo, lo + (uintptr_t)bytes};
}
Range ints_of(const void* p, int64_t n) { return bytes_of(p, n * 4); }   // or floats
// A token array [T, heads, d] with these strides; what would leave the address space ends with it.
Range range_of(const void* p, int64_t T, int64_t heads, int64_t tok, int64_t head, int64_t esz) {
  if (!p) return {};
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  const __int128 hi = (__int128)lo + ((__int128)(T - 1) * tok + (__int128)(heads - 1) * head + kHeadDim) * esz;
  return {lo, hi < (__int128)UINTPTR_MAX ? (uintptr_t)hi : UINTPTR_MAX};
}
bool overlap(const Range& a, const Range& b) { return a.lo < b.hi && b.lo < a.hi; }
bool clear_of(const Range& written, std::initializer_list<Range> others) {
  for (const Range& o : others)
    if (overlap(written, o)) return false;
  return true;
}
Range pool_of(const ckv_paged& pg, const void* pool) {
  return range_of(pool, pg.n_pages, pg.page_size, pg.page_stride, pg.page_stride_row, esize(pg));
}

ckv_status check_tokens(const ckv_paged* pg) {
  if (!pg) return CKV_ERR_INVALID_ARG;
  if (pg->n_units < 1 || pg->n_q_heads < 1 || pg->n_kv_heads < 1 || pg->n_tokens < 0 || pg->max_new < 0)
    return CKV_ERR_INVALID_ARG;
  if (pg->n_q_heads % pg->n_kv_heads) return CKV_ERR_INVALID_ARG;
  if (pg->dtype != CKV_BF16 && pg->dtype != CKV_F32) return CKV_ERR_INVALID_ARG;
  if (pg->head_dim != kHeadDim || pg->n_kv_heads > kMaxKvHeads || pg->n_tokens > (1 << 20) || pg->n_q_heads > 65535)
    return CKV_ERR_UNSUPPORTED;
  if ((int64_t)pg->n_units * pg->n_kv_heads > 65536) return CKV_ERR_UNSUPPORTED;
  if ((int64_t)pg->n_tokens * pg->n_q_heads > (1 << 30)) return CKV_ERR_UNSUPPORTED;   // the kernels count query rows in 32 bits
  return CKV_OK;
}
// Strides of a token array: rows on 16-byte boundaries (that they do not overlap is asked where they are written, see in_place_ok).
bool token_strides(const ckv_paged& pg, int64_t tok, int64_t head, int heads) {
  const int64_t e = esize(pg);
  if (tok < 0 || head < 0 || (tok * e) % 16 || (head * e) % 16) return false;
  if ((heads > 1 && head < kHeadDim) || (pg.n_tokens > 1 && tok < kHeadDim)) return false;
  return tok < ((int64_t)1 << 38) && head < ((int64_t)1 << 38);   // a tensor map's strides end at 2^40 bytes
}
// Rows of 128 elements at base + i * outer + j * inner, i < n_outer, j < n_inner (strides in elements).
struct Rows {
  const void* base;
  int64_t n_outer, outer, n_inner, inner, esz;
  Range range() const { return range_of(base, n_outer, n_inner, outer, inner, esz); }
  // no row shares memory with another: one stride steps over all that the other reaches
  bool apart_from_itself() const {
    return n_outer == 1 || n_inner == 1 || outer >= (n_inner - 1) * inner + kHeadDim || inner >= (n_outer - 1) * outer + kHeadDim;
  }
};
// Whether no row of a is on one of b's.  Arrays that are interleaved (views of a fused projection) have one outer stride; with two
// different ones over the same memory they count as overlapping.
bool apart(const Rows& a, const Rows& b) {
  if (!overlap(a.range(), b.range())) return true;
  const int64_t row = kHeadDim * a.esz, s = a.outer * a.esz;
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.base) - reinterpret_cast<uintptr_t>(a.base));
  const bool steps = a.n_outer > 1 || b.n_outer > 1;
  if (steps && (a.n_outer != b.n_outer || a.outer != b.outer || s < row)) return false;
  // each within an outer step, and beside the other there
  const int64_t at = steps ? ((d % s) + s) % s : 0;
  if (steps && at >= (a.n_inner - 1) * a.inner * a.esz + row && at + (b.n_inner - 1) * b.inner * b.esz + row <= s) return true;
  // or their rows take turns: a[0] b[0] a[1] b[1] ...
  if (a.inner == b.inner && a.inner > 0 && (!steps || a.outer % a.inner == 0)) {
    const int64_t i = a.inner * a.esz, between = ((d % i) + i) % i;
    if (between >= row && between + row <= i) return true;
  }
  // row j of a against row k of b, whichever outer steps bring them closest
  auto meet = [&](int64_t x) {   // x: from one to the other within the same step
    if (!steps) return -row < x && x < row;
    const int64_t r = ((x % s) + s) % s, i = (r - x) / s;   // i steps on it is r away, one step less r - s
    return (r < row && i > -a.n_outer && i < a.n_outer) || (s - r < row && i - 1 > -a.n_outer && i - 1 < a.n_outer);
  };
  if (a.inner == b.inner) {      // only the difference of the two matters
    for (int64_t k = -(a.n_inner - 1); k < b.n_inner; ++k)
      if (meet(d + k * a.inner * a.esz)) return false;
    return true;
  }
  for (int64_t j = 0; j < a.n_inner; ++j)
    for (int64_t k = 0; k < b.n_inner; ++k)
      if (meet(d + (k * b.inner - j * a.inner) * a.esz)) return false;
  return true;
}
// Rows that are turned in place: each is one (token, head) pair's, and none is among the other arrays'.
bool in_place_ok(const Rows& x, std::initializer_list<Rows> others) {
  if (!x.apart_from_itself()) return false;
  for (const Rows& o : others)
    if (o.base && !apart(x, o)) return false;
  return true;
}
ckv_status check_pages(const ckv_paged* pg) {
  if (pg->page_size < 1 || pg->n_pages < 1 || pg->max_pages < 1) return CKV_ERR_INVALID_ARG;
  if (pg->causal != 0 && pg->causal != 1) return CKV_ERR_INVALID_ARG;
  if (!(pg->scale > -3.0e38f && pg->scale < 3.0e38f)) return CKV_ERR_INVALID_ARG;
  const int P = pg->page_size;
  if (P != 16 && P != 32 && P != 64 && P != 128 && P != 256) return CKV_ERR_UNSUPPORTED;
  if ((int64_t)pg->max_pages * P > (1 << 24)) return CKV_ERR_UNSUPPORTED;
  const int64_t e = esize(*pg);
  if ((pg->page_stride * e) % 16 || (pg->page_stride_row * e) % 16) return CKV_ERR_INVALID_ARG;
  if (pg->page_stride_row < kHeadDim) return CKV_ERR_INVALID_ARG;
  if (pg->n_pages > 1 && pg->page_stride < (P - 1) * pg->page_stride_row + kHeadDim) return CKV_ERR_INVALID_ARG;
  if (pg->page_stride_row >= ((int64_t)1 << 32) || pg->page_stride < 0 || pg->page_stride >= ((int64_t)1 << 38))
    return CKV_ERR_UNSUPPORTED;
  return CKV_OK;
}
// Keys and values go to pools that share no row (they may be interleaved).
bool pools_apart(const ckv_paged& pg, const void* k_pages, const void* v_pages) {
  const int64_t e = esize(pg);
  return apart({k_pages, pg.n_pages, pg.page_stride, pg.page_size, pg.page_stride_row, e},
               {v_pages, pg.n_pages, pg.page_stride, pg.page_size, pg.page_stride_row, e});
}
ckv_status check_rotary(const ckv_rotary* r) {
  if (r->rot_dim < 0 || r->rot_dim > kHeadDim) return CKV_ERR_INVALID_ARG;
  if (r->rot_dim % 16) return CKV_ERR_UNSUPPORTED;
  if (r->interleaved != 0 && r->interleaved != 1) return CKV_ERR_INVALID_ARG;
  if (r->rot_dim && !good({r->inv_freq}, 8)) return CKV_ERR_INVALID_ARG;
  if ((r->q_norm_w && !aligned(r->q_norm_w, 4)) || (r->k_norm_w && !aligned(r->k_norm_w, 4))) return CKV_ERR_INVALID_ARG;
  if (!(r->norm_eps >= 0.f && r->norm_eps < 3.0e38f) || !(r->rot_scale > -3.0e38f && r->rot_scale < 3.0e38f))
    return CKV_ERR_INVALID_ARG;
  return CKV_OK;
}
ckv_status check_paged_ws(size_t need, const void* ws, size_t ws_bytes) {
  return ws && aligned(ws, 256) && ws_bytes >= need ? CKV_OK : CKV_ERR_WORKSPACE;
}
constexpr size_t kStatusBytes = 256;   // all that the calls without partial results use
// Where the turned tokens go: over the input (in place) or to a dense array.
Range out_range(const ckv_paged& pg, const void* out, const void* in, const Range& in_range, int heads) {
  return out == in ? in_range : range_of(out, pg.n_tokens, heads, (int64_t)heads * kHeadDim, kHeadDim, esize(pg));
}
Range freq_of(const ckv_rotary* r) { return r ? bytes_of(r->inv_freq, r->rot_dim / 2 * 8) : Range{}; }
Range q_norm_of(const ckv_rotary* r) { return r ? ints_of(r->q_norm_w, kHeadDim) : Range{}; }
Range k_norm_of(const ckv_rotary* r) { return r ? ints_of(r->k_norm_w, kHeadDim) : Range{}; }
Range starts_of(const ckv_paged& pg, const void* starts) { return ints_of(starts, (int64_t)pg.n_units + 1); }
Range heads_of(const ckv_paged& pg, const void* per_head) { return ints_of(per_head, (int64_t)pg.n_units * pg.n_kv_heads); }
Range table_of(const ckv_paged& pg, const void* table) { return ints_of(table, (int64_t)pg.n_units * pg.n_kv_heads * pg.max_pages); }

#define CKV_TRY(expr)                  \
  do {                                 \
    ckv_status st__ = (expr);          \
    if (st__ != CKV_OK) return st__;   \
  } while (0)
#define CKV_CUDA(expr)                               \
  do {                                               \
    if ((expr) != cudaSuccess) return CKV_ERR_CUDA;  \
  } while (0)

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t ckv_paged_workspace_bytes(const ckv_paged* paged) {
  if (check_tokens(paged) != CKV_OK || check_pages(paged) != CKV_OK) return 0;
  return paged_ws(*paged).total;
}

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
