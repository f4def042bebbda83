// Argument checks that the paged entry points share: alignment, strides, and which arrays are apart.
#pragma once
#include <initializer_list>

#include "paged.cuh"

namespace ckv {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool good(std::initializer_list<const void*> ps, size_t a) {
  for (const void* p : ps)
    if (!p || !aligned(p, a)) return false;
  return true;
}
inline int64_t esize(const ckv_paged& pg) { return pg.dtype == CKV_BF16 ? 2 : 4; }

// The bytes an array covers (none: {0, 0}).
struct Range {
  uintptr_t lo = 0, hi = 0;
};
inline Range bytes_of(const void* p, int64_t bytes) {
  if (!p) return {};
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return {lo, lo + (uintptr_t)bytes};
}
inline Range ints_of(const void* p, int64_t n) { return bytes_of(p, n * 4); }   // or floats
// A token array [T, heads, d] with these strides; what would leave the address space ends with it.
inline Range range_of(const void* p, int64_t T, int64_t heads, int64_t tok, int64_t head, int64_t esz) {
  if (!p) return {};
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  const __int128 hi = (__int128)lo + ((__int128)(T - 1) * tok + (__int128)(heads - 1) * head + kHeadDim) * esz;
  return {lo, hi < (__int128)UINTPTR_MAX ? (uintptr_t)hi : UINTPTR_MAX};
}
inline bool overlap(const Range& a, const Range& b) { return a.lo < b.hi && b.lo < a.hi; }
inline bool clear_of(const Range& written, std::initializer_list<Range> others) {
  for (const Range& o : others)
    if (overlap(written, o)) return false;
  return true;
}
inline Range pool_of(const ckv_paged& pg, const void* pool) {
  return range_of(pool, pg.n_pages, pg.page_size, pg.page_stride, pg.page_stride_row, esize(pg));
}

inline ckv_status check_tokens(const ckv_paged* pg) {
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
inline bool token_strides(const ckv_paged& pg, int64_t tok, int64_t head, int heads) {
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
inline bool apart(const Rows& a, const Rows& b) {
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
inline bool in_place_ok(const Rows& x, std::initializer_list<Rows> others) {
  if (!x.apart_from_itself()) return false;
  for (const Rows& o : others)
    if (o.base && !apart(x, o)) return false;
  return true;
}
inline ckv_status check_pages(const ckv_paged* pg) {
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
inline bool pools_apart(const ckv_paged& pg, const void* k_pages, const void* v_pages) {
  const int64_t e = esize(pg);
  return apart({k_pages, pg.n_pages, pg.page_stride, pg.page_size, pg.page_stride_row, e},
               {v_pages, pg.n_pages, pg.page_stride, pg.page_size, pg.page_stride_row, e});
}
inline ckv_status check_rotary(const ckv_rotary* r) {
  if (r->rot_dim < 0 || r->rot_dim > kHeadDim) return CKV_ERR_INVALID_ARG;
  if (r->rot_dim % 16) return CKV_ERR_UNSUPPORTED;
  if (r->interleaved != 0 && r->interleaved != 1) return CKV_ERR_INVALID_ARG;
  if (r->rot_dim && !good({r->inv_freq}, 8)) return CKV_ERR_INVALID_ARG;
  if ((r->q_norm_w && !aligned(r->q_norm_w, 4)) || (r->k_norm_w && !aligned(r->k_norm_w, 4))) return CKV_ERR_INVALID_ARG;
  if (!(r->norm_eps >= 0.f && r->norm_eps < 3.0e38f) || !(r->rot_scale > -3.0e38f && r->rot_scale < 3.0e38f))
    return CKV_ERR_INVALID_ARG;
  return CKV_OK;
}
inline ckv_status check_paged_ws(size_t need, const void* ws, size_t ws_bytes) {
  return ws && aligned(ws, 256) && ws_bytes >= need ? CKV_OK : CKV_ERR_WORKSPACE;
}
constexpr size_t kStatusBytes = 256;   // all that the calls without partial results use
// Where the turned tokens go: over the input (in place) or to a dense array.
inline Range out_range(const ckv_paged& pg, const void* out, const void* in, const Range& in_range, int heads) {
  return out == in ? in_range : range_of(out, pg.n_tokens, heads, (int64_t)heads * kHeadDim, kHeadDim, esize(pg));
}
inline Range freq_of(const ckv_rotary* r) { return r ? bytes_of(r->inv_freq, r->rot_dim / 2 * 8) : Range{}; }
inline Range q_norm_of(const ckv_rotary* r) { return r ? ints_of(r->q_norm_w, kHeadDim) : Range{}; }
inline Range k_norm_of(const ckv_rotary* r) { return r ? ints_of(r->k_norm_w, kHeadDim) : Range{}; }
inline Range starts_of(const ckv_paged& pg, const void* starts) { return ints_of(starts, (int64_t)pg.n_units + 1); }
inline Range heads_of(const ckv_paged& pg, const void* per_head) { return ints_of(per_head, (int64_t)pg.n_units * pg.n_kv_heads); }
inline Range table_of(const ckv_paged& pg, const void* table) { return ints_of(table, (int64_t)pg.n_units * pg.n_kv_heads * pg.max_pages); }

#define CKV_TRY(expr)                  \
  do {                                 \
    ckv_status st__ = (expr);          \
    if (st__ != CKV_OK) return st__;   \
  } while (0)
#define CKV_CUDA(expr)                               \
  do {                                               \
    if ((expr) != cudaSuccess) return CKV_ERR_CUDA;  \
  } while (0)

}  // namespace ckv
