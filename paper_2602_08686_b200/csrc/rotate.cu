// Norms of queries and keys for each head with the position rotation, and the same on the way into a paged cache.
//
// A CTA takes kTokens consecutive tokens.  Cosine and sine of a token's angles are shared by its H + Hkv heads: the CTA
// computes them once, in 64 bits where 32 would lose the angle (position * inv_freq reaches 10^6 radians; reduced to a
// fraction of a turn in fp64 the fp32 sincospi of it is good to an ulp), and keeps them in shared memory.  A row of 128
// elements is one 16-byte piece per thread (16 threads bf16, 32 fp32); the row's sum of squares is a shuffle tree over
// those threads, and a half-split pair's other member is fetched from the thread rot_dim / 2 elements away by a shuffle.
// Everything between the load and the store is fp32, rounded once.
// Bound: HBM for long inputs (each row is read and written once), the launch for a decode step.
#include <cuda_bf16.h>

#include "paged.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 4;

struct RotArgs {
  int Nu, H, Hkv, T;
  int64_t q_tok, q_head, kv_tok, kv_head, qo_tok, qo_head, ko_tok, ko_head;   // strides in elements
  const char *q, *k, *v;
  char *q_out, *k_out;
  const int32_t *positions, *starts;
  const double* inv_freq;
  const float *qw, *kw;
  int rot, interleaved;
  float rot_scale, eps;
  // append only
  const int32_t *lengths, *table;
  char *k_pages, *v_pages;
  int32_t* new_lengths;
  int P, n_pages, max_pages;
  int64_t page_stride, page_row;
  int* status;
};

template <bool BF16>
struct Piece {   // one 16-byte piece of a row
  static constexpr int N = BF16 ? 8 : 4;
  static __device__ __forceinline__ void unpack(const uint4& x, float (&f)[N]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (BF16) {
        f[(2 * i) % N] = __uint_as_float(w[i] << 16);
        f[(2 * i + 1) % N] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        f[i % N] = __uint_as_float(w[i]);
      }
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[N]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (BF16) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f[(2 * i) % N], f[(2 * i + 1) % N]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
      } else {
        w[i] = __float_as_uint(f[i % N]);
      }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

template <bool BF16>
__global__ void __launch_bounds__(kThreads) rotate_kernel(RotArgs a, int tokens_per_cta) {
  constexpr int N = Piece<BF16>::N;
  constexpr int kLanes = kHeadDim / N;              // threads per row
  constexpr int kRows = kThreads / kLanes;          // rows in flight per CTA
  constexpr int E = BF16 ? 2 : 4;
  __shared__ float2 cs[kMaxTokens][kHeadDim / 2];
  __shared__ int s_unit[kMaxTokens], s_first[kMaxTokens], s_end[2];
  const int t0 = blockIdx.x * tokens_per_cta;
  if (threadIdx.x == 0) {
    s_end[0] = min(max(a.starts[0], 0), a.T);
    s_end[1] = min(max(a.starts[a.Nu], 0), a.T);
  }
  if (a.k_pages && threadIdx.x < tokens_per_cta) {   // which unit each token belongs to: the last start at or before it
    const int t = t0 + threadIdx.x;
    int lo = 0, hi = a.Nu - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.starts[mid] <= t) lo = mid; else hi = mid - 1;
    }
    s_unit[threadIdx.x] = lo, s_first[threadIdx.x] = a.starts[lo];
  }
  if (a.new_lengths)
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < (int64_t)a.Nu * a.Hkv; e += (int64_t)gridDim.x * kThreads) {
      int first, count;
      unit_tokens(a.starts, (int)(e / a.Hkv), a.T, first, count);
      a.new_lengths[e] = a.lengths[e] + count;
    }
  const int half = a.rot >> 1;
  for (int e = threadIdx.x; e < tokens_per_cta * half; e += kThreads) {
    const int tk = e / half, i = e - tk * half;
    if (t0 + tk < a.T) {
      double turns = (double)a.positions[t0 + tk] * a.inv_freq[i] * 0.15915494309189533577;   // 1 / (2 pi)
      turns -= rint(turns);
      float sn, co;
      sincospif(2.0f * (float)turns, &sn, &co);
      cs[tk][i] = make_float2(co * a.rot_scale, sn * a.rot_scale);
    }
  }
  __syncthreads();
  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
  const int nq = a.q ? a.H : 0, nk = a.k ? a.Hkv : 0, nv = a.v ? a.Hkv : 0, rows = nq + nk + nv;
  const bool rotates = lane * N < a.rot;
  const int shift = a.interleaved ? 0 : half / N;                     // threads between the members of a half-split pair
  const bool upper = !a.interleaved && lane >= shift && rotates;
  const int partner = rotates && !a.interleaved ? (upper ? lane - shift : lane + shift) : lane;
  const int src_lane = (threadIdx.x & 31) - lane + partner;
  const int total = tokens_per_cta * rows;
  for (int e0 = 0; e0 < total; e0 += kRows) {   // every thread of a warp takes part in the shuffles
    const int e = e0 + slot;
    const int tk = min(e / rows, tokens_per_cta - 1), t = t0 + tk, r = e - (e / rows) * rows;
    const bool live = e < total && t >= s_end[0] && t < s_end[1];
    const int kind = r < nq ? 0 : (r < nq + nk ? 1 : 2), h = r - (kind == 0 ? 0 : (kind == 1 ? nq : nq + nk));
    const char* src = kind == 0 ? a.q : (kind == 1 ? a.k : a.v);
    const int64_t from = kind == 0 ? t * a.q_tok + h * a.q_head : t * a.kv_tok + h * a.kv_head;
    uint4 raw = make_uint4(0u, 0u, 0u, 0u);
    if (live) raw = *reinterpret_cast<const uint4*>(src + from * E + lane * 16);
    float x[N], y[N];
    Piece<BF16>::unpack(raw, x);
    const float* w = kind == 0 ? a.qw : (kind == 1 ? a.kw : nullptr);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
    for (int m = 1; m < kLanes; m <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
    if (w) {
      const float inv = 1.0f / sqrtf(ss * (1.0f / kHeadDim) + a.eps);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = x[i] * inv * w[lane * N + i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = __shfl_sync(0xffffffffu, x[i], src_lane);
    if (kind < 2 && rotates) {
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const float2 c = cs[tk][(lane * N + i) >> 1];
          x[i] = y[i] * c.x - y[i + 1] * c.y;
          x[i + 1] = y[i + 1] * c.x + y[i] * c.y;
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float2 c = cs[tk][(upper ? lane - shift : lane) * N + i];
          x[i] = x[i] * c.x + (upper ? y[i] : -y[i]) * c.y;
        }
      }
    }
    if (!live) continue;
    const uint4 done = kind < 2 && (w || rotates) ? Piece<BF16>::pack(x) : raw;
    if (kind == 0 || !a.k_pages) {
      char* dst = kind == 0 ? a.q_out + (t * a.qo_tok + h * a.qo_head) * E : a.k_out + (t * a.ko_tok + h * a.ko_head) * E;
      *reinterpret_cast<uint4*>(dst + lane * 16) = done;
      continue;
    }
    const int64_t ug = (int64_t)s_unit[tk] * a.Hkv + h;
    const int64_t row = (int64_t)a.lengths[ug] + (t - s_first[tk]);
    const bool in_table = row >= 0 && row < (int64_t)a.max_pages * a.P;
    const int page = in_table ? a.table[ug * a.max_pages + (int)row / a.P] : -1;
    if ((unsigned)page >= (unsigned)a.n_pages) {
      if (lane == 0) report_status(a.status, kStatusPage);
      continue;
    }
    char* dst = kind == 1 ? a.k_pages : a.v_pages;
    *reinterpret_cast<uint4*>(dst + (page * a.page_stride + ((int)row % a.P) * a.page_row) * E + lane * 16) = done;
  }
}

}  // namespace

cudaError_t launch_rotate(const ckv_paged& pg, const ckv_rotary* rot, const void* q, const void* k, const void* v,
                          const int32_t* positions, const int32_t* starts, void* q_out, void* k_out,
                          const int32_t* lengths, const int32_t* table, void* k_pages, void* v_pages,
                          int32_t* new_lengths, int* status, cudaStream_t st) {
  RotArgs a{};
  a.Nu = pg.n_units, a.H = pg.n_q_heads, a.Hkv = pg.n_kv_heads, a.T = pg.n_tokens;
  a.q_tok = pg.q_stride_tok, a.q_head = pg.q_stride_head, a.kv_tok = pg.kv_stride_tok, a.kv_head = pg.kv_stride_head;
  const bool q_in_place = q_out == q, k_in_place = k_out == k;
  a.qo_tok = q_in_place ? a.q_tok : (int64_t)a.H * kHeadDim, a.qo_head = q_in_place ? a.q_head : kHeadDim;
  a.ko_tok = k_in_place ? a.kv_tok : (int64_t)a.Hkv * kHeadDim, a.ko_head = k_in_place ? a.kv_head : kHeadDim;
  a.q = (const char*)q, a.k = (const char*)k, a.v = (const char*)v, a.q_out = (char*)q_out, a.k_out = (char*)k_out;
  a.positions = positions, a.starts = starts;
  if (rot) {
    a.inv_freq = rot->inv_freq, a.qw = rot->q_norm_w, a.kw = rot->k_norm_w, a.rot = rot->rot_dim;
    a.interleaved = rot->interleaved, a.rot_scale = rot->rot_scale, a.eps = rot->norm_eps;
  }
  a.lengths = lengths, a.table = table, a.k_pages = (char*)k_pages, a.v_pages = (char*)v_pages;
  a.new_lengths = new_lengths, a.P = pg.page_size, a.n_pages = pg.n_pages, a.max_pages = pg.max_pages;
  a.page_stride = pg.page_stride, a.page_row = pg.page_stride_row, a.status = status;
  const int per = a.T >= 4 * 148 * 4 ? kMaxTokens : 1;
  const unsigned blocks = (unsigned)((a.T + per - 1) / per);
  if (pg.dtype == CKV_BF16) rotate_kernel<true><<<blocks ? blocks : 1, kThreads, 0, st>>>(a, per);
  else rotate_kernel<false><<<blocks ? blocks : 1, kThreads, 0, st>>>(a, per);
  count_launch();
  return cudaGetLastError();
}

}  // namespace ckv
