// Norms of queries and keys for each head with the position rotation, and the same on the way into a paged cache.
//
// A CTA takes one to eight consecutive tokens.  Cosine and sine of a token's angles are shared by its H + Hkv heads: the CTA
// computes them once, in 64 bits where 32 would lose the angle (position * inv_freq reaches 10^6 radians); its fraction of a
// turn, at most one half, is rounded to fp32 (2^-26 of a turn: 9.4e-8 radians, 1.5 ulp of a sine) for an fp32 sincospi.  16 threads (bf16) or 32 (fp32) share a row of 128
// elements, with two 8-byte pieces each that hold whole pairs: the same place in either half of the rotated dimensions where
// pairs are half a rotation apart, neighbours otherwise.  So no thread needs another's elements, and since a thread keeps its
// dimensions and its token over all the rows it takes, its cosines stay in registers.  (With one 16-byte piece, the
// partner's by shuffles and the cosines from shared memory per row, the 32k prompt took 243 us: instruction issue.)  The
// row's sum of squares is a shuffle tree.  Everything between the load and the store is fp32, rounded once.
// Bound: HBM for long inputs (each row is read and written once; the 32k prompt in 118 to 123 us by card, 0.83 to 0.87 of the measured copy rate), the
// launch and three dependent reads for a decode step (16 sequences: 4 us).
#include <cuda_bf16.h>

#include "paged.cuh"

namespace ckv {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTokens = 8;   // a warp's rows (two in bf16) are one token's up to here
constexpr int kRotBatch = 2;   // rows a thread has under way (more cost registers and with them CTAs: 4 rows, 3 CTAs: the same 120 us
                               // on the prompt, 32 instead of 22 us on the ragged chunk)
constexpr int kCtas = 4;
constexpr int kWaves = 1;

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
  int log_p, n_pages, max_pages;
  int64_t page_stride, page_row;
  int* status;
};

// 8 bytes of a row: four bf16 or two fp32.
template <bool BF16>
struct Piece {
  static constexpr int N = BF16 ? 4 : 2;
  static __device__ __forceinline__ void unpack(const uint2& r, float (&f)[N]) {
    if (BF16) {
      f[0] = __uint_as_float(r.x << 16), f[1] = __uint_as_float(r.x & 0xffff0000u);
      f[2 % N] = __uint_as_float(r.y << 16), f[3 % N] = __uint_as_float(r.y & 0xffff0000u);
    } else {
      f[0] = __uint_as_float(r.x), f[1] = __uint_as_float(r.y);
    }
  }
  static __device__ __forceinline__ uint2 pack(const float (&f)[N]) {
    if (!BF16) return make_uint2(__float_as_uint(f[0]), __float_as_uint(f[1]));
    const __nv_bfloat162 lo = __floats2bfloat162_rn(f[0], f[1]), hi = __floats2bfloat162_rn(f[2 % N], f[3 % N]);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
};
struct Two {   // a thread's share of a row
  uint2 a, b;
};

// The unit that token t belongs to: the last start at or before it.  A warp counts the starts 32 at a time (one round trip for a
// batch of up to 32 units), or halves the range where there are many.
__device__ __forceinline__ int unit_of(const int32_t* starts, int Nu, int t, int lane) {
  if (Nu <= 512) {
    int n = 0;
    for (int u0 = 0; u0 < Nu; u0 += 32) n += __popc(__ballot_sync(0xffffffffu, u0 + lane < Nu && starts[u0 + lane] <= t));
    return max(n - 1, 0);
  }
  int lo = 0, hi = Nu - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (starts[mid] <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// What a thread does to its share of every row of its token.
template <bool BF16>
struct Turn {
  static constexpr int N = Piece<BF16>::N;
  int off_a, off_b;        // bytes from the row's start to its two pieces
  bool rotates, apart;     // its pairs are (a[i], b[i]), or neighbours within the pieces
  float c[N], s[N];        // of pair i: (a[i], b[i]), or the i-th neighbours, a's before b's
  float eps;
};

// One token's heads of one kind: rows src + head * in_stride, head = r0, r0 + step, ... < heads, normed (kNorm, weight w), turned
// and handed to store(head, whether in the first batch, index in the batch, pieces).  kBatch rows are under way at a time; `raw` are the ones already asked for.  All threads
// of a warp go as many rounds (the shuffles want them all); where there is no such token (the last CTA's end) nothing is read.
template <bool BF16, int kBatch, bool kNorm, class Store>
__device__ __forceinline__ void do_heads(const char* src, int64_t in_stride, int heads, int r0, int step, bool token, bool live, const Turn<BF16>& q,
                                         const float* w, Two (&raw)[kBatch], Store&& store) {
  constexpr int N = Piece<BF16>::N, E = BF16 ? 2 : 4;
  float wa[N], wb[N];
  if (kNorm) {
#pragma unroll
    for (int i = 0; i < N; ++i) wa[i] = __ldg(w + q.off_a / E + i), wb[i] = __ldg(w + q.off_b / E + i);
  }
  const char* at = src + (r0 + (int64_t)kBatch * step) * in_stride;
  const int readable = token ? heads : 0;
  for (int r = r0; r - r0 < heads; r += kBatch * step) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int h = r + b * step;
      float x[N], y[N];
      Piece<BF16>::unpack(raw[b].a, x);
      Piece<BF16>::unpack(raw[b].b, y);
      if (kNorm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) ss = fmaf(x[i], x[i], fmaf(y[i], y[i], ss));
#pragma unroll
        for (int m = 1; m < kHeadDim / (2 * N); m <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        const float inv = 1.0f / sqrtf(ss * (1.0f / kHeadDim) + q.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= inv * wa[i], y[i] *= inv * wb[i];
      }
      if (q.rotates) {
        if (q.apart) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float u = x[i] * q.c[i] - y[i] * q.s[i];
            y[i] = y[i] * q.c[i] + x[i] * q.s[i];
            x[i] = u;
          }
        } else {
#pragma unroll
          for (int i = 0; i < N; i += 2) {
            const float u = x[i] * q.c[i / 2] - x[i + 1] * q.s[i / 2], v = y[i] * q.c[N / 2 + i / 2] - y[i + 1] * q.s[N / 2 + i / 2];
            x[i + 1] = x[i + 1] * q.c[i / 2] + x[i] * q.s[i / 2];
            y[i + 1] = y[i + 1] * q.c[N / 2 + i / 2] + y[i] * q.s[N / 2 + i / 2];
            x[i] = u, y[i] = v;
          }
        }
      }
      // (untouched values pack to their own bits)
      if (live && h < heads) store(h, r == r0, b, Two{Piece<BF16>::pack(x), Piece<BF16>::pack(y)});
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (r + (kBatch + b) * step < readable)
        raw[b].a = *reinterpret_cast<const uint2*>(at + q.off_a), raw[b].b = *reinterpret_cast<const uint2*>(at + q.off_b);
      at += step * in_stride;
    }
  }
}

template <bool BF16, int kBatch>
__global__ void __launch_bounds__(kThreads, kCtas) rotate_kernel(const __grid_constant__ RotArgs a, int tokens_per_cta) {
  constexpr int N = Piece<BF16>::N, E = BF16 ? 2 : 4;
  constexpr int kLanes = kHeadDim / (2 * N);        // threads per row
  constexpr int kRows = kThreads / kLanes;          // rows the CTA takes side by side
  __shared__ float2 cs[kMaxTokens][kHeadDim / 2];
  const int t0 = blockIdx.x * tokens_per_cta;
  const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
  const int half = a.rot >> 1;
  // the thread's token, the first of its rows of it, and its share of a row
  const int step = kRows / tokens_per_cta, tk = slot / step, r0 = slot - tk * step;
  const int64_t t = t0 + tk;
  Turn<BF16> turn;
  turn.eps = a.eps, turn.rotates = lane * 2 * N < a.rot, turn.apart = !a.interleaved && turn.rotates;
  turn.off_a = (turn.apart ? lane * N : lane * 2 * N) * E;
  turn.off_b = turn.off_a + (turn.apart ? half : N) * E;
  pdl_wait();
  pdl_launch_dependents();
  const char* q_src = a.q + t * a.q_tok * E;
  const char* k_src = a.k + t * a.kv_tok * E;
  Two raw[kBatch], raw_k[kBatch];
  auto first_rows = [&](const char* src, int64_t stride, int heads, Two (&x)[kBatch]) {
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      x[b].a = x[b].b = make_uint2(0u, 0u);
      if (src && t < a.T && r0 + b * step < heads) {
        const char* at = src + (r0 + b * step) * stride;
        x[b].a = *reinterpret_cast<const uint2*>(at + turn.off_a), x[b].b = *reinterpret_cast<const uint2*>(at + turn.off_b);
      }
    }
  };
  first_rows(a.q ? q_src : nullptr, a.q_head * E, a.H, raw);
  first_rows(a.k ? k_src : nullptr, a.kv_head * E, a.Hkv, raw_k);
  const bool live = t >= min(max(a.starts[0], 0), a.T) && t < min(max(a.starts[a.Nu], 0), a.T);
  // Where the token's rows start in the pools (-1: nowhere), for the first batch while the angles are worked on.
  int64_t pair0 = 0;
  int ahead = 0;
  auto place = [&](int h) -> int64_t {
    const int64_t row = (int64_t)a.lengths[pair0 + h] + ahead;
    const bool in_table = row >= 0 && row < (int64_t)a.max_pages << a.log_p;
    const int page = in_table ? a.table[(pair0 + h) * a.max_pages + ((int)row >> a.log_p)] : -1;
    if ((unsigned)page < (unsigned)a.n_pages) return (page * a.page_stride + ((int)row & ((1 << a.log_p) - 1)) * a.page_row) * E;
    if (lane == 0) report_status(a.status, kStatusPage);
    return -1;
  };
  int64_t at[kBatch];
  if (a.k_pages && a.k) {
    const int u = unit_of(a.starts, a.Nu, (int)t, threadIdx.x & 31);   // a warp's rows are one token's
    pair0 = (int64_t)u * a.Hkv, ahead = (int)t - a.starts[u];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) at[b] = live && r0 + b * step < a.Hkv ? place(r0 + b * step) : -1;
  }
  if (a.new_lengths)
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < (int64_t)a.Nu * a.Hkv; e += (int64_t)gridDim.x * kThreads) {
      int first, count;
      unit_tokens(a.starts, (int)(e / a.Hkv), a.T, first, count);
      a.new_lengths[e] = a.lengths[e] + count;
    }
  for (int e = threadIdx.x; e < tokens_per_cta * half; e += kThreads) {
    const int et = e / half, i = e - et * half;
    if (t0 + et < a.T) {
      double turns = (double)a.positions[t0 + et] * a.inv_freq[i] * 0.15915494309189533577;   // 1 / (2 pi)
      turns -= rint(turns);
      float sn, co;
      sincospif(2.0f * (float)turns, &sn, &co);
      cs[et][i] = make_float2(co * a.rot_scale, sn * a.rot_scale);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float2 x = turn.rotates ? cs[tk][lane * N + i] : make_float2(1.f, 0.f);   // apart or not, the thread's pairs in order
    turn.c[i] = x.x, turn.s[i] = x.y;
  }
  if (a.q) {
    char* dst = a.q_out + t * a.qo_tok * E;
    auto store = [&](int h, bool, int, const Two& x) {
      char* at = dst + h * a.qo_head * E;
      *reinterpret_cast<uint2*>(at + turn.off_a) = x.a, *reinterpret_cast<uint2*>(at + turn.off_b) = x.b;
    };
    if (a.qw) do_heads<BF16, kBatch, true>(q_src, a.q_head * E, a.H, r0, step, t < a.T, live, turn, a.qw, raw, store);
    else do_heads<BF16, kBatch, false>(q_src, a.q_head * E, a.H, r0, step, t < a.T, live, turn, nullptr, raw, store);
  }
  if (!a.k) return;
  auto store_k = [&](int h, bool first, int b, const Two& x) {
    const int64_t to = !a.k_pages ? (t * a.ko_tok + h * a.ko_head) * E : (first ? at[b] : place(h));
    if (to < 0) return;
    char* dst = (a.k_pages ? a.k_pages : a.k_out) + to;
    *reinterpret_cast<uint2*>(dst + turn.off_a) = x.a, *reinterpret_cast<uint2*>(dst + turn.off_b) = x.b;
  };
  if (a.kw) do_heads<BF16, kBatch, true>(k_src, a.kv_head * E, a.Hkv, r0, step, t < a.T, live, turn, a.kw, raw_k, store_k);
  else do_heads<BF16, kBatch, false>(k_src, a.kv_head * E, a.Hkv, r0, step, t < a.T, live, turn, nullptr, raw_k, store_k);
  if (!a.v || !live) return;
  const char* v_src = a.v + t * a.kv_tok * E + lane * 16;
#pragma unroll
  for (int b = 0; b < kBatch; ++b)
    if (at[b] >= 0) *reinterpret_cast<uint4*>(a.v_pages + at[b] + lane * 16) = *reinterpret_cast<const uint4*>(v_src + (r0 + b * step) * a.kv_head * E);
  for (int h = r0 + kBatch * step; h < a.Hkv; h += step) {
    const int64_t to = place(h);
    if (to >= 0) *reinterpret_cast<uint4*>(a.v_pages + to + lane * 16) = *reinterpret_cast<const uint4*>(v_src + h * a.kv_head * E);
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
  a.new_lengths = new_lengths, a.n_pages = pg.n_pages, a.max_pages = pg.max_pages;
  while ((1 << a.log_p) < pg.page_size) ++a.log_p;
  a.page_stride = pg.page_stride, a.page_row = pg.page_stride_row, a.status = status;
  // Tokens of a CTA share its set-up (the reads before the first row, the angles): as many as leave kWaves rounds of CTAs.
  int per = kMaxTokens;
  while (per > 1 && (int64_t)a.T < (int64_t)per * 148 * 3 * kWaves) per /= 2;
  const unsigned blocks = (unsigned)((a.T + per - 1) / per);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks ? blocks : 1), cfg.blockDim = dim3(kThreads), cfg.stream = st;
  cudaLaunchAttribute attr = pdl_attribute();
  cfg.attrs = &attr, cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, pg.dtype == CKV_BF16 ? rotate_kernel<true, kRotBatch> : rotate_kernel<false, kRotBatch>, a, per);
  count_launch();
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ckv
