"""rotate_kernel's own source run on the host (tests/host_cuda.h): every array ends where memory that may not be touched begins, so a
read or write behind it ends the process.  No GPU needed."""
import subprocess

import pytest

import host_cuda

MAIN = r"""
#include "host_cuda.h"
#include "rotate.cu"
#include <random>

namespace ckv {
void count_launch(int) {}
bool pdl_enabled() { return false; }
}  // namespace ckv

using host_cuda::guarded;
template <bool BF16>
struct Tokens {       // [T, heads, 128] inside a wider row, as a fused projection's output holds it; ends with the last row
  static constexpr int E = BF16 ? 2 : 4;
  int64_t T, heads, tok;
  char* p;
  Tokens(int64_t T_, int64_t heads_, int64_t tok_) : T(T_), heads(heads_), tok(tok_), p((char*)guarded(((T_ - 1) * tok_ + heads_ * 128) * E)) {}
  double get(int64_t t, int64_t h, int d) const {
    const char* at = p + ((t * tok + h * 128) + d) * E;
    return BF16 ? (double)__uint_as_float((unsigned)*(const unsigned short*)at << 16) : (double)*(const float*)at;
  }
  void set(int64_t t, int64_t h, int d, float x) {
    char* at = p + ((t * tok + h * 128) + d) * E;
    if (BF16) *(unsigned short*)at = (unsigned short)(__float_as_uint(x) >> 16);
    else *(float*)at = x;
  }
};

template <bool BF16>
int go(int T, int H, int Hkv, bool append, bool norm, int pad) {
  std::mt19937 rng(T + H);
  std::normal_distribution<float> gauss;
  const int rot = 96, P = 16;
  const int64_t wide = (H + 2 * Hkv) * 128;
  Tokens<BF16> q(T, H, wide), k(T, Hkv, wide), v(T, Hkv, wide), qo(T, H, H * 128), ko(T, Hkv, Hkv * 128);
  for (auto* x : {&q, &k, &v})
    for (int t = 0; t < T; ++t)
      for (int h = 0; h < x->heads; ++h)
        for (int d = 0; d < 128; ++d) x->set(t, h, d, gauss(rng));
  int32_t* pos = (int32_t*)guarded(4 * T);
  for (int t = 0; t < T; ++t) pos[t] = 3 * t + 70000;
  int32_t* starts = (int32_t*)guarded(4 * 3);
  starts[0] = 0, starts[1] = T / 3, starts[2] = T - pad;
  double* inv = (double*)guarded(8 * rot / 2);
  for (int i = 0; i < rot / 2; ++i) inv[i] = pow(10000.0, -2.0 * i / rot);
  float* w[2];
  for (auto& x : w) {
    x = (float*)guarded(4 * 128);
    for (int d = 0; d < 128; ++d) x[d] = 1.0f + 0.1f * gauss(rng);
  }
  ckv_rotary r{inv, norm ? w[0] : nullptr, norm ? w[1] : nullptr, rot, 0, 1.25f, 1e-6f};
  ckv_paged pg{};
  pg.n_units = 2, pg.n_q_heads = H, pg.n_kv_heads = Hkv, pg.head_dim = 128, pg.dtype = BF16 ? CKV_BF16 : CKV_F32, pg.n_tokens = T;
  pg.q_stride_tok = pg.kv_stride_tok = wide, pg.q_stride_head = pg.kv_stride_head = 128;
  // the cache: unit u's head g has room for its tokens behind 5 u + g rows
  pg.page_size = P, pg.max_pages = (T + 100) / P + 2, pg.n_pages = 2 * Hkv * pg.max_pages;
  pg.page_stride = P * 128, pg.page_stride_row = 128;
  int32_t *table = nullptr, *lengths = nullptr, *grown = nullptr, *status = nullptr;
  char *kp = nullptr, *vp = nullptr;
  const int E = BF16 ? 2 : 4;
  if (append) {
    table = (int32_t*)guarded(4 * (size_t)pg.n_pages), lengths = (int32_t*)guarded(4 * 2 * Hkv), grown = (int32_t*)guarded(4 * 2 * Hkv);
    status = (int32_t*)guarded(256);
    for (int i = 0; i < pg.n_pages; ++i) table[i] = pg.n_pages - 1 - i;
    for (int u = 0; u < 2; ++u)
      for (int g = 0; g < Hkv; ++g) lengths[u * Hkv + g] = 5 * u + g;
    kp = (char*)guarded((size_t)pg.n_pages * P * 128 * E), vp = (char*)guarded((size_t)pg.n_pages * P * 128 * E);
  }
  ckv::launch_rotate(pg, &r, q.p, k.p, append ? v.p : nullptr, pos, starts, qo.p, append ? nullptr : ko.p, lengths, table, kp, vp, grown,
                     status, nullptr);
  if (append && status[0]) return printf("a page was missed\n"), 1;
  double worst = 0;
  for (int t = 0; t < T; ++t) {
    const bool live = t < starts[2];
    const int u = t >= starts[1];
    for (int kind = 0; kind < 3; ++kind) {
      const Tokens<BF16>& x = kind == 0 ? q : kind == 1 ? k : v;
      if (kind == 2 && !append) continue;
      for (int h = 0; h < x.heads; ++h) {
        double y[128], ss = 0;
        for (int d = 0; d < 128; ++d) y[d] = x.get(t, h, d), ss += y[d] * y[d];
        if (kind < 2) {
          if (norm)
            for (int d = 0; d < 128; ++d) y[d] *= w[kind][d] / sqrt(ss / 128 + 1e-6);
          for (int i = 0; i < rot / 2; ++i) {
            const double c = 1.25 * cos(pos[t] * inv[i]), s = 1.25 * sin(pos[t] * inv[i]), a = y[i], b = y[i + rot / 2];
            y[i] = a * c - b * s, y[i + rot / 2] = b * c + a * s;
          }
        }
        for (int d = 0; d < 128; ++d) {
          double got;
          if (kind == 0) got = qo.get(t, h, d);
          else if (!append) got = ko.get(t, h, d);
          else if (!live) continue;
          else {
            const int row = 5 * u + h + t - starts[u];
            const int page = table[(u * Hkv + h) * pg.max_pages + row / P];
            const char* at = (kind == 1 ? kp : vp) + (((int64_t)page * P + row % P) * 128 + d) * E;
            got = BF16 ? (double)__uint_as_float((unsigned)*(const unsigned short*)at << 16) : (double)*(const float*)at;
          }
          if (!live) {
            if (got != 0) return printf("row %d of no unit was written\n", t), 1;
            continue;
          }
          // half a step of the output's type, and 40 steps of fp32 of the pair's size
          const double tol = (BF16 ? ldexp(1, -8) : 0) * fabs(y[d]) + 40 * ldexp(1, -24) * 12;
          if (kind == 2 ? got != y[d] : !(fabs(got - y[d]) <= tol)) return printf("token %d kind %d head %d dim %d: %g not %g\n", t, kind, h, d, got, y[d]), 1;
          worst = fmax(worst, fabs(got - y[d]));
        }
      }
    }
  }
  if (append)
    for (int i = 0; i < 2 * Hkv; ++i)
      if (grown[i] != lengths[i] + starts[i / Hkv + 1] - starts[i / Hkv]) return printf("length %d\n", i), 1;
  printf("ok %g\n", worst);
  return 0;
}
int main(int, char** v) {
  const int T = atoi(v[2]), H = atoi(v[3]), Hkv = atoi(v[4]), append = atoi(v[5]), norm = atoi(v[6]), pad = atoi(v[7]);
  return v[1][0] == 'b' ? go<true>(T, H, Hkv, append, norm, pad) : go<false>(T, H, Hkv, append, norm, pad);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return host_cuda.build(str(tmp_path_factory.mktemp("rotate")), MAIN)


@pytest.mark.parametrize("append", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,Hkv,norm,pad", [
    (1, 8, 2, 0, 0), (5, 3, 3, 1, 2),
    (889, 12, 12, 1, 1),          # two tokens a CTA, the last one alone
    (1783, 32, 8, 0, 0),          # four: three tokens in the last
    (3553, 12, 5, 0, 3),          # eight: one in the last
    (3559, 8, 6, 1, 0),           # eight: seven in the last
])
def test_no_row_beside_the_arrays(program, T, H, Hkv, dtype, append, norm, pad):
    p = subprocess.run([program, dtype, *map(str, (T, H, Hkv, append, norm, pad))], stdout=subprocess.PIPE, timeout=300)
    assert p.returncode == 0, (p.returncode, p.stdout.decode())
