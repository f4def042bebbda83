"""The fp32 attention's own source (schedule, kernel and join, without clusters) run on the host (tests/host_cuda.h), every array
ending where memory that may not be touched begins.  No GPU needed."""
import subprocess

import pytest

import host_cuda

MAIN = r"""
#include "host_cuda.h"
#include "paged_attend.cu"
#include <random>

namespace ckv {
void count_launch(int) {}
bool pdl_enabled() { return false; }
cudaError_t launch_attend_tc(const ckv_paged&, const WorkArgs&, int64_t, float, const void*, const void*, const void*, void*, float*, cudaStream_t) { return cudaErrorUnknown; }
cudaError_t launch_attend_mma(const ckv_paged&, const WorkArgs&, int64_t, float, const void*, const void*, const void*, void*, float*, cudaStream_t) { return cudaErrorUnknown; }
}  // namespace ckv

using host_cuda::guarded;
// usage: heads, KV heads, table width in pages, causal, units, then tokens of each and rows of each unit's heads
int main(int n_args, char** v) {
  const int H = atoi(v[1]), Hkv = atoi(v[2]), width = atoi(v[3]), causal = atoi(v[4]), Nu = atoi(v[5]), P = 16, G = H / Hkv;
  std::vector<int> count, len;
  for (int i = 0; i < Nu; ++i) count.push_back(atoi(v[6 + i]));
  for (int i = 0; i < Nu * Hkv; ++i) len.push_back(atoi(v[6 + Nu + i]));
  int T = 0;
  int32_t* starts = (int32_t*)guarded(4 * (Nu + 1));
  for (int u = 0; u < Nu; ++u) starts[u] = T, T += count[u];
  starts[Nu] = T;
  std::mt19937 rng(T + H);
  std::normal_distribution<float> gauss;
  auto array = [&](size_t n) {
    float* p = (float*)guarded(4 * n);
    for (size_t i = 0; i < n; ++i) p[i] = gauss(rng);
    return p;
  };
  int32_t *table = (int32_t*)guarded(4 * (size_t)Nu * Hkv * width), *lengths = (int32_t*)guarded(4 * Nu * Hkv);
  int pages = 0;
  for (int i = 0; i < Nu * Hkv; ++i) {
    lengths[i] = len[i];
    for (int s = 0; s < width; ++s) table[(size_t)i * width + s] = s * P < len[i] ? pages++ : -7;
  }
  float *q = array((size_t)T * H * 128), *k = array((size_t)pages * P * 128), *val = array((size_t)pages * P * 128);
  float *out = (float*)guarded((size_t)T * H * 512), *lse = (float*)guarded((size_t)T * H * 4);
  ckv_paged pg{};
  pg.n_units = Nu, pg.n_q_heads = H, pg.n_kv_heads = Hkv, pg.head_dim = 128, pg.dtype = CKV_F32, pg.n_tokens = T, pg.causal = causal;
  pg.page_size = P, pg.n_pages = pages, pg.max_pages = width, pg.page_stride = P * 128, pg.page_stride_row = 128;
  pg.q_stride_tok = H * 128, pg.q_stride_head = 128;
  char* ws = (char*)guarded(ckv::paged_ws(pg).total);
  if (ckv::launch_paged_attend(pg, q, k, val, table, lengths, starts, out, lse, ws, nullptr) != cudaSuccess) return printf("refused\n"), 1;
  const int* status = (const int*)ws;
  double worst = 0;
  for (int u = 0; u < Nu; ++u)
    for (int i = 0; i < count[u]; ++i)
      for (int h = 0; h < H; ++h) {
        const int g = h / G, L = len[u * Hkv + g], room = width * P;
        int sees = causal ? L - count[u] + i + 1 : L;      // rows, of which those the table has no page for are left out
        sees = sees < 0 ? 0 : sees > room ? room : sees;
        const int64_t at = (int64_t)(starts[u] + i) * H + h;
        std::vector<double> x(sees);
        double top = -INFINITY, sum = 0;
        auto row = [&](const float* pool, int j) { return pool + ((int64_t)table[(size_t)(u * Hkv + g) * width + j / P] * P + j % P) * 128; };
        for (int j = 0; j < sees; ++j) {
          for (int d = 0; d < 128; ++d) x[j] += (double)q[at * 128 + d] * row(k, j)[d];
          x[j] /= sqrt(128.0), top = fmax(top, x[j]);
        }
        std::vector<double> o(128);
        for (int j = 0; j < sees; ++j) {
          const double p = exp(x[j] - top);
          sum += p;
          for (int d = 0; d < 128; ++d) o[d] += p * row(val, j)[d];
        }
        for (int d = 0; d < 128; ++d) worst = fmax(worst, fabs(out[at * 128 + d] - (sees ? o[d] / sum : 0)));
        if (!sees) {
          if (lse[at] != -INFINITY) return printf("token %d sees nothing, lse %g\n", i, lse[at]), 1;
        } else {
          worst = fmax(worst, fabs(lse[at] - (top + log(sum))));
        }
      }
  // a logit is off by at most 132 * 2^-24 |q| |k| / sqrt(128) (|q|, |k| < 16), an output by twice that and the sums' depth, times |v| < 6
  const double tol = 6 * 2 * (132 * ldexp(1, -24) * 256 / sqrt(128.0) + 1000 * ldexp(1, -24));
  printf("%s %g status %d\n", worst <= tol ? "ok" : "off by", worst, status[0]);
  return !(worst <= tol);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return host_cuda.build(str(tmp_path_factory.mktemp("attend")), MAIN)


def go(program, H, Hkv, width, causal, counts, lens):
    p = subprocess.run([program, *map(str, (H, Hkv, width, causal, len(counts), *counts, *sum(lens, [])))], stdout=subprocess.PIPE, timeout=300)
    assert p.returncode == 0, (p.returncode, p.stdout.decode())
    return int(p.stdout.decode().split()[-1])


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("counts,lens", [([1], [[40, 700]]), ([3, 0, 1], [[5, 3], [9, 9], [64, 0]]), ([9], [[130, 4]])])
def test_split_form(program, counts, lens, causal):
    """A table too wide for clusters: the schedule splits the work, the join adds the parts."""
    assert go(program, 8, 2, 1200, causal, counts, lens) == 0


@pytest.mark.parametrize("causal", [0, 1])
def test_rows_past_the_table(program, causal):
    """Rows the table has no pages for are left out; the others are seen by the tokens that the lengths say see them."""
    for width, H, counts, more in ((3, 8, [6], (4, 0)), (3, 2, [1, 9], (1, 12, 3, 30)), (3, 2, [40], (39, 2)), (700, 2, [1, 9], (1, 12, 3, 30))):
        lens = [[16 * width + more[u * 2 + g] for g in range(2)] for u in range(len(counts))]
        assert go(program, H, 2, width, causal, counts, lens) == 4096, (width, counts)
