"""ckv_keep_rows' own source (csrc/pages.cu) run on the host (tests/host_cuda.h) with lists that ascend but are no rows: entries below zero, also behind
others of their kind.  The page table lies between memory that may not be touched: a lookup in front of it ends the process.  No GPU needed."""
import subprocess

import pytest

import host_cuda
from test_pages_host import MAIN

PROGRAM = MAIN.split("int main(")[0] + r"""
int main() {
  const int P = 16, Hkv = 2, seqs = 3, pairs = seqs * Hkv, width = 8, n_pages = pairs * width, row = 256, count = 6;
  const int low[][2] = {{-2, -1}, {-1, 0}, {-40000000, -39999999}, {-2147483647 - 1, -2147483647}, {-2147483647 - 1, -1}};
  for (int len : {100, 128})
    for (int span : {20, 100})
      for (int pad : {0, 400})                       // short lists go to warps, long ones to CTAs
        for (const int* pair : low)
          for (int at : {0, 1, 4})                   // where in the list the two are
            for (bool first : {false, true}) {       // the table begins, or ends, where memory that may not be touched is
              ckv_paged pg{};
              pg.n_units = seqs, pg.n_q_heads = pg.n_kv_heads = Hkv, pg.head_dim = 128, pg.dtype = CKV_BF16, pg.page_size = P, pg.n_pages = n_pages;
              pg.max_pages = width, pg.page_stride_row = 128, pg.page_stride = P * 128;
              int32_t* const table = (int32_t*)guarded(4 * pairs * width, !first);
              for (int i = 0; i < pairs * width; ++i) table[i] = (i * 5) % n_pages;
              std::vector<char> content[2];
              char* pools[2];
              for (int k = 0; k < 2; ++k) {
                pools[k] = (char*)guarded((size_t)n_pages * P * row);
                for (int r = 0; r < n_pages * P; ++r) memset(pools[k] + (size_t)r * row, r * 7 + k, row), memcpy(pools[k] + (size_t)r * row, &r, 4);
                content[k].assign(pools[k], pools[k] + (size_t)n_pages * P * row);
              }
              Ints rows, begins, counts(seqs, count), tails(seqs, span), lengths(pairs, len);
              for (int s = 0; s < seqs; ++s) {
                begins.push_back(rows.size());
                for (int i = 0; i < count; ++i) rows.push_back(2 * i + 1);
              }
              rows[begins[1] + at] = pair[0], rows[begins[1] + at + 1] = pair[1];
              for (int i = 0; i < pad; ++i) rows.push_back(3);
              Array d_rows(rows), d_begins(begins), d_counts(counts), d_tails(tails), d_len(lengths), out(Ints(pairs, 7));
              int* const status = (int*)guarded(256);
              if (ckv::launch_keep_rows(pg, ckv::Lists{0, Hkv, seqs}, seqs, d_rows.p, (int)rows.size(), d_begins.p, d_counts.p, d_tails.p, nullptr, d_len.p, table, pools[0],
                                        pools[1], out.p, status, nullptr)) return 1;
              for (int p = 0; p < pairs; ++p) {
                const bool bad = p / Hkv == 1;
                out.want[p] = bad ? len : len - span + count;
                auto where = [&](int j) { return ((size_t)table[p * width + j / P] * P + j % P) * row; };
                for (int k = 0; k < 2 && !bad; ++k)
                  for (int i = 0; i < count; ++i) memcpy(&content[k][where(len - span + i)], &content[k][where(len - span + rows[begins[p / Hkv] + i])], row);
              }
              if (!out.same("lengths")) return 1;
              for (int k = 0; k < 2; ++k)
                if (memcmp(pools[k], content[k].data(), content[k].size())) return printf("pool %d\n", k), 1;
              if (status[63] != 0x434b5631 || status[0] != 4096) return printf("not reported\n"), 1;
              munmap((char*)((uintptr_t)table & ~4095ull), 4096);
              for (int k = 0; k < 2; ++k) munmap(pools[k], content[k].size());
            }
  printf("ok\n");
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return host_cuda.build(str(tmp_path_factory.mktemp("lists")), PROGRAM)


def test_entries_below_zero_behind_others(program):
    p = subprocess.run([program], stdout=subprocess.PIPE, timeout=600)
    assert p.returncode == 0, (p.returncode, p.stdout.decode()[-500:])
