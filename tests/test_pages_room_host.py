"""What `room` of ckv_pages_reserve says, from its own source (csrc/pages.cu) run on the host (tests/host_cuda.h): the free pages that were not handed
out.  A page that all its holders replace in one call is free after it, and counts in the next call's room.  No GPU needed."""
import subprocess

import pytest

import host_cuda
from test_pages_host import MAIN

PROGRAM = MAIN.split("int main(")[0] + r"""
// One page of five rows that `heads` sequences share (`other`: a batch that is not in the call holds it too), in a pool of n_pages.
int main() {
  const int P = 16, width = 3;
  for (int heads : {1, 2, 4, 33, 700})
    for (int other : {0, 1})
      for (int spare : {-1, 0, 1, 5}) {               // pages there are beside those needed
        const int copies = heads + other > 1 ? heads : 0, n_pages = 1 + copies + spare;
        if (n_pages < 1) continue;
        ckv_paged pg{};
        pg.n_units = heads, pg.n_q_heads = pg.n_kv_heads = 1, pg.head_dim = 128, pg.dtype = CKV_BF16, pg.page_size = P, pg.n_pages = n_pages;
        pg.max_pages = width, pg.page_stride_row = 128, pg.page_stride = P * 128;
        char* pools[2];
        for (char*& p : pools) p = (char*)guarded((size_t)n_pages * P * 256);
        for (int k = 0; k < 2; ++k)
          for (int i = 0; i < 5 * 256; ++i) pools[k][(size_t)(n_pages - 1) * P * 256 + i] = (char)(i % 251 + k);
        Ints refs(n_pages, 0), table(heads * width, -5);
        refs[n_pages - 1] = heads + other;
        for (int h = 0; h < heads; ++h) table[h * width] = n_pages - 1;
        Array d_refs(refs), d_held(Ints(heads, 1)), d_len(Ints(heads, 5)), d_table(table), one(Ints(heads, 1)), none(Ints(heads, 0)), room(Ints{-3, -3});
        const size_t bytes = ckv::reserve_ws(heads, n_pages).total;
        char* const ws = (char*)guarded(bytes);
        const ckv::Lists lists{0, 1, heads};
        const bool enough = spare >= 0;
        auto call = [&](Array& more) {
          return ckv::launch_pages_reserve(pg, lists, more.p, d_len.p, d_held.p, d_table.p, d_refs.p, pools[0], pools[1], room.p, ws, nullptr);
        };
        if (call(one)) return 1;
        room.want = enough ? Ints{spare, 0} : Ints{copies + spare, -spare};
        if (enough && copies) {
          for (int h = 0; h < heads; ++h) d_table.want[h * width] = h, d_refs.want[h] = 1;
          d_refs.want[n_pages - 1] = other;
          for (int k = 0; k < 2; ++k)
            for (int h = 0; h < heads; ++h)
              if (memcmp(pools[k] + (size_t)h * P * 256, pools[k] + (size_t)(n_pages - 1) * P * 256, 5 * 256)) return printf("copy %d\n", h), 1;
        }
        if (!room.same("room") || !d_refs.same("refs") || !d_table.same("table") || !d_held.same("held")) return 1;
        // no new rows: all that is free
        if (call(none)) return 1;
        int zero = 0;
        for (int x : d_refs.want) zero += x == 0;
        if (enough && zero != spare + (copies && !other)) return printf("%d are free\n", zero), 1;
        room.want = {zero, 0};
        if (!room.same("room of no rows") || !d_refs.same("refs") || !d_table.same("table")) return 1;
        if (((int*)ws)[63] == 0x434b5631) return printf("reported\n"), 1;
        for (char* p : pools) munmap((char*)((uintptr_t)p & ~4095ull), (size_t)n_pages * P * 256);
      }
  printf("ok\n");
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return host_cuda.build(str(tmp_path_factory.mktemp("room")), PROGRAM)


def test_room(program):
    p = subprocess.run([program], stdout=subprocess.PIPE, timeout=600)
    assert p.returncode == 0, (p.returncode, p.stdout.decode()[-500:])
