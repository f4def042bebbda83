"""The page calls' own sources (csrc/pages.cu) run on the host (tests/host_cuda.h) on states with entries that are none: heads whose `held` is outside
0..max_pages or whose length is negative, and pages that are held though their count is zero.  Such heads are left as they are (a child of
one is empty), all others are treated as ever, and it is reported.  No GPU needed."""
import subprocess

import pytest

import host_cuda
from test_pages_host import MAIN

PROGRAM = MAIN.split("int main(")[0] + r"""
int main(int n_args, char** v) {
  std::mt19937 rng(atoi(v[1]));
  auto any = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  for (int round = 0; round < 12; ++round) {
    const bool many = round == 0;                     // several heads a CTA
    const int layers = any(1, 3), seqs = many ? 70 : any(1, 4), Hkv = any(1, 5), Nu = layers * seqs, pairs = Nu * Hkv, P = 16, width = any(1, 6), spare = any(0, 300);
    const int n_pages = pairs * width + spare;
    ckv_paged pg{};
    pg.n_units = Nu, pg.n_q_heads = pg.n_kv_heads = Hkv, pg.head_dim = 128, pg.dtype = CKV_BF16, pg.page_size = P, pg.n_pages = n_pages;
    pg.max_pages = width, pg.page_stride_row = 128, pg.page_stride = P * 128;
    char* pools[2];
    for (char*& p : pools) p = (char*)guarded((size_t)n_pages * P * 256);
    Ints refs(n_pages, 0), held(pairs), lengths(pairs), table((size_t)pairs * width, -77), at(n_pages);
    for (int i = 0; i < n_pages; ++i) at[i] = i;
    std::shuffle(at.begin(), at.end(), rng);
    std::vector<char> broken(pairs, 0);
    int next = 0;
    for (int p = 0; p < pairs; ++p) {
      held[p] = any(0, width);
      for (int s = 0; s < held[p]; ++s) {
        int& page = table[(size_t)p * width + s];
        page = p && any(0, 2) == 0 && table[(size_t)(p - 1) * width + s] >= 0 && !broken[p - 1] ? table[(size_t)(p - 1) * width + s] : at[next++];
        ++refs[page];
      }
      lengths[p] = any(0, held[p] * P);
      if (any(0, 3) == 0) {
        const int wrong[] = {-1, -1000, width + 1, 2147483647, -2147483647 - 1};
        broken[p] = 1;
        for (int s = held[p]; s < width; ++s) table[(size_t)p * width + s] = at[next++], ++refs[table[(size_t)p * width + s]];   // pages that would be found
        if (any(0, 2)) held[p] = wrong[any(0, 4)];
        else lengths[p] = any(0, 1) ? -1 : -2147483647 - 1;
      }
    }
    const size_t bytes = ckv::reserve_ws(pairs, n_pages).total;
    char* const ws = (char*)guarded(bytes);
    int* const status = (int*)ws;
    Array d_refs(refs), d_held(held), d_len(lengths), d_table(table);
    bool report = false;
    for (char b : broken) report = report || b;
    auto same = [&](const char* what, bool should) {
      const bool said = status[63] == 0x434b5631 && status[0] == 4096;
      memset(ws, 0, 256);
      if (said != should) return printf("%s: reported %d\n", what, said), false;
      return d_refs.same(what) && d_held.same(what) && d_table.same(what);
    };
    memset(ws, 0, bytes);
    // reserve: the others get their pages, the lowest free ones
    {
      const int n_lists = any(0, 1) ? pairs : seqs;
      Ints more(n_lists);
      for (int& x : more) x = any(0, P);
      Array d_more(more), room(Ints{7, 7});
      Ints free_pages, r = refs;
      for (int i = 0; i < n_pages; ++i)
        if (refs[i] == 0) free_pages.push_back(i);
      size_t got = 0;
      auto want_table = table, want_held = held;
      for (int p = 0; p < pairs; ++p) {
        const int n = more[n_lists == pairs && n_lists != seqs ? p : p / Hkv % seqs];
        if (broken[p] || n == 0) continue;
        int slots = (lengths[p] + n + P - 1) / P;
        if (slots > width) slots = width, report = true;
        for (int s = lengths[p] / P; s < slots; ++s) {
          int& page = want_table[(size_t)p * width + s];
          if (s < held[p] && refs[page] <= 1) continue;
          if (s < held[p]) --r[page];
          if (got < free_pages.size()) page = free_pages[got], r[free_pages[got]] = 1;
          ++got;
        }
        want_held[p] = std::max(held[p], slots);
      }
      if (got <= free_pages.size()) d_table.want = table = want_table, d_held.want = held = want_held, d_refs.want = refs = r, room.want = {(int)(free_pages.size() - got), 0};
      else room.want = {(int)free_pages.size(), (int)(got - free_pages.size())};
      if (ckv::launch_pages_reserve(pg, ckv::Lists{n_lists != seqs, Hkv, seqs}, d_more.p, d_len.p, d_held.p, d_table.p, d_refs.p, pools[0], pools[1], room.p, ws, nullptr)) return 1;
      if (!room.same("room") || !same("reserve", report)) return 1;
    }
    report = false;
    for (char b : broken) report = report || b;
    // fork, the old batch going on or not
    const int n_new = any(0, 6), keep_old = any(0, 1), P2 = layers * n_new * Hkv;
    Ints parents(n_new);
    for (int& x : parents) x = any(-1, seqs - 1);
    // pages that nobody has counted, where all only count up
    std::vector<char> uncounted(n_pages, 0);
    if (keep_old && any(0, 1))
      for (int p = 0; p < pairs; ++p)
        if (!broken[p] && held[p] > 0 && any(0, 5) == 0) uncounted[table[(size_t)p * width]] = 1, d_refs.p[table[(size_t)p * width]] = refs[table[(size_t)p * width]] = 0;
    Array d_par(parents), len2(Ints(P2, 7)), held2(Ints(P2, 7)), table2(Ints((size_t)P2 * width, 7));
    for (int p = 0; p < pairs; ++p) {
      int children = 0;
      for (int l = 0; l < n_new; ++l) children += parents[l] == p / Hkv % seqs;
      for (int s = 0; s < held[p] && !broken[p]; ++s) {
        int& count = refs[table[(size_t)p * width + s]];
        report = report || (uncounted[table[(size_t)p * width + s]] && children > 0);
        count += children - !keep_old;
      }
      for (int s = 0; s < n_new; ++s) {
        if (parents[s] != p / Hkv % seqs) continue;
        const int to = (p / Hkv / seqs * n_new + s) * Hkv + p % Hkv;
        len2.want[to] = broken[p] ? 0 : lengths[p], held2.want[to] = broken[p] ? 0 : held[p];
        for (int x = 0; x < held2.want[to]; ++x) table2.want[(size_t)to * width + x] = table[(size_t)p * width + x];
      }
    }
    for (int to = 0; to < P2; ++to)
      if (parents[to / Hkv % n_new] < 0) len2.want[to] = held2.want[to] = 0;
    d_refs.want = refs;
    if (ckv::launch_pages_fork(pg, layers, n_new, d_par.p, d_len.p, d_held.p, d_table.p, d_refs.p, keep_old, len2.p, held2.p, table2.p, status, nullptr)) return 1;
    if (!same("fork", report) || !len2.same("new lengths") || !held2.same("new held") || !table2.same("new table")) return 1;
    // trim the new batch, then the old one if it goes on
    if (n_new) {
      ckv_paged p2 = pg;
      p2.n_units = layers * n_new;
      if (ckv::launch_pages_trim(p2, nullptr, held2.p, table2.p, d_refs.p, status, nullptr)) return 1;
      report = false;
      for (int p = 0; p < P2; ++p) {
        for (int s = 0; s < held2.want[p]; ++s) {
          int& count = refs[table2.want[(size_t)p * width + s]];
          --count;
        }
        held2.want[p] = 0;
      }
      d_refs.want = refs;
      if (!held2.same("held after the end") || !same("end", report)) return 1;
    }
    if (keep_old) {
      const bool lengths_too = any(0, 1);
      Ints shorter(pairs);
      for (int p = 0; p < pairs; ++p) shorter[p] = lengths[p] < 0 ? lengths[p] : any(0, lengths[p]);
      Array d_short(shorter);
      report = false;
      for (int p = 0; p < pairs; ++p) {
        if (held[p] < 0 || held[p] > width || (lengths_too && lengths[p] < 0)) { report = true; continue; }
        const int keep = lengths_too ? (shorter[p] + P - 1) / P : 0;
        for (int s = keep; s < held[p]; ++s) {
          if (uncounted[table[(size_t)p * width + s]]) report = true;
          else --refs[table[(size_t)p * width + s]];
        }
        held[p] = std::min(held[p], keep);
      }
      d_refs.want = refs, d_held.want = held;
      if (ckv::launch_pages_trim(pg, lengths_too ? d_short.p : nullptr, d_held.p, d_table.p, d_refs.p, status, nullptr)) return 1;
      if (!same("trim", report)) return 1;
    }
    for (char* p : pools) munmap((char*)((uintptr_t)p & ~4095ull), (size_t)n_pages * P * 256);
  }
  printf("ok\n");
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return host_cuda.build(str(tmp_path_factory.mktemp("counts")), PROGRAM)


@pytest.mark.parametrize("seed", range(8))
def test_heads_that_are_none(program, seed):
    p = subprocess.run([program, str(seed)], stdout=subprocess.PIPE, timeout=600)
    assert p.returncode == 0, (p.returncode, p.stdout.decode()[-500:])
