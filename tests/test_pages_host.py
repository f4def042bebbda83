"""The page calls' own sources (csrc/pages.cu) run on the host (tests/host_cuda.h), every array ending where memory that may not be
touched begins, against a statement of each call one entry at a time.  No GPU needed."""
import subprocess

import pytest

import host_cuda

MAIN = r"""
#include "host_cuda.h"
#include <random>
inline bool __all_sync(unsigned mask, bool x) { return __ballot_sync(mask, x) == 0xffffffffu; }
inline int __reduce_min_sync(unsigned mask, int x) { return -__reduce_max_sync(mask, -x); }
inline bool __syncthreads_and(bool x) {
  static int no = 0;
  no += !x;
  __syncthreads();
  const bool all = no == 0;
  __syncthreads();
  no = 0;
  __syncthreads();
  return all;
}
template <class T>
T __ldcg(const T* p) { return *p; }
template <class T>
void __stcg(T* p, T x) { *p = x; }
inline bool __syncthreads_or(bool x) { return !__syncthreads_and(!x); }
inline void atomicMin(int* p, int x) { *p = x < *p ? x : *p; }
inline int atomicAdd(int* p, int x) { return (*p += x) - x; }
inline int atomicSub(int* p, int x) { return (*p -= x) + x; }
#include "pages.cu"
namespace ckv {
void count_launch(int) {}
bool pdl_enabled() { return false; }
}
using host_cuda::guarded;
typedef std::vector<int> Ints;

struct Array {                 // a guarded copy of ints, and what it should become
  int32_t* p;
  Ints want;
  Array(const Ints& x) : p((int32_t*)guarded(4 * (x.empty() ? 1 : x.size()))), want(x) { std::copy(x.begin(), x.end(), p); }
  bool same(const char* name) const {
    for (size_t i = 0; i < want.size(); ++i)
      if (p[i] != want[i]) return printf("%s[%zu] is %d, not %d\n", name, i, p[i], want[i]), false;
    return true;
  }
};

int main(int n_args, char** v) {
  const int seed = atoi(v[1]);
  std::mt19937 rng(seed);
  auto any = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  const bool bad_pages = any(0, 3) == 0;
  for (int round = 0; round < 5; ++round) {
    const bool many = round == 0 && seed % 4 == 0;      // a warp a pair
    const int layers = many ? 40 : any(1, 3), seqs = many ? 3 : any(1, 4), Hkv = many ? 5 : any(1, 5), Nu = layers * seqs, pairs = Nu * Hkv, P = 16 << any(0, 2);
    const int n_pages = any(0, 2) ? any(1, many ? 2500 : 400) : any(1000, 2500), width = any(1, 9), E = any(0, 1) ? 2 : 4, row = 128 * E;
    ckv_paged pg{};
    pg.n_units = Nu, pg.n_q_heads = pg.n_kv_heads = Hkv, pg.head_dim = 128, pg.dtype = E == 2 ? CKV_BF16 : CKV_F32;
    pg.page_size = P, pg.n_pages = n_pages, pg.max_pages = width;
    pg.page_stride_row = 128 + 8 * any(0, 1), pg.page_stride = P * pg.page_stride_row;
    const size_t pool_bytes = ((size_t)(n_pages - 1) * pg.page_stride + (P - 1) * pg.page_stride_row + 128) * E;
    // a state: pages handed out at random, some of them to several heads
    Ints refs(n_pages, 0), held(pairs), lengths(pairs), table((size_t)pairs * width), fresh;
    for (int i = 0; i < n_pages; ++i) fresh.push_back(i);
    std::shuffle(fresh.begin(), fresh.end(), rng);
    for (int i = 0; i < n_pages; ++i)
      if (any(0, 2) == 0) refs[fresh[n_pages - 1 - i]] += any(0, 1);   // other batches' pages
    size_t at = 0;
    for (int p = 0; p < pairs; ++p) {
      held[p] = any(0, width);
      for (int s = 0; s < width; ++s) {
        int& page = table[(size_t)p * width + s];
        page = -77;
        if (s >= held[p]) continue;
        if (p && any(0, 3) == 0 && s < held[p - 1] && (unsigned)table[(size_t)(p - 1) * width + s] < (unsigned)n_pages) page = table[(size_t)(p - 1) * width + s];
        else if (at < fresh.size()) page = fresh[at++];
        else { held[p] = s; page = -77; continue; }
        ++refs[page];
        if (bad_pages && any(0, 30) == 0) --refs[page], page = any(0, 1) ? n_pages : -1;
      }
      lengths[p] = any(0, held[p] * P);
    }
    char* pools[2];
    std::vector<char> content[2];
    for (int k = 0; k < 2; ++k) {
      pools[k] = (char*)guarded((pool_bytes + 15) / 16 * 16);
      content[k].resize(pool_bytes);
      for (char& c : content[k]) c = (char)rng();
      memcpy(pools[k], content[k].data(), pool_bytes);
    }
    auto place = [&](int page, int r) { return ((size_t)page * pg.page_stride + (size_t)r * pg.page_stride_row) * E; };
    char* ws = (char*)guarded(ckv::reserve_ws(pairs, n_pages).total);
    for (size_t i = 256; i < ckv::reserve_ws(pairs, n_pages).total; ++i) ws[i] = (char)rng();
    int* status = (int*)ws;
    bool report = false;
    auto fine = [&](int page) { return (unsigned)page < (unsigned)n_pages; };
    auto checked = [&](const char* what) {
      for (int k = 0; k < 2; ++k)
        if (memcmp(pools[k], content[k].data(), pool_bytes)) return printf("%s: pool %d\n", what, k), false;
      const bool said = status[63] == 0x434b5631 && status[0] == 4096;
      if (said != report) return printf("%s: reported %d, not %d\n", what, said, report), false;
      memset(ws, 0, 256);
      report = false;
      return true;
    };
    memset(ws, 0, 256);
    Array dev_refs(refs), dev_held(held), dev_len(lengths), dev_table(table);
    // -------------------------------------------------------- reserve
    {
      const int n_lists = any(0, 1) ? pairs : seqs;
      Ints more(n_lists);
      for (int& x : more) x = any(0, 3) == 0 ? 0 : any(0, 1) ? any(1, 3) : any(1, 4 * P);
      Array dev_more(more), room(Ints{5, 5});
      const ckv::Lists lists{n_lists != seqs, Hkv, seqs};
      if (ckv::launch_pages_reserve(pg, lists, dev_more.p, dev_len.p, dev_held.p, dev_table.p, dev_refs.p, pools[0], pools[1], room.p, ws, nullptr)) return 1;
      Ints r2 = refs, t2 = table, h2 = held, frees;
      for (int i = 0; i < n_pages; ++i)
        if (refs[i] == 0) frees.push_back(i);
      size_t next = 0;
      std::vector<char> c2[2] = {content[0], content[1]};
      for (int p = 0; p < pairs; ++p) {
        const int n = more[n_lists == pairs && n_lists != seqs ? p : p / Hkv % seqs];
        if (n <= 0) continue;
        int slots = (lengths[p] + n + P - 1) / P;
        if (slots > width) slots = width, report = true;
        for (int s = lengths[p] / P; s < slots; ++s) {
          int& page = t2[(size_t)p * width + s];
          const bool copy = s < held[p];
          if (copy && !fine(page)) { report = true; continue; }
          if (copy && refs[page] <= 1) continue;
          if (!copy && s < held[p]) continue;
          const int got = next < frees.size() ? frees[next] : -1;
          ++next;
          if (got < 0) continue;
          if (copy) {
            --r2[page];
            for (int j = 0; s == lengths[p] / P && j < lengths[p] % P; ++j)
              for (int k = 0; k < 2; ++k) memcpy(&c2[k][place(got, j)], &content[k][place(page, j)], row);
          }
          page = got, r2[got] = 1;
        }
        // growth in front of what the pair will write (lengths below held - 1 pages) cannot be: slots from held on
        h2[p] = std::max(h2[p], slots);
      }
      if (next <= frees.size()) {
        refs = r2, table = t2, held = h2;
        for (int k = 0; k < 2; ++k) content[k] = c2[k];
        room.want = {(int)(frees.size() - next), 0};
      } else {
        room.want = {(int)frees.size(), (int)(next - frees.size())};
      }
      dev_refs.want = refs, dev_held.want = held, dev_table.want = table;
      if (!room.same("room") || !dev_refs.same("refs") || !dev_held.same("held") || !dev_table.same("table") || !checked("reserve")) return 1;
    }
    // ----------------------------------------------------------- fork
    {
      const int n_new = any(0, 7), keep_old = any(0, 1), P2 = layers * n_new * Hkv;
      Ints parents(n_new);
      for (int& x : parents) x = any(0, 9) == 0 ? -1 : (bad_pages && any(0, 9) == 0) ? (any(0, 1) ? seqs : -2) : any(0, seqs - 1);
      Array dev_par(parents), len2(Ints(P2, 7)), held2(Ints(P2, 7)), table2(Ints((size_t)P2 * width, 7));
      if (ckv::launch_pages_fork(pg, layers, n_new, dev_par.p, dev_len.p, dev_held.p, dev_table.p, dev_refs.p, keep_old, len2.p, held2.p, table2.p, status, nullptr)) return 1;
      Ints r2 = refs;
      for (int l = 0; l < layers; ++l)
        for (int s = 0; s < n_new; ++s)
          for (int g = 0; g < Hkv; ++g) {
            const int to = (l * n_new + s) * Hkv + g, par = parents[s];
            if (par < -1 || par >= seqs) report = true;
            const bool has = par >= 0 && par < seqs;
            const int from = has ? (l * seqs + par) * Hkv + g : 0;
            len2.want[to] = has ? lengths[from] : 0, held2.want[to] = has ? held[from] : 0;
            for (int x = 0; has && x < held[from]; ++x) {
              table2.want[(size_t)to * width + x] = table[(size_t)from * width + x];
              if (fine(table[(size_t)from * width + x])) ++r2[table[(size_t)from * width + x]];
            }
          }
      for (int p = 0; p < pairs; ++p)
        for (int x = 0; x < held[p]; ++x) {
          const int page = table[(size_t)p * width + x];
          int children = 0;
          for (int y : parents) children += y == p / Hkv % seqs;
          if (children == 0 && keep_old) continue;
          if (children == 1 && !keep_old) continue;
          if (!fine(page)) report = true;
          else if (!keep_old) --r2[page];
        }
      // (an old batch whose sequence has one child hands its pages over: nothing counts)
      for (int p = 0; p < pairs && !keep_old; ++p) {
        int children = 0;
        for (int y : parents) children += y == p / Hkv % seqs;
        for (int x = 0; children == 1 && x < held[p]; ++x)
          if (fine(table[(size_t)p * width + x])) --r2[table[(size_t)p * width + x]];
      }
      refs = r2, dev_refs.want = refs;
      if (!len2.same("new lengths") || !held2.same("new held") || !table2.same("new table") || !dev_refs.same("refs after a fork") || !checked("fork")) return 1;
      // the new ones end
      ckv_paged p2 = pg;
      p2.n_units = layers * n_new;
      if (n_new > 0) {
        if (ckv::launch_pages_trim(p2, nullptr, held2.p, table2.p, dev_refs.p, status, nullptr)) return 1;
        for (int p = 0; p < P2; ++p) {
          for (int x = 0; x < held2.want[p]; ++x) {
            if (fine(table2.want[(size_t)p * width + x])) --refs[table2.want[(size_t)p * width + x]];
            else report = true;
          }
          held2.want[p] = 0;
        }
        dev_refs.want = refs;
        if (!held2.same("held after the end") || !dev_refs.same("refs after the end") || !checked("end")) return 1;
      }
      if (!keep_old) {               // the old ones are back
        for (int p = 0; p < pairs; ++p)
          for (int x = 0; x < held[p]; ++x)
            if (fine(table[(size_t)p * width + x])) ++refs[table[(size_t)p * width + x]];
        std::copy(refs.begin(), refs.end(), dev_refs.p);
      }
    }
    // ----------------------------------------------------------- keep
    {
      const bool tails = any(0, 1);
      const int n_lists = tails && any(0, 1) ? seqs : pairs;
      const bool by_seq = n_lists == seqs;
      Ints tail(n_lists), begins(n_lists), counts(n_lists), rows;
      for (int i = 0; i < any(0, 3); ++i) rows.push_back(-5);
      std::vector<bool> broken(n_lists);
      const bool longer = any(0, 1);
      for (int i = 0; i < n_lists; ++i) {
        int least = 1 << 20;
        for (int p = 0; p < pairs; ++p)
          if ((by_seq ? p / Hkv % seqs : p) == i) least = std::min(least, lengths[p]);
        tail[i] = tails ? any(0, least) : least;
        begins[i] = rows.size();
        const int share = any(1, 8);
        for (int x = 0; x < tail[i]; ++x)
          if (any(0, share) > 0 || x < 3) rows.push_back(x);
        counts[i] = rows.size() - begins[i];
        if (bad_pages && counts[i] > 1 && any(0, 4) == 0) {
          broken[i] = true;
          const int how = any(0, 3);
          if (how == 0) rows.back() = rows[rows.size() - 2];
          if (how == 1) rows.back() = tail[i];
          if (how == 2) rows[begins[i]] = -1;
          if (how == 3) counts[i] = tail[i] + 1;
        }
      }
      if (longer) rows.resize(rows.size() + 40 * n_lists, 9);     // room: lists are expected to be long
      Array dev_rows(rows), dev_b(begins), dev_c(counts), dev_t(tail), out(Ints(pairs, 7));
      const ckv::Lists lists{!by_seq, Hkv, seqs};
      const bool with_refs = any(0, 1);
      if (ckv::launch_keep_rows(pg, lists, n_lists, dev_rows.p, (int)rows.size(), dev_b.p, dev_c.p, tails ? dev_t.p : nullptr, with_refs ? dev_refs.p : nullptr,
                                dev_len.p, dev_table.p, pools[0], pools[1], out.p, status, nullptr)) return 1;
      bool unsure = false;
      for (int p = 0; p < pairs; ++p) {
        const int l = by_seq ? p / Hkv % seqs : p, base = tails ? lengths[p] - tail[l] : 0;
        bool ok = !broken[l];
        if (!tails && by_seq) ok = ok && tail[l] <= lengths[p];
        auto entry = [&](int i) { return rows[begins[l] + i]; };
        int first = 0;
        while (ok && first < counts[l] && entry(first) == first) ++first;
        for (int i = first; ok && i < counts[l]; ++i) {
          const int from = table[(size_t)p * width + (base + entry(i)) / P], to = table[(size_t)p * width + (base + i) / P];
          if (!fine(from) || !fine(to)) { ok = false; break; }
          if (refs[to] > 1) {
            if (with_refs) ok = false;
            else unsure = true;         // a page of several heads moved by each of them: not allowed
          }
        }
        if (!ok) { report = true, out.want[p] = lengths[p]; continue; }
        out.want[p] = base + counts[l];
        for (int i = first; i < counts[l]; ++i)
          for (int k = 0; k < 2; ++k) {
            auto where = [&](int r) { return place(table[(size_t)p * width + r / P], r % P); };
            memmove(&content[k][where(base + i)], &content[k][where(base + entry(i))], row);
          }
      }
      if (!out.same("kept lengths")) return 1;
      if (unsure)
        for (int k = 0; k < 2; ++k) content[k].assign(pools[k], pools[k] + pool_bytes);
      if (!checked("keep")) return 1;
      // what is behind the rows left goes back
      if (ckv::launch_pages_trim(pg, out.p, dev_held.p, dev_table.p, dev_refs.p, status, nullptr)) return 1;
      for (int p = 0; p < pairs; ++p) {
        const int keep = (out.want[p] + P - 1) / P;
        for (int x = keep; x < held[p]; ++x) {
          if (fine(table[(size_t)p * width + x])) --refs[table[(size_t)p * width + x]];
          else report = true;
        }
        held[p] = std::min(held[p], keep);
      }
      dev_refs.want = refs, dev_held.want = held;
      if (!dev_refs.same("refs after trim") || !dev_held.same("held after trim") || !checked("trim")) return 1;
    }
  }
  printf("ok\n");
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    return host_cuda.build(str(tmp_path_factory.mktemp("pages")), MAIN)


@pytest.mark.parametrize("seed", range(12))
def test_random_states(program, seed):
    """Reserve, fork, end, keep and trim on random states: shared pages, exhausted pools, bad pages and lists among them."""
    p = subprocess.run([program, str(seed)], stdout=subprocess.PIPE, timeout=600)
    assert p.returncode == 0, (p.returncode, p.stdout.decode()[-500:])
