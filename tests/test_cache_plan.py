"""The plan of the chunks' attention over the paged cache, on the CPU.

The kernel's own planning code (cache_plan.cuh) is compiled for the host and run by 32 lanes that take
turns: whatever the lengths, windows and blocks, the items' key tiles make up every unit's list exactly once,
a cut unit's partial results are the ones that are joined, and no number leaves the scratch's arrays.
"""
import subprocess

import pytest

from paper_2608_27922_gb300 import build as B

SRC = r"""
#include "cache_plan.cuh"
#include <csetjmp>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <map>
#include <random>
#include <tuple>
#include <ucontext.h>
#include <vector>
using namespace dkv::cache;
using namespace dkv::cache::chunk;

// ---- 32 lanes that take turns, each as far as the next thing that they do together
static const int STACK = 1 << 16;
static ucontext_t start[32], home;
static jmp_buf at[32], back;
static bool begun[32], over[32];
static unsigned given[32], shared[32];
static int current;
static std::function<void(int)> body;
static std::vector<char> stacks(32 * STACK);

static void lane_main() {
  body(current);
  over[current] = true;
  _longjmp(back, 1);
}
namespace dkv { namespace cache { namespace chunk {
int host_lane() { return current; }
const unsigned* host_warp(unsigned mine) {
  given[current] = mine;
  if (_setjmp(at[current]) == 0) _longjmp(back, 1);
  return shared;
}
}}}
static void run_warp(std::function<void(int)> f) {
  body = f;
  for (int i = 0; i < 32; ++i) begun[i] = over[i] = false;
  for (;;) {
    int ended = 0;
    for (volatile int i = 0; i < 32; i = i + 1) {
      current = i;
      if (_setjmp(back) == 0) {
        if (begun[i]) _longjmp(at[i], 1);
        begun[i] = true;
        getcontext(&start[i]);
        start[i].uc_stack.ss_sp = &stacks[i * STACK];
        start[i].uc_stack.ss_size = STACK;
        start[i].uc_link = &home;
        makecontext(&start[i], lane_main, 0);
        setcontext(&start[i]);
      }
    }
    for (int i = 0; i < 32; ++i) ended += over[i];
    if (ended == 32) return;
    if (ended) { puts("lanes disagree"); exit(1); }
    memcpy(shared, given, sizeof(shared));
  }
}

struct Seen { int cut, even, longer, uneven, uncut; };

static int check(const std::vector<std::pair<int, int>>& seqs, int H, int G, int ctas, Mask m, Seen& seen) {
  int32_t status[2] = {0, 0};
  std::vector<int32_t> len, row{0}, table(seqs.size() * 4, 0);
  int rows = 0, most = 1;
  for (auto& s : seqs) {
    rows += s.first;
    row.push_back(rows);
    len.push_back(s.second);
    most = most > s.first ? most : s.first;
  }
  if (rows == 0) return 0;
  Job j{};
  j.c.status = status; j.c.H = H; j.c.d = 128; j.c.page_len = 16; j.c.page_log2 = 4; j.c.n_pages = 4;
  j.s = Seqs{table.data(), len.data(), row.data(), (int)seqs.size(), 1 << 20, rows};
  j.m = m; j.G = G; j.TQ = BQ / G; j.max_rows = most;
  j.cut = (int64_t)H * ((rows + 2 * j.TQ - 1) / (2 * j.TQ)) < CUT_ROUNDS * ctas;

  // the units as the definition has them: tiles of their lists, by (sequence, head, place)
  std::map<std::tuple<int, int, int>, int> tiles;
  int units = 0, first = -1, longest = 0;
  bool ends_even = true;
  for (int b = 0; b < (int)seqs.size(); ++b) {
    const int n = seqs[b].first, L = seqs[b].second, nu = (n + 2 * j.TQ - 1) / (2 * j.TQ);
    for (int t = 0; t < nu; ++t) {
      const int t0 = t * 2 * j.TQ, k = n - t0 < 2 * j.TQ ? n - t0 : 2 * j.TQ;
      const List l = list_of(m, k, L - n + t0, L);
      for (int h = 0; h < H; ++h) tiles[{b, h, t}] = l.n;
      longest = l.n > longest ? l.n : longest;
      if (t == 0 || t == nu - 1) {
        if (first < 0) first = l.n;
        ends_even &= l.n == first;
      }
      units += H;
      // a tile that a token sees is on the list
      for (int i : {0, k / 2, k - 1}) {
        const int p = L - n + t0 + i;
        if (p < 0) continue;
        const int64_t e0 = m.block ? ((int64_t)p / m.block + 1) * m.block : L;
        const int end = e0 < L ? (int)e0 : L, lo = m.window && m.window < end ? end - m.window : 0;
        for (int x : {lo, end - 1, 0, m.sinks - 1}) {
          if (x < 0 || x >= end || !(x >= lo || x < m.sinks)) continue;
          const int kt = x / BK;
          if (!(kt < l.ns || (kt >= l.w0 && l.ns + (kt - l.w0) < l.n))) return 1;
        }
      }
    }
  }

  Plan plan{};
  std::vector<Item> items;
  run_warp([&](int lane) {
    Known k{};
    const Plan p = make_plan(j, ctas, k);
    if (lane == 0) plan = p;
  });
  if (plan.units != units || plan.items < 0 || (plan.C == 0 && plan.items != units)) return 2;
  if (plan.C > 0 && (plan.items > MAX_ITEMS || plan.C < MIN_PART || !j.cut)) return 3;
  items.resize(plan.items);
  run_warp([&](int lane) {
    Cursor cursor{};
    const Plan p = make_plan(j, ctas, cursor.k);
    if (p.C == 0 && j.s.n > 1 && j.s.n <= 32) order(cursor.k, j.s.n);
    for (int i = 0; i < p.items; ++i) {
      List l{};
      const Item x = make_item(j, p, i, cursor, l);
      if (lane == 0) items[i] = x;
    }
  });
  // every unit's tiles once
  std::map<std::tuple<int, int, int>, std::map<int, std::pair<int, int>>> got;   // first tile -> (end, item)
  int parts = 0;
  for (int i = 0; i < plan.items; ++i) {
    const Item& x = items[i];
    if (!x.state) continue;
    const int t0 = x.r0 - row[x.b], t = t0 / (2 * j.TQ);
    if (t0 % (2 * j.TQ)) return 4;
    auto unit = tiles.find({x.b, x.h, t});
    if (unit == tiles.end()) return 5;
    if (x.i0 < 0 || x.i1 < x.i0 || x.i1 > unit->second) return 6;
    if (!got[{x.b, x.h, t}].emplace(x.i0, std::make_pair(x.i1, i)).second) return 7;
    parts += x.part >= 0;
  }
  if (parts > MAX_PARTS || got.size() != tiles.size()) return 8;
  for (auto& u : got) {
    int to = 0;
    for (auto& p : u.second) {
      if (p.first != to) return 9;
      to = p.second.first;
      if ((items[p.second.second].part >= 0) != (u.second.size() > 1)) return 10;
    }
    if (to != tiles[u.first]) return 11;                    // tiles that nobody attends to
  }
  // what is joined
  seen.uncut += plan.C == 0;
  if (plan.C == 0) return 0;
  seen.cut++;
  (plan.whole >= 0 ? seen.even : seen.uneven)++;
  seen.longer += plan.whole >= 0 && ends_even && longest > first;
  const int4 stored = stored_plan(plan);
  std::vector<Joined> list(units);
  run_warp([&](int lane) {
    for (int u = stored.z > 0 ? stored.z : 0; u < stored.x; ++u) {
      const Joined x = joined(j, stored, u);
      if (lane == 0) list[u] = x;
    }
  });
  size_t joins = 0;
  for (int u = stored.z > 0 ? stored.z : 0; u < stored.x; ++u) {
    const Joined& x = list[u];
    auto& unit = got[{x.u.b, x.u.h, x.u.t}];
    if ((x.n > 1 ? (size_t)x.n : 1) != unit.size()) return 12;   // partial results that nobody made, or joins
    if (x.n < 2) continue;
    if (x.n > MAX_CUT) return 13;
    int s = 0;
    for (auto& p : unit) {
      if (p.second.second != x.at + s * x.step) return 14;
      ++s;
    }
    joins += x.n;
  }
  if ((int)joins != parts || status[0]) return 15;
  return 0;
}

// Places of partial results that no item has stored: whatever is there instead, none outside the array.
static int check_slots() {
  std::vector<int> slot(MAX_ITEMS);
  const int junk[] = {-1, -7, MAX_PARTS, MAX_PARTS + 1, 2147483647, -2147483647 - 1, (int)0xff800000u, 0x7fc00000};
  for (int i = 0; i < MAX_ITEMS; ++i) slot[i] = i % 3 ? junk[i % 8] : i % MAX_PARTS;
  for (int i : {-2147483647 - 1, -1, MAX_ITEMS, MAX_ITEMS + 5, 2147483647})
    if (slot_of(slot.data(), i) != -1) return 1;
  for (int i = 0; i < MAX_ITEMS; ++i)
    if (slot_of(slot.data(), i) != (i % 3 ? -1 : i % MAX_PARTS)) return 2;
  return 0;
}

// Sequences that claim the same rows over and over: no work, an error.
static int check_claims() {
  for (int pairs : {1, 2, 40, 2048}) {
    const int rows = 1000;
    int32_t status[2] = {0, 0};
    std::vector<int32_t> row{0}, len, table(2 * pairs, 0);
    for (int i = 0; i < pairs; ++i) {
      row.push_back(rows);                                  // all rows, then back to the first one
      row.push_back(0);
      len.push_back(9000);
      len.push_back(9000);
    }
    Job j{};
    j.c.status = status; j.c.H = 2; j.c.d = 128; j.c.page_len = 16; j.c.page_log2 = 4; j.c.n_pages = 4;
    j.s = Seqs{table.data(), len.data(), row.data(), 2 * pairs, 1 << 20, rows};
    j.G = 1; j.TQ = BQ; j.max_rows = rows; j.cut = 1;
    Plan plan{};
    run_warp([&](int lane) {
      Known k{};
      const Plan p = make_plan(j, 152, k);
      if (lane == 0) plan = p;
    });
    if (status[0] == 0) return 1;
    if (pairs > 1 ? plan.units != 0 || plan.items != 0 : plan.units != 8) return 2;
  }
  return 0;
}

// What the query tiles of a sequence's units see: key tiles that some token sees a key of, that all see all of.
static int check_spans(int n, int L, int G, Mask m) {
  const int TQ = BQ / G;
  for (int t0 = 0; t0 < n; t0 += 2 * TQ) {
    const int k = n - t0 < 2 * TQ ? n - t0 : 2 * TQ, p0 = L - n + t0;
    const Span sp[2] = {span_of(m, k, p0, L, 0, TQ), span_of(m, k, p0, L, 1, TQ)};
    const Edges others[2] = {edges_of(sp[1], 0), edges_of(sp[0], 1)};
    for (int kt = 0; kt * BK < L; ++kt) {
      bool some[2] = {false, false}, every[2] = {true, true};
      for (int i = 0; i < k; ++i) {
        const int g = i / TQ, p = p0 + i;
        if (p < 0) {
          every[g] = false;
          continue;
        }
        const int64_t e0 = m.block ? ((int64_t)p / m.block + 1) * m.block : L;
        const int end = e0 < L ? (int)e0 : L, lo = m.window && m.window < end ? end - m.window : 0;
        const int a = kt * BK, z = a + BK, sk = m.window ? m.sinks : 0;
        some[g] |= a < end && (z > lo || a < sk);
        every[g] &= z <= end && (a >= lo || z <= sk);   // (by window and sinks together: counts as partly)
      }
      bool partly = false;
      for (int g = 0; g < 2; ++g) {
        if (some[g] && !active(sp[g], kt)) return 1;
        if (active(sp[g], kt) && all_seen(sp[g], kt) && !every[g]) return 2;
        partly |= active(sp[g], kt) && !all_seen(sp[g], kt);
      }
      for (int g = 0; g < 2; ++g)                       // both treat a tile as one does
        if (active(sp[g], kt) && (!all_seen(sp[g], kt) || in(others[g], kt)) != partly) return 3;
    }
  }
  return 0;
}

static Mask mask(int window, int sinks, int block) { return Mask{1.f, window, sinks, block, inverse_of(block)}; }

int main(int argc, char** argv) {
  if (argc == 1) return check_slots();
  if (argc == 2) return check_claims();
  if (argc == 4) {
    std::mt19937 g(atoi(argv[1]));
    auto upto = [&](int lo, int hi) { return lo + (int)(g() % (unsigned)(hi - lo + 1)); };
    for (int i = 0; i < atoi(argv[2]); ++i) {
      const int G = upto(1, 3) < 3 ? upto(1, 8) : 1, n = upto(1, 700), L = upto(0, 9) ? n + upto(0, 1500) : upto(0, n);
      const int window = upto(0, 4) ? upto(1, 1500) : 0, sinks = upto(0, 2) ? upto(0, 1500) : 0;
      const int kind = upto(0, 4), block = kind == 0 ? 0 : kind < 3 ? 1 : upto(2, 600);
      if (int e = check_spans(n, L, G, mask(window, sinks, block)))
        return printf("case %d: %d (%d tokens of %d, groups of %d, window %d, sinks %d, block %d)\n", i, e, n, L, G, window, sinks, block), 1;
    }
    return 0;
  }
  Seen seen{};
  // one unit in the middle straddles two blocks and sees more than the first and the last one
  if (int e = check({{824, 11264}}, 8, 1, 152, mask(2048, 0, 512), seen)) return printf("straddling unit: %d\n", e), 1;
  if (seen.longer != 1) return printf("straddling unit: not cut as units of one length\n"), 1;
  std::mt19937 g(atoi(argv[1]));
  auto pick = [&](std::initializer_list<int> v) { return v.begin()[g() % v.size()]; };
  auto upto = [&](int lo, int hi) { return lo + (int)(g() % (unsigned)(hi - lo + 1)); };
  for (int i = 0; i < atoi(argv[2]); ++i) {
    const bool windows = i % 2;                             // long windows over a few equal sequences: mostly cut
    const int G = windows ? pick({1, 1, 3, 5, 7}) : pick({1, 1, 2, 3, 4, 5, 7, 8, 16, 33, 128});
    const int H = windows ? pick({1, 2, 8, 12}) : pick({1, 2, 3, 8, 12, 40});
    const int n_seq = windows ? pick({1, 1, 2}) : pick({1, 1, 2, 3, 5, 40, 66}), top = n_seq > 5 ? 60 : 1200;
    const int past = windows ? 30000 : pick({100, 3000, 12000, 30000});
    std::vector<std::pair<int, int>> s;
    const int same = upto(1, top), far = upto(0, past), alike = windows || pick({0, 1});
    for (int b = 0; b < n_seq; ++b) {
      const int n = alike ? same : upto(0, top), odd = upto(0, 19);
      s.push_back({n, odd == 0 ? upto(0, n) : n + (alike ? far : upto(0, past))});
    }
    const int window = windows ? upto(1000, 6000) : pick({0, upto(1, 300), upto(500, 12000)});
    const int block = windows ? pick({1, 512, upto(100, 1000)}) : pick({0, 1, 1, 512, upto(2, 600), 4680});
    if (int e = check(s, H, G, pick({152, 152, 148, 132, 5}), mask(window, pick({0, 0, 4, 700, 2147483647}), block), seen))
      return printf("case %d: %d (%d heads, groups of %d, %d sequences, first %d of %d, window %d, block %d)\n", i, e, H, G,
                    n_seq, s[0].first, s[0].second, window, block), 1;
  }
  printf("%d %d %d %d\n", seen.uncut, seen.even, seen.longer, seen.uneven);
  return 0;
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    try:
        nvcc = B.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cu").write_text(SRC)
    subprocess.check_call([nvcc, *B.ARCH, "-O2", "-U_FORTIFY_SOURCE", "-std=c++17", "-I", B.ROOT + "/include", "-I", B.CSRC, str(d / "plan.cu"), "-o",
                           str(d / "plan")])
    return str(d / "plan")


@pytest.mark.parametrize("seed", range(4))
def test_items_make_up_the_units(walk, seed):
    r = subprocess.run([walk, str(seed), "300"], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    uncut, even, longer, uneven = map(int, r.stdout.split())
    assert uncut > 20 and even > 20 and longer > 2 and uneven > 20   # plans of every kind were walked


def test_places_that_no_item_stored(walk):
    """After a CTA has given up waiting, the joining kernel finds anything in the places of partial results."""
    assert subprocess.run([walk], timeout=60).returncode == 0


def test_rows_claimed_more_than_once(walk):
    """A row_start that goes back and forth gives every other sequence all rows: the call's work stays that of its rows."""
    assert subprocess.run([walk, "claims"], timeout=60).returncode == 0


@pytest.mark.parametrize("seed", range(2))
def test_tiles_that_are_seen(walk, seed):
    """Which key tiles a query tile sees, in part and whole, and that both query tiles of a unit agree on those in which
    some row's view ends."""
    r = subprocess.run([walk, str(seed), "3000", "spans"], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
