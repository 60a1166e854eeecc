"""Refusals and structures of the calls on pages, norms and chosen pages, on the CPU; slots of tiles."""
import ctypes
import os
import random
import shutil
import subprocess
import tempfile

import pytest

from paper_2608_27922_gb300 import build as B


def _lib():
    from paper_2608_27922_gb300 import dkv
    try:
        return dkv, dkv.lib()
    except RuntimeError:
        B.build()
        return dkv, dkv.lib()


def test_refusals_before_any_cuda_call():
    dkv, L = _lib()
    mem = (ctypes.c_char * 4096)()
    at = (ctypes.addressof(mem) + 255) & ~255
    ARG, SHAPE = 1, 2
    pairs = lambda *p: (ctypes.c_int32 * 4)(*p)

    def how(**kw):
        f = dict(theta=at, q_weight=None, k_weight=None, eps=1e-6, norm=1, layout=0, n_axes=1, axis_pairs=pairs(64))
        f.update(kw)
        return ctypes.byref(dkv.dkv_norm_rope_t(**f))

    def rope(h, d=128, coord=at, rows=4, Hq=2, Q=at, q=(512, 128), Qo=at, qo=(512, 128), Hk=0):
        return L.dkv_norm_rope(d, h, coord, rows, Hq, Q, *q, Qo, *qo, Hk, None, 0, 0, None, 0, 0, None)
    for wrong in (dict(theta=None), dict(theta=at + 2), dict(q_weight=at + 1), dict(k_weight=at + 2), dict(eps=0.0), dict(eps=-1.0),
                  dict(eps=float("nan")), dict(norm=2), dict(layout=2), dict(layout=-1), dict(n_axes=0), dict(n_axes=5),
                  dict(axis_pairs=pairs(63)), dict(axis_pairs=pairs(65)), dict(n_axes=2, axis_pairs=pairs(65, -1)),
                  dict(n_axes=2, axis_pairs=pairs(2 ** 31 - 1, 2 ** 31 - 1))):
        assert rope(how(**wrong)) == ARG, wrong
    assert rope(None) == ARG
    for kw in (dict(coord=None), dict(Q=None), dict(Qo=None), dict(Q=at + 8), dict(q=(512, 129)), dict(qo=(512, 120)),
               dict(qo=(64, 128)), dict(q=(0, 128)), dict(qo=(1024, 128)), dict(q=(-512, 128))):
        assert rope(how(), **kw) == ARG, kw
    for kw in (dict(d=96), dict(rows=0), dict(rows=(1 << 20) + 1), dict(Hq=0), dict(Hq=-1), dict(Hq=4097), dict(Hk=4097)):
        assert rope(how(), **kw) == SHAPE, kw
    # nothing without a handle
    N = None
    assert L.dkv_cache_write_norm_rope(N, N, N, N, 1, 0, N, 0, 0, N, 0, 0, N, 0, 0, N, 0, 0, N) == ARG
    assert L.dkv_cache_fork(N, N, N, N, N, N) == ARG
    assert L.dkv_cache_extend_scratch_size(N, 1) == 0 and L.dkv_cache_compact_scratch_size(N, 1) == 0
    assert L.dkv_cache_extend(N, N, N, N, N, 0, N) == ARG
    assert L.dkv_cache_release(N, N, N, N, N, N) == ARG
    assert L.dkv_cache_compact(N, N, N, N, 0, N, N, N, 0, N) == ARG
    assert L.dkv_cache_summarise(N, N, N, N, N) == ARG
    assert L.dkv_cache_choose(N, N, N, N, 1, 1, 0, 0, N, N, N) == ARG
    assert L.dkv_cache_attend_chosen(N, N, N, 1, 1, 0, 0, N, 0, 0, N, N, N) == ARG


def test_struct_layouts():
    """The binding's structures against the header's, as a C compiler sees it."""
    dkv, _ = _lib()
    if not shutil.which("gcc"):
        pytest.skip("gcc unavailable")
    names = ("dkv_norm_rope_t", "dkv_cache_table_t", "dkv_cache_summaries_t", "dkv_cache_choose_t", "dkv_cache_chosen_t")
    lines, want = [], []
    for n in names:
        t = getattr(dkv, n)
        lines.append(f'printf("%zu ", sizeof({n}));')
        want.append(ctypes.sizeof(t))
        for f, *_ in t._fields_:
            lines.append(f'printf("%zu ", offsetof({n}, {f}));')
            want.append(getattr(t, f).offset)
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "p.c"), os.path.join(d, "p")
        open(c, "w").write('#include <stdio.h>\n#include <stddef.h>\n#include "dkv.h"\nint main(void) {' + "".join(lines) + "return 0;}")
        subprocess.check_call(["gcc", "-I", B.ROOT + "/include", c, "-o", exe])
        assert [int(x) for x in subprocess.check_output([exe]).split()] == want


SRC = r"""
#include "cache_internal.h"
#include <set>
#include <vector>
using namespace dkv::cache;
int main() {
  // every tile of every sequence has a slot of its own, below rows / tile + n, and the search finds its sequence
  unsigned r = 1;
  auto rnd = [&](int m) { r = r * 1664525u + 1013904223u; return (int)((r >> 8) % (unsigned)m); };
  for (int round = 0; round < 4000; ++round) {
    const int n = 1 + rnd(7), tile = 1 + rnd(round % 3 ? 9 : 128);
    std::vector<int32_t> start{rnd(3)};
    for (int b = 0; b < n; ++b) start.push_back(start.back() + (rnd(4) ? rnd(40) : 0));
    const int rows = start.back() + rnd(5) + (start.back() == 0);
    Seqs s{nullptr, nullptr, start.data(), n, 1, rows};
    std::set<int> seen;
    for (int b = 0; b < n; ++b)
      for (int i = 0; i < start[b + 1] - start[b]; i += tile) {
        const int slot = first_slot(s, tile, b) + i / tile;
        if (slot < 0 || slot >= rows / tile + n || !seen.insert(slot).second || seq_of_slot(s, tile, slot) != b) return 1;
      }
  }
  // row starts that contradict themselves: the search stays inside
  const int edges[] = {-2147483647 - 1, -1, 0, 5, 40, 2147483647};
  for (int a : edges) for (int b : edges) for (int c : edges) for (int slot : {0, 1, 41, 1 << 20}) {
    const int32_t start[] = {a, b, c};
    Seqs s{nullptr, nullptr, start, 2, 1, 40};
    const int x = seq_of_slot(s, 1, slot);
    if (x < 0 || x >= 2) return 2;
  }
  return 0;
}
"""


def test_slots_of_tiles(tmp_path):
    try:
        nvcc = B.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    src, exe = tmp_path / "slots.cu", tmp_path / "slots"
    src.write_text(SRC)
    subprocess.check_call([nvcc, *B.ARCH, "-std=c++17", "-I", B.ROOT + "/include", "-I", B.CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)]).returncode == 0


SEARCH = r"""
#include "cache_internal.h"
#include <vector>
using namespace dkv::cache;
int main() {
  unsigned r = 3;
  auto rnd = [&](int m) { r = r * 1664525u + 1013904223u; return (int)((r >> 8) % (unsigned)m); };
  for (int n : {1, 2, 31, 32, 33, 63, 64, 65, 1000, 1023, 1024, 1025, 1056, 1057, 2049, 4095, 4096})
    for (int kind = 0; kind < 6; ++kind) {
      const int tile = kind == 0 ? 1 : 1 + rnd(kind < 3 ? 5 : 128);
      std::vector<int32_t> start{rnd(2)};
      for (int b = 0; b < n; ++b) start.push_back(start.back() + (kind == 5 ? 0 : rnd(3) ? rnd(kind == 1 ? 2 : 60) : 0));
      const int rows = start.back() + rnd(9) + 1;
      Seqs s{nullptr, nullptr, start.data(), n, 1, rows};
      for (int slot = 0; slot < rows / tile + n; slot += n > 64 ? 1 + rnd(4) : 1) {
        int want = 0;
        for (int lo = 0, hi = n; lo < hi;) {   // the first sequence whose slots begin behind this one
          const int mid = (lo + hi) / 2;
          if (start[mid] / tile + mid <= slot) want = mid, lo = mid + 1; else hi = mid;
        }
        if (seq_of_slot(s, tile, slot) != want) return 1;
      }
      // starts that contradict themselves
      const int edges[] = {-2147483647 - 1, -1, 0, 5, rows, 2147483647};
      for (auto& x : start) if (rnd(3) == 0) x = edges[rnd(6)];
      for (int i = 0; i < 200; ++i) {
        SlotSearch w{0, n};
        const int slot = rnd(3) ? rnd(rows / tile + n) : edges[rnd(6)];
        for (bool last = false; !last;) {
          last = w.step() == 1;
          uint32_t mask = 0;
          for (int lane = 0; lane < 32; ++lane) {
            const int b = w.at(lane);
            if (b < w.lo || b >= w.lo + w.n) return 2;
            mask |= (uint32_t)w.past(s, tile, slot, lane, start[b]) << lane;
          }
          const int lo = w.lo, before = w.n, k = w.narrow(mask);
          if (k < 0 || k > 31 || w.n < 1 || w.lo < lo || w.lo + w.n > lo + before || (last && w.n != 1)) return 3;
        }
        if (w.lo < 0 || w.lo >= n) return 4;
      }
    }
  return 0;
}
"""


def test_search_of_a_slot(tmp_path):
    """The search that the kernels' warps make, lane by lane: the definition's sequence, or one inside for starts that do not ascend."""
    try:
        nvcc = B.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    src, exe = tmp_path / "search.cu", tmp_path / "search"
    src.write_text(SEARCH)
    subprocess.check_call([nvcc, *B.ARCH, "-std=c++17", "-I", B.ROOT + "/include", "-I", B.CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)], timeout=120).returncode == 0


class _Bar:
    def __init__(self, n):
        self.n = self.c = n
        self.phase = 0

    def arrive(self):
        self.c -= 1
        if self.c == 0:
            self.c, self.phase = self.n, self.phase + 1

    def passed(self, parity):
        return (self.phase & 1) != parity


def _walk(n, N, seed):
    """The barriers of attention over chosen pages (k_chosen_tc.cu) on n key tiles with N tiles of K and of V, its roles taking
    turns at random, copies and products ending late: nobody is stuck, and nothing is read or overwritten too soon."""
    r = random.Random(seed)
    kf, ke, vf, ve = ([_Bar(1) for _ in range(N)] for _ in range(4))
    sf, pf, of = _Bar(1), [_Bar(4), _Bar(4)], _Bar(1)
    pipe, copies, arriving = [], [], []
    s_done, o_half, o_done, landed = [False] * n, [False] * n, [False] * n, {}

    def produce():
        order = [("k", 0)] if n else []
        for i in range(n):
            order += [("v", i)] + ([("k", i + 1)] if i + 1 < n else [])
        for what, i in order:
            while i >= N and not (ke if what == "k" else ve)[i % N].passed((i // N - 1) & 1):
                yield
            assert i < N or (s_done if what == "k" else o_done)[i - N]
            copies.append((what, i))
            yield

    def issue():
        for i in range(n):
            while not kf[i % N].passed((i // N) & 1):
                yield
            assert landed["k", i % N] == i
            pipe.append((s_done, i, [sf, ke[i % N]]))
            while not vf[i % N].passed((i // N) & 1):
                yield
            for half in (0, 1):
                while not pf[half].passed(i & 1):
                    yield
                assert landed["v", i % N] == i
                pipe.append((o_done if half else o_half, i, [ve[i % N]] + ([of] if i + 1 == n else []) if half else []))

    def soft():
        for i in range(n):
            while not sf.passed(i & 1):
                yield
            assert s_done[i] and (i == 0 or o_done[i - 1]) and not o_half[i]
            if r.random() < 0.3:                       # a tile that some row does not see whole
                while not vf[i % N].passed((i // N) & 1):
                    yield
                assert landed["v", i % N] == i and not o_done[i]
            for half in (0, 1):
                pf[half].arrive()
                yield
        while n and not of.passed(0):
            yield
        assert all(o_done)

    roles = [produce(), issue()] + [soft() for _ in range(4)]
    for step in range(100000):
        if not roles:
            return
        k = r.randrange(len(roles) + 3)
        if k < len(roles):
            try:
                next(roles[k])
            except StopIteration:
                roles.pop(k)
        elif k == len(roles) and pipe:
            done, i, bars = pipe.pop(0)
            done[i] = True
            r.shuffle(bars)
            if bars:
                arriving.append(bars)
        elif k == len(roles) + 1 and arriving:
            arriving[0].pop(0).arrive()
            if not arriving[0]:
                arriving.pop(0)
        elif k == len(roles) + 2 and copies:
            what, i = copies.pop(r.randrange(len(copies)))
            landed[what, i % N] = i
            (kf if what == "k" else vf)[i % N].arrive()
    raise AssertionError(("stuck", n, N, seed))


@pytest.mark.parametrize("N", [1, 2])
def test_barriers_of_attention_over_chosen_pages(N):
    for n in range(9):
        for seed in range(40):
            _walk(n, N, seed)
