"""The paged cache's index arithmetic and refusals on the CPU.

The device code's own helpers (cache_internal.h: a sequence's rows and length inside the
call's buffers, a position's row in the pool) are compiled for the host and walked over
arrays that contradict themselves; whatever those hold, nothing may leave its buffer.
"""
import ctypes
import subprocess

import pytest

from paper_2608_27922_gb300 import build as B

SRC = r"""
#include "cache_internal.h"
#include <cstdio>
#include <vector>
using namespace dkv::cache;
int main() {
  const int edges[] = {-2147483647 - 1, -9, -1, 0, 1, 5, 16, 17, 40, 41, 1 << 29, 2147483647};
  for (int log2 : {4, 8})
    for (int len : edges)
      for (int a : edges)
        for (int z : edges) {
          int32_t status[2] = {0, 0};
          Pool c{};
          c.status = status; c.H = 3; c.page_len = 1 << log2; c.page_log2 = log2; c.n_pages = 7;
          const int max_pages = 5, rows = 40;
          std::vector<int32_t> table = {0, 6, -1, 7, 2147483647, 3, 3, 3, 3, 3}, lens = {len, 3}, start = {a, z, z};
          Seqs s{table.data(), lens.data(), start.data(), 2, max_pages, rows};
          const Seq q = seq_at(c, s, 0);
          if (q.r0 < 0 || q.n < 0 || q.r0 + q.n > rows) return 1;
          if (q.len < 0 || q.len > max_pages * c.page_len) return 2;
          const bool good = a >= 0 && z >= a && z <= rows && len >= 0 && len <= max_pages * c.page_len;
          if (good != (status[0] == 0)) return 3;
          if (good && (q.r0 != a || q.n != z - a || q.len != len)) return 4;
          for (int row : {0, 1, 39}) {
            const int b = seq_of_row(s, row);
            if (b < 0 || b >= 2) return 5;
          }
          for (int pos = 0; pos < q.len; ++pos) {
            status[0] = 0;
            const int64_t at = pool_row(c, s, 0, 2, pos);
            const int page = table[pos >> log2];
            if ((at >= 0) != (page >= 0 && page < 7) || (at >= 0) != (status[0] == 0)) return 6;
            if (at >= 0 && at != (int64_t)(page * 3 + 2) * c.page_len + pos % c.page_len) return 7;
          }
        }
  // the mask, against its definition
  for (int block : {0, 1, 2, 3, 7, 16, 4680, 2147483646, 2147483647})
    for (int window : {0, 1, 5, 2147483647})
      for (int len : {1, 2, 17, 1 << 30})
        for (int p : {0, 1, 2, 6, 7, 15, 16, 4679, 4680, (1 << 30) - 2, (1 << 30) - 1}) {
          if (p >= len) continue;
          const Mask m{1.f, window, 0, block, inverse_of(block)};
          const int e = visible_end(m, p, len);
          const int64_t want = block == 0 ? len : ((int64_t)p / block + 1) * block;
          if (e != (want < len ? want : len)) return 8;
          const int f = window_first(m, e);
          if (f != (window == 0 || window >= e ? 0 : e - window)) return 9;
        }
  return 0;
}
"""


def test_indices_stay_inside(tmp_path):
    try:
        nvcc = B.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    src, exe = tmp_path / "index.cu", tmp_path / "index"
    src.write_text(SRC)
    subprocess.check_call([nvcc, *B.ARCH, "-std=c++17", "-I", B.ROOT + "/include", "-I", B.CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)]).returncode == 0


def test_refusals_before_any_cuda_call():
    from paper_2608_27922_gb300 import dkv
    try:
        L = dkv.lib()
    except RuntimeError:
        B.build()
        L = dkv.lib()
    h = ctypes.c_void_p()
    mem = (ctypes.c_char * 4096)()
    at = (ctypes.addressof(mem) + 255) & ~255
    bufs = lambda **kw: ctypes.byref(dkv.dkv_cache_buffers_t(**{**dict(k=at, v=at, k_scale=at, v_scale=at, status=at), **kw}))
    create = lambda H, d, page, n, fmt, b: L.dkv_cache_create(ctypes.byref(h), H, d, page, n, fmt, b)
    ARG, SHAPE = 1, 2
    assert create(2, 128, 16, 4, 0, None) == ARG
    assert create(2, 128, 16, 4, 2, bufs()) == ARG
    for H, d, page, n in ((0, 128, 16, 4), (4097, 128, 16, 4), (2, 96, 16, 4), (2, 128, 0, 4), (2, 128, 8, 4), (2, 128, 48, 4),
                          (2, 128, 512, 4), (2, 128, 16, 0), (2, 128, 16, -1), (2, 128, 16, (1 << 30) + 1)):
        assert create(H, d, page, n, 0, bufs()) == SHAPE
    for wrong in (dict(k=None), dict(v=None), dict(status=None), dict(k=at + 16), dict(v=at + 64), dict(status=at + 4)):
        assert create(2, 128, 16, 4, 0, bufs(**wrong)) == ARG
    for wrong in (dict(k_scale=None), dict(v_scale=None), dict(k_scale=at + 8)):
        assert create(2, 128, 16, 4, 1, bufs(**wrong)) == ARG
    assert h.value is None
    L.dkv_cache_destroy(None)
    assert L.dkv_cache_write(None, None, None, None, 1, 0, 0, 0, 0, None) == ARG
    assert L.dkv_cache_read(None, None, None, None, None, 1, 0, 0, 0, 0, None) == ARG
    assert L.dkv_cache_attend(None, None, None, 1, 1, 0, 0, None, 0, 0, None, None, 0, None) == ARG
    assert L.dkv_cache_attend_scratch_size(None, 1, 1, 1, 1) == 0
    assert L.dkv_cache_sync(None) == ARG


def test_struct_layouts():
    """The binding's structures against the header's, as a C compiler sees it."""
    import os
    import shutil
    import tempfile
    from paper_2608_27922_gb300 import dkv
    if not shutil.which("gcc"):
        pytest.skip("gcc unavailable")
    src = r'''
#include <stdio.h>
#include <stddef.h>
#include "dkv.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu\n", sizeof(dkv_cache_buffers_t), sizeof(dkv_cache_seqs_t), sizeof(dkv_cache_attend_t),
         offsetof(dkv_cache_buffers_t, status), offsetof(dkv_cache_seqs_t, n_seq), offsetof(dkv_cache_attend_t, max_rows));
  return 0;
}
'''
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "p.c"), os.path.join(d, "p")
        open(c, "w").write(src)
        subprocess.check_call(["gcc", "-I", B.ROOT + "/include", c, "-o", exe])
        got = [int(x) for x in subprocess.check_output([exe]).split()]
    b, s, a = dkv.dkv_cache_buffers_t, dkv.dkv_cache_seqs_t, dkv.dkv_cache_attend_t
    assert got == [ctypes.sizeof(b), ctypes.sizeof(s), ctypes.sizeof(a), b.status.offset, s.n_seq.offset, a.max_rows.offset]
