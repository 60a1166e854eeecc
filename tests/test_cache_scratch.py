"""The calls' numbers in scratch that nobody clears, on the CPU: what one attention kernel leaves in shared
memory, and what a program's own tensors leave in it, is no count of the other's."""
import subprocess

import pytest

from paper_2608_27922_gb300 import build as B

SRC = r"""
#include "cache_internal.h"
#include <vector>
using namespace dkv::cache;
static bool chunk_takes(uint64_t word, uint64_t call) { return (word >> CHUNK_COUNT_BITS) == chunk_number(call); }
static bool rows_takes(uint64_t word, uint64_t call) { return (word >> ROWS_COUNT_BITS) == rows_number(call); }
static const uint64_t LAST_CHUNK = (NUMBER_TOPS << (48 - CHUNK_COUNT_BITS)) - 1, LAST_ROWS = (NUMBER_TOPS << (48 - ROWS_COUNT_BITS)) - 1;
// Whether some call of a kernel takes the word for a count.
static bool some_chunk(uint64_t word) {
  return (word >> CHUNK_COUNT_BITS) >= chunk_number(0) && (word >> CHUNK_COUNT_BITS) <= chunk_number(LAST_CHUNK);
}
static bool some_rows(uint64_t word) {
  return (word >> ROWS_COUNT_BITS) >= rows_number(0) && (word >> ROWS_COUNT_BITS) <= rows_number(LAST_ROWS);
}
int main() {
  std::vector<uint64_t> calls;
  for (uint64_t n = 0; n < 70000; ++n) calls.push_back(n);
  for (uint64_t n = 1; n < (1ull << 40); n = n * 3 / 2 + 1) for (uint64_t k : {n - 1, n, n + 1}) calls.push_back(k);
  for (uint64_t k : {LAST_CHUNK - 1, LAST_CHUNK, LAST_CHUNK + 1, LAST_ROWS - 1, LAST_ROWS, LAST_ROWS + 1}) calls.push_back(k);
  for (uint64_t n : calls) {
    // a call's own counts are its own, from none to the most, and nobody else's
    for (uint64_t count : {0ull, 1ull, 151ull, (1ull << ROWS_COUNT_BITS) - 1}) {
      const uint64_t w = rows_number(n) << ROWS_COUNT_BITS | count;
      if (!rows_takes(w, n) || rows_takes(w, n + 1) || some_chunk(w) || !some_rows(w)) return 1;
    }
    for (uint64_t count : {0ull, 1ull, 151ull, (1ull << CHUNK_COUNT_BITS) - 1}) {
      const uint64_t w = chunk_number(n) << CHUNK_COUNT_BITS | count;
      if (!chunk_takes(w, n) || chunk_takes(w, n + 1) || some_rows(w) || !some_chunk(w)) return 2;
    }
  }
  // all words of either kernel are apart: numbers ascend up to the last one
  if (chunk_number(LAST_CHUNK) >> (48 - CHUNK_COUNT_BITS) != 0xffbe || rows_number(LAST_ROWS) >> (48 - ROWS_COUNT_BITS) != 0x7fbe) return 3;
  // what programs leave: infinities and NaNs of 16, 32 and 64 bits beside anything, small integers, bytes all alike
  const uint64_t low[] = {0, 1, 0xff80, 0x7f80, 0x3f80, 0xffff, 0xdeadbeef, 0xff800000, 0x7fc00000, 0xffffffff};
  const uint64_t high16[] = {0xff80, 0x7f80, 0xff7f, 0x7f7f, 0x7fc0, 0xffc0, 0x7fff, 0xffff, 0xfc00, 0x7c00, 0x7e00, 0xfe00, 0x7ff0, 0xfff0, 0x7ff8, 0xfff8};
  for (uint64_t h : high16)
    for (uint64_t m : {0ull, 1ull, 0xff80ull, 0x3c00ull, 0xffffull, (unsigned long long)h})
      for (uint64_t l : low) {
        const uint64_t w = h << 48 | m << 32 | l;
        if (some_chunk(w) || some_rows(w)) return 4;
      }
  for (int64_t i = -(1 << 22); i <= (1 << 22); ++i)
    for (uint64_t w : {(uint64_t)i, (uint64_t)(uint32_t)i << 32 | (uint32_t)i, (uint64_t)(uint32_t)i << 32})
      if (some_chunk(w) || some_rows(w)) return 5;
  for (uint64_t b = 0; b < 256; ++b) {
    const uint64_t w = b * 0x0101010101010101ull;
    if (some_chunk(w) || some_rows(w)) return 6;
  }
  return 0;
}
"""


def test_numbers_stay_apart(tmp_path):
    try:
        nvcc = B.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    src, exe = tmp_path / "numbers.cu", tmp_path / "numbers"
    src.write_text(SRC)
    subprocess.check_call([nvcc, *B.ARCH, "-O2", "-std=c++17", "-I", B.ROOT + "/include", "-I", B.CSRC, str(src), "-o", str(exe)])
    assert subprocess.run([str(exe)], timeout=120).returncode == 0
