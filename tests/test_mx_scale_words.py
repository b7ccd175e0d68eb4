"""Rows of scales of no whole words are put together from the aligned words that hold them. The function that does it, taken from the
kernel's source and compiled for the host: every byte is the row's or zero, and no word is read that lies behind the array."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2604_23996_gb300.build import CSRC

HARNESS = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <vector>
using std::max;
using std::min;
#define __device__
#define __forceinline__ inline
static const uint8_t *lo, *hi;                   // the array
static long outside = 0;
static uint8_t shared[4096];
static uint32_t __ldg(const uint32_t* p) {
  const uint8_t* q = reinterpret_cast<const uint8_t*>(p);
  if (q < lo || q + 4 > hi) ++outside;
  uint32_t v;
  memcpy(&v, p, 4);
  return v;
}
static uint32_t __funnelshift_r(uint32_t a, uint32_t b, uint32_t s) {
  return static_cast<uint32_t>(((static_cast<uint64_t>(b) << 32) | a) >> (s & 31));
}
template <int n> void cp_async(uint32_t, const void*, int) {}
static void store(uint32_t dst, const uint32_t (&v)[4]) { memcpy(shared + dst, v, 16); }
FUNCTION
template <bool kTail>
static long wrong() {
  long bad = 0;
  outside = 0;
  for (int n = 1; n < 40; ++n)
    for (int R = 1; R < 140; R += R < 12 ? 1 : 13) {
      const int bytes = R * n;
      std::vector<uint8_t> memory(bytes + 64 + 16, 0xee);
      uint8_t* x = memory.data() + (16 - reinterpret_cast<uintptr_t>(memory.data()) % 16) % 16;
      for (int i = 0; i < bytes; ++i) x[i] = static_cast<uint8_t>(1 + i % 201);
      lo = x;
      hi = x + bytes;
      uint32_t tail = 0;
      for (int i = 0; i < bytes % 4; ++i) tail |= static_cast<uint32_t>(x[bytes - bytes % 4 + i]) << (8 * i);
      for (int r = 0; r < 32; ++r)
        for (int at = 0; at < n + 16; at += 16) {
          int there[4];
          for (int i = 0; i < 4; ++i) there[i] = r + 32 * i < R ? min(max(n - at, 0), 16) : 0;
          fetch_scales<0, kTail>(0u, x + static_cast<long long>(r) * n + at, 32ll * n, there, x, hi, tail);
          for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 16; ++j) bad += shared[1024 * i + j] != (j < there[i] ? x[(r + 32 * i) * n + at + j] : 0);
        }
    }
  return bad;
}
int main() {
  const long with_tail = wrong<true>(), out_tail = outside, without = wrong<false>(), out_without = outside;
  printf("%ld %ld %ld %ld\n", with_tail, out_tail, without, out_without);
}
"""


def test_no_word_behind_the_array_is_read(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    with open(os.path.join(CSRC, "expert_mx.cu")) as f:
        text = f.read()
    a = text.index("template <int kBytes, bool kTail, int kUnits>")
    function = text[a:text.index("\n}\n", a) + 3]
    function, n = re.subn(r'asm volatile\("st\.shared\.v4\.u32.*?: "memory"\);', "store(dst + 1024 * i, out);", function, flags=re.S)
    assert n == 1
    (tmp_path / "harness.cpp").write_text(HARNESS.replace("FUNCTION", function))
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wno-unknown-pragmas", "-o", tmp_path / "harness", tmp_path / "harness.cpp"], check=True)
    out = subprocess.run([tmp_path / "harness"], check=True, capture_output=True, text=True).stdout.split()
    wrong, outside, wrong_whole, outside_whole = map(int, out)
    assert wrong == 0 and outside == 0
    assert wrong_whole == 0 and outside_whole > 0       # whole words alone: the same bytes, and words behind the array
