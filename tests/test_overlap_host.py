"""Outputs that lie over inputs are refused; rows that lie between the other's are not."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2608_08340_gb300 import _lib
from paper_2608_08340_gb300 import build as lib_build

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2608_08340_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <random>
#include "overlap.h"
using oprag::Rows;
int main() {
  std::mt19937 g(1);
  auto pick = [&](int lo, int hi) { return static_cast<int64_t>(lo + g() % (hi - lo + 1)); };
  int found = 0;
  for (int i = 0; i < 400000; ++i) {
    Rows a{1000, pick(0, 6), pick(1, 9), 0}, b{static_cast<uintptr_t>(pick(900, 1100)), pick(0, 6), pick(1, 9), 0};
    a.stride = a.bytes + pick(0, 12);
    b.stride = i % 2 ? b.bytes + pick(0, 12) : a.stride;
    if (b.bytes > b.stride) b.bytes = b.stride;
    bool used[2000] = {}, meets = false;
    for (int64_t r = 0; r < a.rows; ++r)
      for (int64_t x = 0; x < a.bytes; ++x) used[a.at + r * a.stride + x] = true;
    for (int64_t r = 0; r < b.rows; ++r)
      for (int64_t x = 0; x < b.bytes; ++x) meets |= used[b.at + r * b.stride + x];
    if (oprag::overlap(a, b) != meets || oprag::overlap(b, a) != meets) {
      std::printf("%d: %d\n", i, meets);
      return 1;
    }
    found += meets;
  }
  return found > 50000 && found < 350000 ? 0 : 2;
}
"""


def test_the_rule_against_marked_bytes(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    (tmp_path / "overlap.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "overlap")
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC,
                    str(tmp_path / "overlap.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return _lib.load()


@pytest.fixture(scope="module")
def base():
    """An address on 256 bytes of memory that no call below reads."""
    b = ctypes.create_string_buffer(1 << 16)
    yield (ctypes.addressof(b) + 255) // 256 * 256
    del b


def _refused(lib, rc):
    assert rc == -1 and "overlap" in lib.oprag_last_error().decode(), lib.oprag_last_error()


def test_distillation_refuses_a_gradient_over_its_scores(lib, base):
    apart = base + (1 << 15)

    def call(z, stride, grad, grad_stride, q=4):
        return lib.oprag_distill(z, 0, stride, q, 32, apart, apart, 5, 1.0, None, apart, grad,
                                 grad_stride, None)

    _refused(lib, call(base, 32, base, 48))               # another stride
    _refused(lib, call(base, 48, base, 32))
    _refused(lib, call(base, 64, base + 16, 64))          # another offset
    _refused(lib, call(base + 16, 64, base, 64))
    _refused(lib, call(base, 40, base + 40 * 4 * 2, 40))  # two rows on
    _refused(lib, call(base, 32, base + 4, 32, q=1))


def test_the_lookup_refuses_an_output_over_its_table(lib, base):
    def call(table, stride, out, count=3):
        return lib.oprag_embed_lookup(table, 0, 10, 16, stride, base + (1 << 15), 0, count, 1.0,
                                      out, 0, None)

    _refused(lib, call(base, 16, base))
    _refused(lib, call(base, 16, base + 9 * 64))
    _refused(lib, call(base, 48, base + 64, count=3))     # across a gap and the next row
    _refused(lib, call(base + 64, 16, base))


def test_the_lookups_gradient_refuses_an_output_over_its_input(lib, base):
    apart, bytes_ = base + (1 << 15), ctypes.c_int64(0)
    assert lib.oprag_embed_lookup_grad_workspace(15, 4, 16, ctypes.byref(bytes_)) == 0

    def call(grad, ts, ks, out):
        return lib.oprag_embed_lookup_grad(grad, 0, 3, 5, 16, ts, ks, apart, 0, 4, 1.0, out, 0,
                                           apart, bytes_.value, None)

    _refused(lib, call(base, 80, 16, base))
    _refused(lib, call(base, 80, 16, base + 14 * 64))     # the last token
    _refused(lib, call(base, 16, 0, base + 2 * 64))       # a gradient per text
    _refused(lib, call(base + 3 * 64, 1600, 16, base))
    _refused(lib, call(base, 400, 16, base + 4 * (400 - 16)))
