"""Arrays that lie between each other's elements: the library's own check, built on the
host, against the elements themselves, and what the C ABI refuses."""
import os
import shutil
import subprocess

import pytest

from paper_2609_16915_amd import build as B
from test_decode_cpu import ALIAS, AT, L, keep, read, write  # noqa: F401

PROGRAM = r"""
#include <cstdio>
#include <random>
#include <vector>
#include "clear_checks.hpp"
using namespace rosetta;
std::mt19937 rng(5);
size_t pick(size_t lo, size_t hi) { return lo + rng() % (hi - lo + 1); }
// An array of up to three levels at `at`, and the bytes that are its own.
Array make(size_t at, size_t elem, const Runs *like, std::vector<char> *own) {
  Runs r[3];
  size_t len = pick(1, 4);
  for (int i = 2; i >= 0; --i) {
    r[i].n = pick(1, i ? 3 : 4);
    r[i].len = len;
    r[i].stride = len + (rng() % 2 ? pick(0, 9) : 0);
    if (like && rng() % 8) r[i].stride = like[i].stride * 4 / elem < len ? len : like[i].stride * 4 / elem;
    len = (r[i].n - 1) * r[i].stride + len;
  }
  Array a{"", (void *)at, r[0].n, r[0].len, r[0].stride, elem, true, {r[1], r[2]}};
  if (rng() % 4 == 0) {  // all of a row its own
    a.inner[0] = a.inner[1] = Runs{0, 0, 0};
    r[1] = r[2] = Runs{1, r[0].len, r[0].len};
  }
  own->assign(4096, 0);
  for (size_t i = 0; i < r[0].n; ++i)
    for (size_t j = 0; j < r[1].n; ++j)
      for (size_t k = 0; k < r[2].n; ++k)
        for (size_t l = 0; l < r[2].len * elem; ++l)
          (*own)[at + (i * r[0].stride + j * r[1].stride + k * r[2].stride) * elem + l] = 1;
  return a;
}
int main() {
  long missed = 0, refused = 0, apart = 0, meet = 0, exact = 0;
  for (int n = 0; n < 400000; ++n) {
    std::vector<char> x, y;
    const bool same = rng() % 2;
    const Array a = make(pick(900, 1300), 4, nullptr, &x);
    const Runs like[3] = {{0, 0, a.stride}, a.inner[0], a.inner[1]};
    const Array b = make(pick(900, 1300), rng() % 2 ? 4 : 1, a.inner[0].n ? like : nullptr, &y);
    bool shares = false;
    for (size_t i = 0; i < x.size(); ++i) shares |= x[i] && y[i];
    const bool said = overlap(a, b);
    if (said != overlap(b, a)) ++missed;
    if (shares && !said) ++missed;
    if (!shares && said) {
      ++refused;
      // exact where every level of both is there, and as far apart
      bool alike = a.inner[0].n && b.inner[0].n;
      for (int i = 0; i < 3; ++i)
        alike &= a.level(i).n > 1 && b.level(i).n > 1 && a.level(i).stride * a.elem == b.level(i).stride * b.elem;
      if (alike) ++exact;
    }
    if (!shares && !said) ++apart;
    if (shares) ++meet;
  }
  std::printf("%ld missed, %ld not exact; %ld meet, %ld apart, %ld refused\n", missed, exact, meet, apart, refused);
  return missed || exact || meet < 10000 || apart < 10000;
}
"""


@pytest.mark.skipif(not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")),
                    reason="needs hipcc")
def test_overlap_is_that_of_the_elements(tmp_path):
    src, exe = tmp_path / "overlap.hip", tmp_path / "overlap"
    src.write_text(PROGRAM)
    subprocess.run([B.hipcc(), "-O1", "-std=c++17", f"--offload-arch={B.ARCH}", f"-I{B.INCLUDE}",
                    f"-I{B.CSRC}", str(src), "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout


# keys and values in turn within a page: [pages][page][2][heads][dim], [pages][heads][2][page][dim]
PLACES = dict(page_stride=4096, head_stride=64, place_stride=256)
HEADS = dict(page_stride=4096, head_stride=2048, place_stride=64)


@pytest.mark.parametrize("call", [write, keep])
@pytest.mark.parametrize("kw", [
    dict(PLACES, v=AT[0] + 112), dict(PLACES, v=AT[0] + 64), dict(PLACES, v=AT[0] + 192),
    dict(PLACES, v=AT[0] + 256 + 64), dict(PLACES, v=AT[0] + 16 * 256 - 64),
    dict(HEADS, v=AT[0] + 1008), dict(HEADS, v=AT[0] + 1040), dict(HEADS, v=AT[0] + 64),
    dict(HEADS, v=AT[0] + 4096 + 1008),
    dict(scale_head_stride=32, scale_page_stride=64, v_scale=AT[2] + 4 * 15),
    dict(scale_head_stride=32, scale_page_stride=64, v_scale=AT[2] + 4 * 17),
])
def test_parts_that_meet(L, call, kw):  # noqa: F811
    assert call(L, **kw) == ALIAS


def test_outputs_that_meet(L):  # noqa: F811
    # [rows][heads][2][dim], not far enough apart
    for by in (0, 63, 65, 127 + 256):
        assert read(L, krs=256, khs=128, vrs=256, vhs=128, vp=AT[7] + 2 * by) == ALIAS
