"""Arithmetic of the paged memory that host and device share, compiled for the
host from the library's own header: the dealing of equal tiles to workgroups and
the pages of tokens, at every length that the header allows."""
import ctypes
import os
import subprocess

import pytest

from paper_2606_10671_amd import build

SOURCE = r"""
#include "paged_internal.h"
using namespace fademem;
extern "C" {
int page(int P, int key) {
  PagedView v;
  set_page_division(&v, P);
  return page_of(v, key);
}
int cut(int len, int parts, int j) { return even_cut(len, parts, j); }
// The segments of a plan of `total` tiles of `units` units, workgroup by workgroup: (task, u0, u1, slot) each.
// Returns their number, or -1 beyond `most`.
int segments(int total, int units, int kind, int most, int* out, int* plan) {
  const TileShape shapes[3] = {kPagedWideBf16, kPagedWideBf16D64, kPagedWideF32};
  EvenPlan e;
  const int groups = even_plan(total, units, shapes[kind], &e);
  plan[0] = groups, plan[1] = e.heads, plan[2] = e.rem, plan[3] = e.tail_len, plan[4] = shapes[kind].groups;
  int n = 0;
  for (int g = 0; g < groups; ++g)
    for (int k = 0, m = even_segments(e, g); k < m; ++k, ++n) {
      if (n >= most) return -1;
      const EvenSegment s = even_segment(e, g, k);
      out[4 * n] = s.task, out[4 * n + 1] = s.u0, out[4 * n + 2] = s.u1, out[4 * n + 3] = s.slot;
    }
  return n;
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_host")
    src, out = d / "host.cpp", d / "host.so"
    src.write_text(SOURCE)
    rocm = os.path.dirname(os.path.dirname(build.HIPCC))
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"),
                    "-I", os.path.join(build.ROOT, "include"), "-I", os.path.join(build.PKG, "csrc"), str(src), "-o", str(out)],
                   check=True, timeout=300)
    return ctypes.CDLL(str(out))


@pytest.mark.parametrize("P", [1, 2, 3, 5, 7, 16, 31, 33, 48, 63, 64, 100, 127, 129, 300, 1000, 4680, 32767, 32769, 65535, 65536])
def test_pages_of_tokens(lib, P):
    """Around every kind of multiple up to the longest sequence, whose end (2^30) is asked for too."""
    keys = {0, 1, 2, (1 << 30) - 1, 1 << 30}
    for base in (0, 1 << 10, 1 << 20, 1 << 24, 1 << 28, 1 << 29, (1 << 30) - 3 * P):
        for k in range(4):
            m = (base // P + k) * P
            keys |= {m - 1, m, m + 1, m + P // 2}
    for key in sorted(k for k in keys if 0 <= k <= 1 << 30):
        assert lib.page(P, key) == key // P, key


UNITS = [1, 5, 6, 7, 74, 383, 9143, (1 << 22) - 1, 1 << 22, (1 << 22) + 1, (1 << 23) + 5, (1 << 24) - 1, (1 << 24) + 1]


@pytest.mark.parametrize("units", UNITS)
def test_cuts_are_exact(lib, units):
    for parts in (1, 2, 3, 85, 127, 170, 255, 256, 511, 512):
        assert [lib.cut(units, parts, j) for j in range(parts + 1)] == [j * units // parts for j in range(parts + 1)]


@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("units", UNITS)
def test_every_unit_of_every_tile_is_dealt_once(lib, units, kind):
    most = 1 << 14
    out, plan = (ctypes.c_int * (4 * most))(), (ctypes.c_int * 5)()
    for total in (1, 2, 3, 7, 100, 129, 228, 255, 256, 257, 300, 511, 512, 513, 800, 1720):
        n = lib.segments(total, units, kind, most, out, plan)
        assert 0 < n and plan[0] <= plan[4]
        parts, slots = {}, []
        for i in range(n):
            task, u0, u1, slot = out[4 * i: 4 * i + 4]
            assert 0 <= task < total and 0 <= u0 < u1 <= units
            parts.setdefault(task, []).append((u0, u1, slot))
            if slot >= 0:
                slots.append(slot)
        assert sorted(parts) == list(range(total))
        for p in parts.values():
            p.sort()
            assert p[0][0] == 0 and p[-1][1] == units and all(a[1] == b[0] for a, b in zip(p, p[1:]))
            assert (len(p) > 1) == (p[0][2] >= 0)  # shared tiles leave their parts in slots, the others do not
        assert len(set(slots)) == len(slots) and all(s < 2 * plan[4] for s in slots)
