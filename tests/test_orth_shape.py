"""The shapes that Newton-Schulz products run in (csrc/orth_shape.h, plain C++), compiled here and
checked over many sizes and devices: what the kernel takes for granted holds whatever the
estimates say."""
import os
import shutil
import subprocess

import pytest

import paper_2102_08550_gb300 as P
from tests.test_server_update_refusals import orth, refused

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2102_08550_gb300", "csrc")

DRIVER = r"""
#include <cstdio>
#include <initializer_list>
#include "orth_shape.h"
using namespace oscars;
static long seen = 0, split = 0, bad = 0;
static void check(const NsProduct& p, const NsRoom& r) {
  const NsShape s = ns_shape(p, r);
  ++seen;
  split += s.split > 1;
  const int nk = (p.K + kNsK - 1) / kNsK;
  const long long covered_m = 128LL * s.mt, covered_n = 1LL * s.BN * s.nt;
  const long long tiles = p.sym && !s.full ? s.nt * (s.nt + 1LL) / 2 : 1LL * (s.mt / s.cl) * s.nt;
  bool ok = (s.cl == 1 || s.cl == 2) && s.BN % (64 * s.cl) == 0 && s.BN >= 64 && s.BN <= kNsMaxBN && s.mt % s.cl == 0;
  ok = ok && covered_m >= p.M && covered_n >= p.N && covered_m - p.M < 128 * s.cl && covered_n - p.N < s.BN;
  ok = ok && s.units == tiles * p.batch && (!p.sym || s.BN == 128 * s.cl) && (!s.full || p.sym);
  // K in parts: each has a K-block, a CTA's columns are whole groups of 32, the clusters run at once
  ok = ok && (s.split == 1 || s.split == 2 || s.split == 4) && nk >= s.split && (s.split == 1 || (s.cl == 1 && s.BN % s.split == 0 && s.BN / s.split % 32 == 0));
  ok = ok && (s.split == 1 || s.units <= (s.split == 2 ? r.pairs : r.fours));
  // shared memory: staging, the ring, a split tile's sums, barriers
  const long long smem = 1024LL + kNsStgBytes + 1LL * s.stages * ns_stage_bytes(p, s.BN, s.cl) + (s.split > 1 ? 128LL * s.BN * 4 : 0) + kNsBarBytes;
  ok = ok && s.stages >= 2 && s.stages <= kNsMaxStages && smem <= kNsSmem;
  if (!ok && bad++ < 10)
    std::printf("sym %d batch %d %d x %d x %d halves %d %d: cl %d BN %d split %d stages %d\n", p.sym, p.batch, p.M, p.N, p.K, p.a_halves, p.b_halves, s.cl, s.BN, s.split, s.stages);
}
int main() {
  const int sides[] = {1, 10, 64, 65, 128, 129, 130, 192, 200, 256, 257, 300, 333, 384, 385, 500, 512, 640, 700, 784, 1000, 1001, 1024, 1400, 1537, 2048, 2500, 4096, 8192, 65536};
  const int halves[][2] = {{1, 1}, {1, 2}, {2, 1}, {2, 2}};
  const NsRoom rooms[] = {{152, 76, 36}, {152, 76, 38}, {148, 74, 33}, {132, 66, 30}, {16, 8, 4}, {1, 1, 1}, {1000, 500, 250}};
  for (const NsRoom& r : rooms)
    for (int m : sides)
      for (int n : sides)
        for (int batch : {1, 2, 3, 7, 16, 64, 1000})
          for (const auto& h : halves) {
            const int s = m < n ? m : n, l = m < n ? n : m;
            check({true, batch, s, s, l, h[0], h[0]}, r);
            check({true, batch, s, s, s, h[0], h[0]}, r);
            check({false, batch, m, n, s, h[0], h[1]}, r);
          }
  for (int bn = 64; bn <= kNsMaxBN; bn += 64)
    for (int sp : {1, 2, 4})
      if (ns_split_fits(bn, sp) != (bn / sp % 32 == 0 && bn % sp == 0)) { ++bad; std::printf("ns_split_fits(%d, %d)\n", bn, sp); }
  std::printf("seen %ld split %ld bad %ld fits(192, 4) %d\n", seen, split, bad, ns_split_fits(192, 4));
  return bad != 0;
}
"""


def test_every_shape_is_one_the_kernel_can_run(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "shapes.cpp", tmp_path / "shapes"
    src.write_text(DRIVER)
    subprocess.run([cxx, "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
    assert "fits(192, 4) 0" in r.stdout and "split 0 " not in r.stdout, r.stdout


@pytest.mark.parametrize("batch,rows,cols", [(65535, 65536, 65536), (65535, 8200, 8200), (65535, 1100, 65536), (16384, 65536, 4096)])
def test_more_tiles_than_are_counted(oscars_lib, batch, rows, cols):
    """The numbers of such tiles leave 32 bits; no workspace of that size exists, but the call only sees what it is told."""
    for dtype in (P.F32, P.BF16):
        refused(P.oscars_orthogonalize_workspace, batch, rows, cols, dtype)
        refused(orth, batch=batch, rows=rows, cols=cols, ldg=cols, ldo=cols, bsg=rows * cols, bso=rows * cols, dtype=dtype, n=1 << 62)


def test_the_largest_that_are(oscars_lib):
    for batch, rows, cols in [(1, 65536, 65536), (512, 65536, 65536), (65535, 1, 65536), (65535, 65536, 1), (65535, 1000, 4000)]:
        assert P.oscars_orthogonalize_workspace(batch, rows, cols, P.F32) > 0
