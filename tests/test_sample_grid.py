"""The sampler's bins (csrc/sample_grid.h) in a host program: where logits lie that a row may
hold, down to -infinity, and those that the search for a border looks at, up to the largest
number.  A conversion of a number beyond an integer's range, which C++ leaves undefined, ends
the program."""

import shutil
import subprocess

import pytest

from paper_2608_13076_amd import build

PROGRAM = r"""
#include <cfloat>
#include <cstdio>
#define __device__
#define __forceinline__ inline
#include "sample_grid.h"
using namespace spade;

static int bad = 0, seen = 0, in_window = 0;

static void check(double inv, float m, float l) {
  const double inv_T = row_inv_T(inv, m);
  const Grid g(inv_T, m);
  const long double d = l == m ? 0.0L : ((long double)m - (long double)l) * (long double)inv_T;
  if (l <= m && m > -INFINITY) {  // a token of a row whose largest logit is m
    int step;
    float rest;
    const int j = g.place(l, step, rest);
    ++seen;
    bool ok = step >= 0 && step < kSteps;
    if (l > -INFINITY && d <= 40.0L) {
      // bins are 32 / 126 wide: a distance of d reaches the bin d / width below the top or the next one
      ++in_window;
      ok = ok && j >= (int)(d / kBin) - 1 && j <= (int)(d / kBin) + 2 && rest >= 0.f && rest <= 1.f;
    } else {
      ok = ok && j > kLastBin + 1;
    }
    if (!ok) {
      ++bad;
      printf("inv_T %g m %g l %g: bin %d step %d rest %g, distance %Lg\n", inv, m, l, j, step, rest, d);
    }
  }
  if (l >= -FLT_MAX && l <= FLT_MAX && m > -INFINITY)
    for (int bin = 0; bin <= kLastBin; bin += 42) {  // any finite number
      const bool in = g.reaches(l, bin);
      bool want = l >= m;
      if (l < m) {
        int step;
        float rest;
        want = d <= 40.0L && g.place(l, step, rest) <= bin;
      }
      if (in != want) {
        ++bad;
        printf("inv_T %g m %g l %g: reaches bin %d: %d\n", inv, m, l, bin, in);
      }
    }
}

int main() {
  const float x[] = {0.f, 1e-45f, 1e-30f, 1e-3f, 0.7f, 1.f, 1.0000001f, 3.f, 17.5f, 4096.f, 1e6f, 3e9f, 1.7e10f, 1e20f, 1e38f, FLT_MAX};
  // temperatures: infinite, the largest to the smallest number
  const double inv[] = {0.0, 1.0 / FLT_MAX, 1e-30, 1e-6, 0.02, 1.0, 1.4, 1000.0, 1e6, 1e12, 1e30, 1.0 / 1.4e-45};
  for (double i : inv)
    for (float a : x)
      for (int s = -1; s <= 1; s += 2) {
        const float m = s * a;
        for (float b : x) {
          check(i, m, b);
          check(i, m, -b);
        }
        for (int k = 0; k < 400; ++k)  // distances up to and beyond the window
          if (i > 0) check(i, m, (float)fmax((double)m - 0.11 * k / i, -FLT_MAX));
        check(i, m, m);
        check(i, m, nextafterf(m, -FLT_MAX));
        check(i, m, -INFINITY);
        check(i, -INFINITY, -INFINITY);
      }
  int step;
  float rest;
  const Grid none(row_inv_T(1.0, -INFINITY), -INFINITY);  // a slice without a logit
  if (none.place(-INFINITY, step, rest) <= kLastBin + 1) ++bad;
  printf("%d placed, %d in reach, %d wrong\n", seen, in_window, bad);
  return bad != 0 || in_window < 10000;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_places_of_any_logit(tmp_path):
    src, exe = tmp_path / "grid.cpp", tmp_path / "grid"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wno-unknown-pragmas", "-fsanitize=float-cast-overflow",
                    "-fno-sanitize-recover=all", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
