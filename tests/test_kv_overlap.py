"""The check that an output lies on no input, against an enumeration of the elements (no GPU)."""
import os
import subprocess

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = r'''
#include <cstdio>
#include "ps_kv_overlap.cuh"
int main() {
  long long xp, xs0, xs1, xh, yp, ys0, ys1, yh, T, D;
  while (scanf("%lld %lld %lld %lld %lld %lld %lld %lld %lld %lld", &xp, &xs0, &xs1, &xh, &yp, &ys0, &ys1, &yh, &T, &D) == 10) {
    const pskv::HeadRuns x{(const void*)(xp * 2 + 1024), xs0, xs1, xh}, y{(const void*)(yp * 2 + 1024), ys0, ys1, yh};
    printf("%d %d\n", (int)pskv::heads_overlap(x, y, T, D), (int)pskv::heads_overlap(x, x, T, D, true));
  }
}
'''


def elements(p, s0, s1, heads, T, D):
    return (p + np.arange(T)[:, None, None] * s0 + np.arange(heads)[:, None] * s1 + np.arange(D)).ravel()


def test_against_enumeration(tmp_path):
    src, exe = tmp_path / "main.cpp", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.run(["g++", "-O1", "-I" + os.path.join(ROOT, "paper_2608_01657_gb300", "csrc"), str(src), "-o", str(exe)], check=True)
    r = np.random.RandomState(1)
    cases = []
    for i in range(12000):
        D, T, xh, yh = 8 * r.randint(1, 4), r.randint(1, 6), r.randint(1, 6), r.randint(1, 6)
        xs = [8 * r.randint(0, 40), 8 * r.randint(0, 12)]
        if i % 3 == 0:    # token-major, as they mostly are
            xs = [xh * D + 8 * r.randint(0, 30), D]
        elif i % 3 == 1:  # head-major
            xs = [D, T * D + 8 * r.randint(0, 9)]
        ys = [list(xs), [xs[0], D], [yh * D, D], [8 * r.randint(0, 40), 8 * r.randint(0, 12)]][r.choice(4, p=[0.55, 0.1, 0.15, 0.2])]
        cases.append((8 * r.randint(0, 60), *xs, xh, 8 * r.randint(0, 60), *ys, yh, T, D))
    got = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True,
                         check=True).stdout.split()
    seen = set()
    for c, both, self in zip(cases, got[::2], got[1::2]):
        xp, xs0, xs1, xh, yp, ys0, ys1, yh, T, D = c
        x, y = elements(xp, xs0, xs1, xh, T, D), elements(yp, ys0, ys1, yh, T, D)
        want = len(np.intersect1d(x, y)) > 0, len(np.unique(x)) < len(x)
        assert (both == "1", self == "1") == want, c
        inside = x.min() <= y.max() and y.min() <= x.max()
        seen.add((want[0], inside, xs0 == ys0 and xs1 == ys1))
    assert {(True, True, True), (False, True, True), (True, True, False), (False, True, False), (False, False, True)} <= seen
