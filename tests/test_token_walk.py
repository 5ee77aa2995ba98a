"""The walk of the rotation kernels' workers over their tokens, on the host: every token once, up to the most that a call takes."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_37842_amd", "csrc")
# stdin: "from step tokens"; stdout: groups (one more than a walk of that length has, if it does not end), tokens, the least
# and the last token
PROGRAM = r"""
#include <cstdio>
#include "token_walk.h"
int main() {
  long long from, step, n;
  while (std::scanf("%lld %lld %lld", &from, &step, &n) == 3) {
    eogp::TokenWalk w((int)from, (int)step, (int)n);
    const long long most = n / (64 * step) + 1;
    long long groups = 0, count = 0, least = -1, last = -1;
    while (groups <= most && w.next()) {
      ++groups;
      if (least < 0 || w.at(0) < least) least = w.at(0);
      for (int k = 0; k < 64 && w.has(k); ++k) {
        ++count;
        last = w.at(k);
      }
    }
    std::printf("%lld %lld %lld %lld\n", groups, count, least, last);
  }
}
"""
CASES = [(f, s, n) for s in (1, 4, 1020, 4096, 8192) for f in (0, s - 1) for n in (
    1, 63, 64 * s, 64 * s + f + 1, 2 ** 31 - 64 * s, 2 ** 31 - 64 * s + 1, 2 ** 31 - 8192, 2 ** 31 - 1) if s > 4 or n < 2 ** 24]


def test_walks_end(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-fwrapv", f"-I{CSRC}", str(src), "-o", str(exe)], check=True,
                   capture_output=True, text=True)
    text = "".join(f"{f} {s} {n}\n" for f, s, n in CASES)
    out = subprocess.run([str(exe)], input=text, check=True, capture_output=True, text=True).stdout
    for (f, s, n), line in zip(CASES, out.splitlines(), strict=True):
        count = max(0, -(-(n - f) // s))
        want = (-(-count // 64), count, f if count else -1, f + (count - 1) * s if count else -1)
        assert tuple(map(int, line.split())) == want, (f, s, n)
