"""The shares of attention's line of tiles: they cover it without a gap or an overlap, for lines as long as a call may have.  CPU only: the
header that the kernels use is compiled as plain C++."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include "dart_shares.h"
using dart::attend::Shares;
int main()
{
    long long line, items;
    int n, least;
    while (scanf("%lld %lld %d %d", &line, &items, &n, &least) == 4) {
        const Shares s = Shares::of((int)line, items, n, least);
        long long at = 0, largest = 0, smallest = line + 1;
        for (int w = 0; w < n; ++w) {
            const long long size = s.size(w);
            if (size < 0 || (size > 0 && s.begin(w) != at) || s.begin(w) < 0) return printf("bad %lld %lld %d %d: worker %d at %d, %lld\n", line, items, n, least, w, s.begin(w), size), 1;
            at += size;
            if (size > largest) largest = size;
            if (size < smallest) smallest = size;
        }
        if (at != line) return printf("bad %lld %lld %d %d: %lld covered\n", line, items, n, least, at), 1;
        printf("%lld %lld\n", smallest, largest);
    }
    return 0;
}
"""

LONGEST = 2**31 - 2


@pytest.fixture(scope="module")
def shares(tmp_path_factory):
    d = tmp_path_factory.mktemp("shares")
    src = d / "shares.cpp"
    src.write_text(PROGRAM)
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    subprocess.check_call([cxx, "-std=c++17", "-O1", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", "-I",
                           os.path.join(ROOT, "paper_2502_11494_b200", "csrc"), "-o", str(d / "shares"), str(src)])

    def run(cases):
        r = subprocess.run([str(d / "shares")], input="\n".join("%d %d %d %d" % c for c in cases), capture_output=True, text=True)
        assert r.returncode == 0, r.stdout[-300:] + r.stderr[-300:]
        got = [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]
        assert len(got) == len(cases)
        return got

    return run


@pytest.mark.parametrize("n", [1, 2, 148, 296, 1184])
def test_shares_cover_the_line(shares, n):
    near = [2**30, 2**31, 2**30 + 2**29, 3 * 2**28, n, 5 * n, 1000 * n]
    lines = sorted({x + d for x in near for d in range(-3, 4) if 0 <= x + d <= LONGEST} | set(range(0, 70)) | {LONGEST})
    cases = [(x, i, n, 1) for x in lines for i in (1, 64, max(1, x // 3))]
    for (line, _, _, _), (small, large) in zip(cases, shares(cases)):
        assert large - small <= 1 and large <= line // n + 1


def test_least_shares_cover_the_line(shares):
    r = random.Random(5)
    cases = [(min(LONGEST, int(2 ** r.uniform(0, 31))), int(2 ** r.uniform(0, 29)), r.choice((148, 296, 1184, 37)), r.choice((1, 4))) for _ in range(4000)]
    shares(cases)
