"""The limit of a kernel's wait (csrc/dhq_wait.h), compiled for the host with a clock of the test's own."""
import shutil
import subprocess

import pytest

from paper_2508_13478_b200 import build

PROGRAM = r"""
#include "dhq_wait.h"
#include <cstdio>
#include <initializer_list>
int main()
{
    const unsigned long long limit = 2000000000ull;
    int bad = 0;
    auto expect = [&](const char *what, bool good) { if (!good) std::printf("%s\n", what), bad = 1; };
    for (unsigned long long start : {0ull, 5000000000ull, ~0ull - 30000ull}) { // (the clock may be anywhere, and wrap)
        unsigned long long t = start;
        volatile int failed = 0;
        auto now = [&] { return t; };
        // many waits, of 40 us each, in a block that is far older than the limit in the end
        bool all = true;
        for (int i = 0; i < 100000; ++i) {
            int tries = 0;
            all = all && dhq::wait_bounded([&] { t += 20000; return ++tries == 3; }, now, limit, &failed);
        }
        expect("short waits of an old block", all && !failed);
        // put aside for ten seconds between an attempt and the next one, which succeeds
        int tries = 0;
        expect("a pause before success", dhq::wait_bounded([&] { t += ++tries == 2 ? 10000000000ull : 20000; return tries == 2; }, now, limit, &failed) && !failed);
        // something that never comes
        const unsigned long long before = t;
        long count = 0;
        expect("a wait without end", !dhq::wait_bounded([&] { t += 20000; ++count; return false; }, now, limit, &failed) && failed);
        expect("its length", t - before > limit && t - before < limit + 200000 && count < 101000);
        // another wait of the block gave up
        count = 0;
        expect("given up elsewhere", !dhq::wait_bounded([&] { ++count; return false; }, now, limit, &failed) && count == 1);
        expect("there at once", dhq::wait_bounded([] { return true; }, now, limit, &failed));
    }
    return bad;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="needs g++")
def test_a_wait_is_limited_by_its_own_length(tmp_path):
    source = tmp_path / "wait.cpp"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC, "-o", str(tmp_path / "wait"), str(source)], check=True)
    ran = subprocess.run([str(tmp_path / "wait")], capture_output=True, text=True, timeout=60)
    assert ran.returncode == 0, ran.stdout
