"""How the SMs are divided between the two passes of axon_attn_shared: CTAs that work it out for themselves, in different
kernels, have to agree to the last bit, so it is arithmetic of whole numbers. The header is compiled here as C++, at two
levels of optimisation, and compared with the same formula in Python."""
import os
import random
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_19889_gb300", "csrc")

PROGRAM = """
#include <stdio.h>
#include "own_split.h"
int main() {
  unsigned pages, rows, cost;
  int d, S, sms;
  while (scanf("%u %u %u %d %d %d", &pages, &rows, &cost, &d, &S, &sms) == 6) {
    const unsigned own = own_work(pages, rows, d);
    printf("%u %u\\n", own, split_time(own, cost, S, sms));
  }
}
"""


def expected(pages, rows, cost, d, S, sms):
    pages, rows, cost = min(pages, 2 ** 28), min(rows, 2 ** 25), min(cost, 2 ** 28 - 1)
    own = (pages * 5 // 2 if d == 64 else pages * 5) + rows * 50
    return own, min(max(64 + own // S, cost * 16 // (sms - S), 160), 2 ** 22 - 1)


def cases(n):
    r = random.Random(1)
    yield from [(0, 0, 1, 128, 2, 4), (2 ** 32 - 1, 2 ** 32 - 1, 2 ** 32 - 1, 128, 1, 512), (2 ** 31 - 1, 1, 5, 64, 2, 152),
                # sums that fp32 rounds otherwise when a product is fused with them
                (12775694, 518, 3889217, 128, 76, 152), (5624345, 1049, 990717, 128, 96, 152)]
    for _ in range(n):
        sms = r.randrange(4, 513)
        yield (int(2 ** r.uniform(0, 31)), int(2 ** r.uniform(0, 26)), int(2 ** r.uniform(0, 31)), r.choice([64, 128]),
               r.randrange(1, sms), sms)


@pytest.mark.parametrize("level", ["-O0", "-O3"])
def test_whole_numbers(tmp_path, level):
    source, program = tmp_path / "split.cpp", tmp_path / "split"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", level, "-Wall", "-Wextra", "-Werror", "-I" + CSRC, str(source), "-o", str(program)], check=True)
    asked = list(cases(20000))
    out = subprocess.run([str(program)], input="\n".join(" ".join(map(str, c)) for c in asked), text=True, capture_output=True,
                         check=True).stdout
    got = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert got == [expected(*c) for c in asked]


def test_no_floating_point_decides():
    with open(os.path.join(CSRC, "attn_shared.cuh")) as f:
        body = re.search(r"AXON_DEV int own_sms\(.*?\n}\n", f.read(), re.S).group(0)
    assert not re.search(r"float|double|\df\b|__f", body)
