"""Workgroups' turns at the units of a launch (csrc/turns.h), compiled for the host."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2403_16863_amd", "csrc")
PROGRAM = """
#include <cstdio>
#include <cstdlib>
#include "turns.h"
// Units seen by the workgroups [from, to) of `step`, each begun at its turn `skip`; "lost" where one is handed a unit outside [0, count).
int main(int, char** v) {
    const unsigned count = strtoul(v[1], 0, 10), step = strtoul(v[2], 0, 10), skip = strtoul(v[3], 0, 10);
    unsigned long long seen = 0, sum = 0;
    for (unsigned g = 0; g < step; ++g) {
        Turns t = {decltype(Turns::at)(g + skip * step), decltype(Turns::step)(step), decltype(Turns::count)(count)};
        for (; t.left(); t.next(), ++seen) {
            if (t.at < 0 || (unsigned)t.at >= count) return printf("lost"), 0;
            sum += (unsigned)t.at - skip * step;
        }
    }
    printf("%llu %llu", seen, sum);
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    where = tmp_path_factory.mktemp("turns")
    (where / "turns.cpp").write_text(PROGRAM)
    # -fwrapv: a sum that leaves its type is what the GPU would make of it, not undefined
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", f"-I{CSRC}", "-o", str(where / "turns"), str(where / "turns.cpp")], check=True)
    return str(where / "turns")


@pytest.mark.parametrize("count", [1, 511, 512, 513, 5000, 2 ** 31 - 513, 2 ** 31 - 512, 2 ** 31 - 511, 2 ** 31 - 1])
@pytest.mark.parametrize("step", [1, 256, 512])
def test_every_unit_is_taken_once(program, count, step):
    """Up to 2^31 - 1 units, as many as there are tokens at most: none is taken twice, and none behind the last."""
    step = min(step, count)
    skip = max(0, count // step - 3)                                    # (the last turns alone)
    rest = count - skip * step
    out = subprocess.run([program, str(count), str(step), str(skip)], capture_output=True, text=True, timeout=20, check=True).stdout
    assert out == f"{rest} {rest * (rest - 1) // 2}"
