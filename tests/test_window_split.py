"""The choice of how many CTAs share a unit's rows (csrc/sh_window_split.h), compiled for the host."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "sh_window_split.h"
int main(int n, char **a) {      // units rows row_bytes rate slots x 4
    const int slots[4] = {atoi(a[5]), atoi(a[6]), atoi(a[7]), atoi(a[8])};
    const shwin::Shape s = shwin::best_split(atoll(a[1]), atoll(a[2]), atoi(a[3]), slots, atof(a[4]));
    printf("%d %.9g\n", s.S, s.us);
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    where = tmp_path_factory.mktemp("split")
    (where / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2305_17118_b200", "csrc"), "-o", str(where / "split"),
                    str(where / "main.cpp")], check=True)

    def call(units, rows, slots, row_bytes=512, rate=5.8e4):
        done = subprocess.run([str(where / "split"), *map(str, (units, rows, row_bytes, rate, *slots))], capture_output=True, text=True, check=True)
        s, us = done.stdout.split()
        return int(s), float(us)

    return call


def test_few_units_over_many_rows_share_and_many_units_do_not(split):
    slots = (148, 148, 144, 136)
    assert split(8, 16384, slots)[0] == 8
    assert split(9216, 410, slots)[0] == 1
    assert split(8, 60, slots)[0] == 1


@pytest.mark.parametrize("units", [1, 8, 100, 5000])
@pytest.mark.parametrize("rows", [1, 128, 4096, 1 << 20])
def test_clusters_without_a_place_are_never_chosen(split, units, rows):
    """A device (or a part of one) may hold no cluster of a size; what it holds is chosen, single CTAs at the least."""
    for slots in ((148, 148, 144, 0), (148, 148, 0, 0), (148, 0, 0, 0), (0, 0, 0, 0), (20, 0, 8, 0), (148, 0, 0, 128)):
        s, us = split(units, rows, slots)
        assert s == 1 or slots[s.bit_length() - 1] >= s
        assert us < 1e300
