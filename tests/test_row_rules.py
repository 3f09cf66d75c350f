"""How rows are counted (csrc/pilc_row_rules.hpp) up to the largest numbers of them, compiled with the host compiler."""
import os
import subprocess

import pytest

RULES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2206_05279_amd", "csrc", "pilc_row_rules.hpp")

# for `rows step first`: how many rows beginning with `first` a workgroup goes through, the last of them, and workgroups of 32 rows
_PROGRAM = """
#include <cstdio>
#include "%s"
int main()
{
    unsigned rows, step, first;
    while (scanf("%%u %%u %%u", &rows, &step, &first) == 3) {
        uint32_t row = first;
        unsigned long long seen = 0;
        for (bool more = row < rows; more && seen < (1ull << 33); more = pilc::next_row(row, step, rows - 1)) ++seen;
        printf("%%llu %%u %%u\\n", seen, row, pilc::div_up(rows, 32u));
    }
}
""" % RULES


@pytest.mark.parametrize("rows", [1, 31, 32, 33, 40961, 2 ** 31, 2 ** 32 - 40961, 2 ** 32 - 40960, 2 ** 32 - 32, 2 ** 32 - 31, 2 ** 32 - 1])
def test_every_row_is_met_once_and_the_count_ends(rows, tmp_path):
    (tmp_path / "rules.cpp").write_text(_PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-o", str(tmp_path / "rules"), str(tmp_path / "rules.cpp")], check=True)
    asked = [(step, first) for step in (40960, 4096, 1 << 20) for first in {0, min(step, rows) - 1, step - 1}]
    out = subprocess.run([str(tmp_path / "rules")], input="".join("%d %d %d\n" % (rows, *a) for a in asked), capture_output=True, text=True,
                         check=True, timeout=60).stdout
    for (step, first), line in zip(asked, out.splitlines()):
        want = range(first, rows, step)
        seen, last, blocks = map(int, line.split())
        assert seen == len(want) and last == (want[-1] if seen else first) and blocks == (rows + 31) // 32
