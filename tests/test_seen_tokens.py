"""Which tokens of a paged cache a query sees (csrc/osdn_plan.h), compiled for the CPU, for lengths that are none too: attention walks from there by tiles
in 32 bits, and ends."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_13473_amd", "csrc")
MAIN = r"""
#include "osdn_plan.h"
#include <cstdio>
using namespace osdn;
int main() {
    int length, seq, n, most, window, shift, pages, unit;
    while (std::scanf("%d %d %d %d %d %d %d %d", &length, &seq, &n, &most, &window, &shift, &pages, &unit) == 8) {
        const Seen s = seen_tokens(length, seq, n, most, window, shift, pages);
        std::printf("%d %d %d %d %d\n", s.lo, s.end, s.broken, seen_begin(s), seen_units(s, unit));
    }
    return 0;
}
"""
TOP, MOST = 2 ** 31 - 1, 0x7fffff00        # (the largest max_length)


@pytest.fixture(scope="module")
def seen(tmp_path_factory):
    d = tmp_path_factory.mktemp("seen")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all", "-I", CSRC, "-o", str(d / "seen"), str(d / "main.cpp")], check=True)

    def ask(rows):
        text = "\n".join(" ".join(str(x) for x in r) for r in rows)
        out = subprocess.run([str(d / "seen")], input=text, capture_output=True, text=True, check=True).stdout
        return [[int(x) for x in line.split()] for line in out.splitlines()]

    return ask


def test_tokens_that_are_seen(seen):
    asked = [(length, 0, 1, most, window, shift, pages, unit)
             for length in (-TOP - 1, -TOP, -1, 0, 1, 31, 32, 33, 1000, 4096, 4097, 131072, MOST - 1, MOST, MOST + 1, TOP - 31, TOP - 1, TOP)
             for most in (0, 1, 33, 4096, 131072, MOST) for window in (0, 1, 31, 32, 33, 1000, MOST, TOP)
             for shift, pages in ((4, 256), (0, 4096), (30, 1), (4, TOP)) for unit in (16, 32, 64, 128)]
    for (length, _, _, most, window, shift, pages, unit), (lo, end, broken, begin, units) in zip(asked, seen(asked)):
        kept = length <= most and length <= pages << shift
        assert broken == (length > 0 and not kept)
        assert (lo, end) == ((max(0, length - window) if window else 0, length) if length > 0 and kept else (0, 0))
        assert begin == lo - lo % 32 and units == max(1, -(-(end - begin) // unit))
        # the walk of four wavefronts: a tile each in turn, the pages of the one behind it looked up
        assert 0 <= lo <= end <= most and end - 1 + 128 + 31 <= TOP and begin + 3 * 32 + 31 <= TOP


def test_sequences_that_are_not_there(seen):
    for seq, n, broken in ((0, 1, 0), (1, 1, 1), (-1, 5, 1), (4, 5, 0), (5, 5, 1), (TOP, TOP, 1), (-TOP - 1, TOP, 1)):
        assert seen([(40, seq, n, 100, 0, 4, 10, 128)])[0][:3] == ([0, 0, 1] if broken else [0, 40, 0])


def test_without_a_token_the_sequence_is_not_asked_for(seen):
    for length in (0, -1, -TOP - 1):
        for seq in (0, -1, 5, TOP, -TOP - 1):
            assert seen([(length, seq, 5, 100, 7, 4, 10, 128)]) == [[0, 0, 0, 0, 1]]
