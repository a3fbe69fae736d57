"""Where the selection of pages ends: how many pages a sequence may have, and that counting them stays in 32 bits up to there."""
import os
import subprocess

import pytest

from paper_2605_13473_amd import binding as ob
from tests.test_heads_abi import PARAM, SHAPE
from tests.test_pages_abi import choice, pages, select

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_13473_amd", "csrc")
MAIN = r"""
#include "osdn_plan.h"
#include <cstdio>
#include <initializer_list>
using namespace osdn;
// The page counter of score_kernel, walked in 64 bits: the largest value that any wavefront's takes, with the places of a step
int main() {
    long long worst = 0;
    const int most = SELECT_MAX_PAGES;
    for (int B : {1, 2, 64, 65535})
        for (int hk : {1, 2, 8})
            for (int side : {1, 2, 4})
                for (int pages : {most, most - 1, most - 255, most / 2 + 1}) {
                    const unsigned chunks = select_chunks(B, hk, side, pages);
                    const long long stride = 16LL * chunks;
                    for (unsigned wave : {0u, 1u, 4 * chunks - 1}) {
                        long long p = 4LL * wave;
                        if (p < pages) p += (pages - 1 - p) / (SELECT_STEPS * stride) * (SELECT_STEPS * stride);      // the last round
                        const long long end = p + SELECT_STEPS * stride + 64;
                        if (end > worst) worst = end;
                    }
                }
    for (long long count : {(long long)most, most - 1LL}) {             // select_kernel: the runs of 512 threads
        const long long run = (count + 511) / 512;
        for (long long end : {count + 511, 511 * run})
            if (end > worst) worst = end;
    }
    std::printf("%d %lld\n", most, worst);
}
"""


def test_pages_are_counted_in_32_bits(tmp_path):
    (tmp_path / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", str(tmp_path / "limits"), str(tmp_path / "main.cpp")], check=True)
    most, worst = map(int, subprocess.run([str(tmp_path / "limits")], capture_output=True, text=True, check=True).stdout.split())
    assert most == 2 ** 30 and worst < 2 ** 31


@pytest.mark.parametrize("page,length", [(1, 2 ** 30 + 1), (1, 2 ** 31 - 256), (1, 2 ** 31 - 262144)])
def test_more_pages_than_are_counted_are_refused(page, length):
    p = choice(B=1, Hq=1, Hk=1, max_length=length)
    g = pages(page_size=page, max_pages=2 ** 31 - 1, table_stride=2 ** 31 - 1, n_seqs=1)
    assert ob.osdn_page_select_workspace_bytes(p, page) == 0
    assert select(p, g, ws=None, size=0) == SHAPE
    assert ob.osdn_page_select_workspace_bytes(choice(B=1, Hq=1, Hk=1, max_length=2 ** 30), 1) == 8 * 2 ** 30


def test_more_pages_than_are_counted_are_not_chosen():
    g = pages(page_size=1, max_pages=2 ** 31 - 1, table_stride=2 ** 31 - 1, n_seqs=1)
    for n in (2 ** 30 + 1, 2 ** 31 - 256):
        assert select(choice(B=1, Hq=1, Hk=1, pages=n), g, chosen=None) == PARAM


def test_bounds_of_more_pages_than_a_launch_has_wavefronts(tmp_path):
    """All pages that B sequences may hold, as page_bounds takes them where it is not told how many tokens are new."""
    (tmp_path / "main.cpp").write_text('#include "osdn_plan.h"\n#include <cstdio>\nint main() { long long n; while (std::scanf("%lld", &n) == 1) std::printf("%u\\n", osdn::bounds_workgroups(n)); }\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", str(tmp_path / "workgroups"), str(tmp_path / "main.cpp")], check=True)
    asked = [1, 4, 5, 1000, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, 2048 * 4096 * 8, 2 ** 31 - 1]
    got = subprocess.run([str(tmp_path / "workgroups")], input="\n".join(map(str, asked)), capture_output=True, text=True, check=True).stdout.split()
    for n, w in zip(asked, map(int, got)):
        assert 1 <= w and 256 * w < 2 ** 32 and (4 * w >= n or w == 2 ** 22)
