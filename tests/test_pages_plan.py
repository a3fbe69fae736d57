"""The rules for the work of a cache's pages and of a cache in 4 bits (csrc/osdn_plan.h), compiled for the CPU."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_13473_amd", "csrc")
MAIN = r"""
#include "osdn_plan.h"
#include <cstdio>
#include <cstring>
using namespace osdn;
// decode: B rows max_length window K bf16 part_heads heads_together asked -> row_group units shares unit
// plan: tokens -> workgroups;  heads: groups heads -> heads of a wavefront;  select: B Hk heads_a_block pages bytes -> itself chunks
int main(int, char **argv) {
    long long a[9];
    const char *what = argv[1];
    const int n = what[0] == 'd' ? 9 : what[0] == 'p' ? 1 : what[0] == 'h' ? 2 : 5;
    for (;;) {
        for (int i = 0; i < n; ++i)
            if (std::scanf("%lld", a + i) != 1) return 0;
        if (what[0] == 'd') {
            const DecodePlan p = decode_plan(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], true);
            std::printf("%d %lld %d %d\n", p.row_group, p.units, p.shares, decode_mx_unit(p.row_group));
        } else if (what[0] == 'p') {
            std::printf("%d\n", plan_workgroups(a[0]));
        } else if (what[0] == 'h') {
            std::printf("%d\n", heads_mx_per_wave(a[0], a[1]));
        } else {
            std::printf("%d %u\n", (int)select_scores_itself(a[0] * a[1], a[3], a[4]), select_chunks(a[0], a[1], a[2], a[3]));
        }
    }
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", str(d / "rules"), str(d / "main.cpp")], check=True)

    def ask(what, rows):
        text = "\n".join(" ".join(str(int(x)) for x in r) for r in rows)
        return [[int(x) for x in line.split()] for line in subprocess.run([str(d / "rules"), what], input=text, capture_output=True, text=True, check=True).stdout.splitlines()]

    return ask


def test_attention_over_4_bits(rule):
    asked = [(B, r, L, win, K, bf, ph, tog, ask) for B in (1, 8, 64, 512, 65535) for r in (1, 2, 3, 4, 6, 16) for L in (0, 1, 127, 128, 129, 1000, 4096, 131072) for win in (0, 33, 1000)
             for K in (64, 128, 256) for bf in (0, 1) for ph in (1, 16) for tog in (0, 1) for ask in (0, -1, 7)]
    for (B, r, L, win, K, bf, ph, tog, ask), (together, units, shares, unit) in zip(asked, rule("decode", asked)):
        seen = min(L, win + 31) if win else L
        assert together in (1, 2, 4) and r % together == 0
        assert unit == 128 // together and units == max(1, -(-seen // unit))
        if ask:
            assert shares == max(ask, 0)
        else:
            assert 0 <= shares <= min(B * r // together * units, 1024)


def test_places_of_many_tokens(rule):
    asked = [(n,) for n in (1, 256, 1024, 1025, 4096, 4097, 8192, 65536, 10 ** 6, 2 ** 20, 2 ** 21, 2 ** 31 - 1)]
    for (n,), (w,) in zip(asked, rule("plan", asked)):
        assert 1 <= w <= 256 and (w == 1) == (n <= 1024)
        per = -(-n // w)
        assert (w - 1) * per < n <= w * per and w * per < 2 ** 31 + 256             # every part begins inside


def test_heads_of_a_wavefront(rule):
    asked = [(g, h) for g in (1, 2, 255, 4096, 16384, 10 ** 6, 2 ** 31) for h in (1, 3, 8, 64, 1000)]
    for (g, h), (n,) in zip(asked, rule("heads", asked)):
        assert 1 <= n <= h


def test_scores_of_pages(rule):
    asked = [(B, hk, t, n, by) for B in (1, 4, 64, 1024, 65535) for hk in (1, 2, 8, 32) for t in (1, 2, 4) for n in (1, 15, 16, 17, 256, 4096, 4097, 131072, 2 ** 27) for by in (256, 2048)]
    for (B, hk, t, n, by), (itself, chunks) in zip(asked, rule("select", asked)):
        assert not itself or n <= 4096                                             # (a row's keys are in registers)
        assert 1 <= chunks <= -(-n // 16) and B * -(-hk // t) * chunks <= B * hk + 5 * 256 + B * hk
