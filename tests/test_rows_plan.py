"""The rules that cut the work of the operators around the recurrence (csrc/osdn_plan.h), compiled for the CPU: every block of rows and every
unit of tokens falls to one wavefront or share, and what a second kernel joins is what the first one left."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_13473_amd", "csrc")
MAIN = r"""
#include "osdn_plan.h"
#include <algorithm>
#include <cstdio>
#include <cstring>
#include <map>
#include <vector>
using namespace osdn;
// heads: tokens Hq Hk K bf16 values backward -> q_blocks k_blocks blocks per_part parts workgroups, 1 if the parts cover the blocks
// decode: B rows max_length window K bf16 part_heads heads_together asked -> row_group units shares unit
// cut: W rows B u_0 .. u_(B-1) -> 1 if the shares cover the rows' units, every slot is written once, and a row's parts are found where they were left
int main(int, char **argv) {
    if (!std::strcmp(argv[1], "heads")) {
        long long tokens; int Hq, Hk, K, bf, v, b;
        while (std::scanf("%lld %d %d %d %d %d %d", &tokens, &Hq, &Hk, &K, &bf, &v, &b) == 7) {
            const HeadsPlan h = heads_plan(tokens, Hq, Hk, K, bf, v, b);
            int covered = 0;
            for (int p = 0; p < h.parts; ++p) {
                const int n = std::min(h.blocks, (p + 1) * h.per_part) - p * h.per_part;
                if (n < 1) covered = -1 << 30;
                covered += n;
            }
            std::printf("%d %d %d %d %d %d %d\n", h.q_blocks, h.k_blocks, h.blocks, h.per_part, h.parts, h.workgroups, covered == h.blocks);
        }
    } else if (!std::strcmp(argv[1], "decode")) {
        int B, rows, L, win, K, bf, ph, tog, ask;
        while (std::scanf("%d %d %d %d %d %d %d %d %d", &B, &rows, &L, &win, &K, &bf, &ph, &tog, &ask) == 9) {
            const DecodePlan p = decode_plan(B, rows, L, win, K, bf, ph, tog, ask);
            std::printf("%d %lld %d %d\n", p.row_group, p.units, p.shares, decode_unit(K, bf, p.row_group));
        }
    } else {
        int W, rows, B;
        while (std::scanf("%d %d %d", &W, &rows, &B) == 3) {
            std::vector<int> u(B);
            long long total = 0;
            for (int &x : u) { (void)!std::scanf("%d", &x); total += x; }
            const Shares s((int)(total * rows), W);
            std::vector<int> start, len;                    // the rows in the list
            for (int b = 0, at = 0; b < B; ++b)
                for (int r = 0; r < rows; ++r, at += u[b]) { start.push_back(at); len.push_back(u[b]); }
            std::map<int, std::pair<int, int>> left;        // slot -> row, first unit
            std::vector<int> seen(total * rows, 0);
            bool ok = s.begin(0) == 0 && s.begin(W) == total * rows;
            for (int w = 0; w < W && ok; ++w) {
                int r = 0;
                for (int at = s.begin(w); at < s.begin(w + 1);) {
                    while (at >= start[r] + len[r]) ++r;
                    const int to = std::min(start[r] + len[r], s.begin(w + 1));
                    for (int i = at; i < to; ++i) { ++seen[i]; ok = ok && s.owner(i) == w; }
                    if (at != start[r] || to != start[r] + len[r]) ok = ok && left.emplace(part_slot(w, at == s.begin(w)), std::make_pair(r, at - start[r])).second;
                    at = to;
                }
            }
            for (int x : seen) ok = ok && x == 1;
            size_t read = 0;
            for (size_t r = 0; r < start.size(); ++r) {
                const int w = s.owner(start[r]), n = s.owner(start[r] + len[r] - 1) - w + 1;
                if (n == 1) continue;
                const int first = part_slot(w, start[r] == s.begin(w));
                int before = -1;
                for (int i = 0; i < n; ++i, ++read) {
                    const auto it = left.find(part_of_row(first, i));
                    ok = ok && it != left.end() && it->second.first == (int)r && it->second.second > before && part_of_row(first, i) < 2 * W;
                    if (it != left.end()) before = it->second.second;
                }
            }
            std::printf("%d\n", ok && read == left.size());
        }
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", str(d / "plan"), str(d / "main.cpp")], check=True)

    def ask(what, rows):
        text = "\n".join(" ".join(str(int(x)) for x in r) for r in rows)
        out = subprocess.run([str(d / "plan"), what], input=text, capture_output=True, text=True, check=True).stdout
        return [[int(x) for x in line.split()] for line in out.splitlines()]

    return ask


def test_every_block_of_rows_falls_to_one_wavefront(plan):
    asked = [(t, hq, hk, K, bf, v, b) for t in (1, 2, 27, 500, 1531, 4096, 16384, 65536, 10 ** 6) for hq, hk in ((0, 1), (1, 0), (1, 1), (5, 3), (16, 4), (32, 8), (64, 64), (1000, 7))
             for K in (64, 128, 256) for bf in (0, 1) for v, b in ((0, 0), (1, 0), (0, 1))]
    for (t, hq, hk, K, bf, v, b), (qb, kb, blocks, per, parts, wgs, ok) in zip(asked, plan("heads", asked)):
        rows = 1024 // (K * (2 if bf else 4))
        assert ok and qb == -(-hq // rows) and kb == -(-hk // rows) and blocks == qb + kb * (1 + v)
        assert 1 <= wgs <= (1024 if b else 16384) and 4 * wgs <= t * parts + 3


def test_decode_plans(plan):
    asked = [(B, r, L, win, K, bf, ph, tog, ask) for B in (1, 8, 64, 512, 65535) for r in (1, 2, 3, 4, 6, 16) for L in (0, 1, 127, 128, 129, 1000, 4096, 131072) for win in (0, 33, 1000)
             for K in (64, 128, 256) for bf in (0, 1) for ph in (1, 16) for tog in (0, 1) for ask in (0, -1, 7)]
    for (B, r, L, win, K, bf, ph, tog, ask), (together, units, shares, unit) in zip(asked, plan("decode", asked)):
        seen = min(L, win + 31) if win else L
        assert together in (1, 2, 4) and r % together == 0
        assert unit == (128 if bf and K <= 128 else 64) // together and units == max(1, -(-seen // unit))
        if ask:
            assert shares == max(ask, 0)
        else:
            assert 0 <= shares <= min(B * r // together * units, 768)
            assert shares > 0 or seen <= 384 or B * r >= 128
        assert tog or (K == 64 and bf) or together == 1 or (shares == 0 and seen <= 128)


def test_shares_cover_and_are_joined(plan):
    rng = random.Random(5)
    asked = [(1, 1, 1, 1), (7, 2, 1, 3), (3, 1, 3, 1, 1, 1), (4, 1, 2, 2, 2), (5, 3, 2, 4, 1), (1000, 2, 2, 3, 5), (512, 4, 1, 1024)]
    for _ in range(400):
        B, rows = rng.randint(1, 12), rng.choice([1, 1, 2, 4, 5])
        u = [rng.choice([1, 1, 2, rng.randint(1, 40), rng.randint(1, 300)]) for _ in range(B)]
        asked.append((rng.choice([1, 2, 3, 8, rng.randint(1, 600), rows * sum(u), rows * B]), rows, B, *u))
    assert all(r == [1] for r in plan("cut", asked))
