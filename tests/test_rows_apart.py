"""Rows that are written must not stand in one another: the rule (csrc/osdn_plan.h), compiled for the CPU, against all pairs of rows, and what the entry
points refuse by it (no pointer is used)."""
import ctypes
import itertools
import os
import random
import subprocess

import pytest

from paper_2605_13473_amd import binding as ob
from tests.test_heads_abi import FAKE, SHAPE, cache, norm_params, rows

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_13473_amd", "csrc")
MAIN = r"""
#include "osdn_plan.h"
#include <cstdio>
int main() {
    long long n[3], s[3];
    int K;
    while (std::scanf("%lld %lld %lld %lld %lld %lld %d", &n[0], &n[1], &n[2], &s[0], &s[1], &s[2], &K) == 7) std::printf("%d\n", osdn::rows_apart(n, s, K));
    return 0;
}
"""


@pytest.fixture(scope="module")
def apart(tmp_path_factory):
    d = tmp_path_factory.mktemp("apart")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, "-o", str(d / "apart"), str(d / "main.cpp")], check=True)

    def ask(asked):
        text = "\n".join(" ".join(str(x) for x in (*n, *s, K)) for n, s, K in asked)
        out = subprocess.run([str(d / "apart")], input=text, capture_output=True, text=True, check=True).stdout
        return [int(line) for line in out.split()]

    return ask


def _meet(n, s, K):
    at = sorted(sum(i * x for i, x in zip(ijk, s)) for ijk in itertools.product(*(range(m) for m in n)))
    return any(b - a < K for a, b in zip(at, at[1:]))


def test_no_two_rows_of_what_is_taken_meet(apart):
    rng = random.Random(2)
    asked = [(tuple(rng.choice([1, 1, 2, 3, 5]) for _ in range(3)), tuple(rng.choice([-1, 1]) * rng.choice([0, 3, 4, 5, 8, 12, 16, 20, 24, 60, 100]) for _ in range(3)), 4) for _ in range(4000)]
    taken = 0
    for (n, s, K), ok in zip(asked, apart(asked)):
        assert not (ok and _meet(n, s, K))
        taken += ok
    assert taken > 500


def test_parts_and_orders_of_arrays_are_taken(apart):
    rng, asked = random.Random(3), []
    for _ in range(2000):
        wide, order = [rng.choice([1, 2, 3, 7]) for _ in range(3)], rng.sample(range(3), 3)
        row, steps = 64 + rng.choice([0, 1, 8]), [0, 0, 0]
        for axis in order:
            steps[axis] = row
            row *= wide[axis]
            row += rng.choice([0, 0, 5])                                # (padded)
        n, s = [], []
        for m, x in zip(wide, steps):                                   # every other entry, backwards, fewer
            by = rng.choice([1, 1, 2, -1, -2])
            n.append(rng.randint(1, max(1, m // abs(by))))
            s.append(x * by)
        asked.append((tuple(n), tuple(s), 64))
    assert all(apart(asked))
    big = 2 ** 62
    assert apart([((65535, 2 ** 31 - 1, 2), (big, 2 ** 31, 64), 64), ((2, 2, 2), (-2 ** 63, big, 64), 64), ((2, 2, 1), (big, big, 0), 64)]) == [1, 1, 0]


@pytest.mark.parametrize("kw", [dict(token=64, head=64), dict(token=64, head=128), dict(batch=256, token=256), dict(batch=128, token=256), dict(batch=-512), dict(token=-64, head=64)], ids=str)
def test_outputs_whose_rows_meet_are_refused(kw):
    L, p, r, bad = ob.lib(), norm_params(), ctypes.byref(rows()), ctypes.byref(rows(**kw))
    fwd = lambda a, b: L.osdn_qk_norm_fwd(ctypes.byref(p), r, r, None, None, None, None, a, b, None)
    assert fwd(bad, r) == SHAPE and fwd(r, bad) == SHAPE
    bwd = lambda a, b: L.osdn_qk_norm_bwd(ctypes.byref(p), r, r, None, None, None, None, r, r, a, b, None, None, None, 0, None)
    assert bwd(bad, r) == SHAPE and bwd(r, bad) == SHAPE
    assert L.osdn_paged_append(ctypes.byref(p), ctypes.byref(cache()), r, r, r, None, None, None, FAKE, None, bad, None) == SHAPE


@pytest.mark.parametrize("kw", [dict(batch=64), dict(batch=128), dict(batch=-192)], ids=str)
def test_results_of_attention_whose_rows_meet_are_refused(kw):
    r, bad = ctypes.byref(rows()), ctypes.byref(rows(**kw))
    p = ob.make_decode_params(2, 4, 4, 64, True, 100)
    assert ob.lib().osdn_paged_decode(ctypes.byref(p), ctypes.byref(cache()), r, FAKE, None, bad, None, None, 0, None) == SHAPE


@pytest.mark.parametrize("kw", [dict(k_token=64, k_head=64), dict(v_token=64, v_head=64), dict(k_page=256, k_token=256), dict(v_page=128), dict(k_head=512)], ids=str)
def test_a_cache_whose_rows_meet_is_not_appended_to(kw):
    r, c = ctypes.byref(rows()), cache(**kw)
    assert ob.lib().osdn_paged_append(ctypes.byref(norm_params()), ctypes.byref(c), r, r, r, None, None, None, FAKE, None, r, None) == SHAPE
