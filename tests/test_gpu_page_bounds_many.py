"""Bounds of pages, more of them than a launch has wavefronts."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob

pytestmark = pytest.mark.gpu


def test_all_pages_that_many_sequences_may_hold():
    """2100 rows of 4096 pages, eight heads: 6.9e7 pages and heads that may have new tokens.  The first sequence's, one in the middle's and the last one's have some."""
    g = torch.Generator(device="cuda").manual_seed(1)
    B, most, Hk, K, page = 2100, 4096, 8, 64, 4
    assert B * most * Hk > 2 ** 26
    table = torch.full((B, most), -1, dtype=torch.int32, device="cuda")
    rows = {0: [3, 0], 1234: [5], B - 1: [1, 4, 2]}
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    for b, pages in rows.items():
        table[b, :len(pages)] = torch.tensor(pages, dtype=torch.int32)
        lengths[b] = page * len(pages)
    table[B - 1, most - 1] = 6                                      # the very last page of the last row
    cached = torch.zeros_like(lengths)
    keys = torch.randn(8, page, Hk, K, device="cuda", generator=g).bfloat16()
    bounds = torch.zeros(8, Hk, 2, K, dtype=torch.bfloat16, device="cuda")
    ob.page_bounds(keys, table, cached, lengths, bounds)
    want = torch.stack([keys.amin(1), keys.amax(1)], dim=2)
    want[6:] = 0
    assert torch.equal(bounds, want)
    lengths[B - 1] = page * most
    cached[B - 1] = page * (most - 1)
    ob.page_bounds(keys, table, cached, lengths, bounds, max_new=page * most)
    want[6] = torch.stack([keys[6].amin(0), keys[6].amax(0)], dim=1)
    assert torch.equal(bounds, want)
