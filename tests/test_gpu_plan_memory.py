"""What a server keeps of a plan holds no more memory than it has a use for."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("slots", [False, True])
@pytest.mark.parametrize("B,tokens", [(1, 1), (7, 4096), (7, 4097), (300, 8193), (64, 10 ** 6)])
def test_kept_results_do_not_hold_the_places_of_the_tokens(B, tokens, slots):
    i32 = dict(dtype=torch.int32, device="cuda")
    table, free, n_free = torch.full((B, 4), -1, **i32), torch.arange(4 * B, **i32), torch.full((1,), 4 * B, **i32)
    cached, fresh = torch.zeros(B, **i32), torch.full((B,), min(tokens // B, 30), **i32)
    p = ob.paged_plan(table, cached, fresh, free, n_free, 8, tokens, want_slots=slots)
    for name in ("lengths", "starts", "n_free"):
        assert p[name].untyped_storage().nbytes() <= 2 ** 16 + 4 * (2 * B + 2)
    n = int(fresh[0])
    assert torch.equal(p["lengths"], fresh) and p["starts"].tolist() == [n * b for b in range(B + 1)] and int(p["n_free"]) == 4 * B - B * -(-n // 8)
    assert torch.equal(p["positions"][0, :B * n], torch.arange(n, **i32).repeat(B)) and torch.equal(p["seq"][0, :B * n], torch.arange(B, **i32).repeat_interleave(n))
    assert bool((p["positions"][0, B * n:] == -1).all()) and bool((p["seq"][0, B * n:] == -1).all())
    if slots:
        want = table.repeat_interleave(n, 0).gather(1, (p["positions"][0, :B * n] // 8)[:, None].long())[:, 0].long() * 8 + p["positions"][0, :B * n] % 8
        assert torch.equal(p["slots"][:B * n], want) and bool((p["slots"][B * n:] == -1).all())
