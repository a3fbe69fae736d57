"""The interval of tests/decode_bounds.py, on the CPU: it holds for the arithmetic that it is derived from, and values out of their place fall out of it."""
import pytest
import torch

from tests.decode_bounds import attention, outside


def _row(n, K=128):
    g = torch.Generator().manual_seed(n)
    q = (2.0 * torch.randn(K, generator=g)).bfloat16().double()
    k, v = (torch.randn(n, K, generator=g).bfloat16().double() for _ in range(2))
    return q, k, v, K ** -0.5


def _two_parts(p):
    """A weight as the sum of two bf16 numbers: the bits of the number below it, cut off, and the rest rounded."""
    bits = p.float().view(torch.int32)
    first = ((bits - 1).clamp(min=0) & -65536).view(torch.float32)
    return first.double() + (p.float() - first).bfloat16().double()


@pytest.mark.parametrize("n", [1, 33, 1531, 20000])
def test_what_the_interval_holds_and_what_not(n):
    q, k, v, scale = _row(n)
    want, e = attention(q, k, v, scale)
    s = scale * (k @ q)
    p = torch.exp(s - s.max())
    rounded = lambda x: x.float().bfloat16().double()
    assert not outside(rounded(_two_parts(p) @ v / p.sum()), want, e).any()
    if n == 1:
        return
    for moved in (torch.zeros_like(v[:128]), v[:128].flip(0)):         # a unit of tokens whose values are lost, or not in their order
        w = v.clone()
        w[:128] = moved[: len(w)]
        assert outside(rounded(p @ w / p.sum()), want, e).any()


def test_two_parts_of_a_weight():
    p = torch.rand(100000, generator=torch.Generator().manual_seed(1), dtype=torch.float64).float().double()
    p = torch.cat([p, 2.0 ** -torch.arange(0, 100, dtype=torch.float64), torch.zeros(1, dtype=torch.float64)])
    assert ((_two_parts(p) - p).abs() <= 2.0 ** -16 * p).all()
