"""Codes of keys that fp32 does not settle: codes and scales are those of the definition in 64 bits, to the bit."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import heads_reference as ref
from tests import pages_reference as pages
from tests.test_gpu_paged_mx import make_cache, make_table

pytestmark = pytest.mark.gpu


def append(k, table_of_angles=None, weight=None, norm="none", interleaved=False):
    """(what the cache holds, what it is to hold), codes and scales of the tokens' keys; and the keys in 64 bits."""
    T, K = k.shape[1], k.shape[3]
    g = torch.Generator(device="cuda").manual_seed(1)
    table, n_pages = make_table([T], 16, 0, 2)
    pos = torch.arange(T, dtype=torch.int32)[None]
    cache = make_cache(g, n_pages, 16, k.shape[2], K)
    hp = ob.NormHyper(norm=norm, interleaved=interleaved)
    ob.paged_append_mx(k, torch.zeros_like(k), cache, table.cuda(), pos.cuda(), weight_k=weight, rotary=table_of_angles, hp=hp)
    z = ref.norm_rows(ref.f64(k), ref.f64(weight), ref.f64(table_of_angles), pos.long(), norm, hp.eps, interleaved)
    at = table[0, pos[0].long() // 16].long(), pos[0].long() % 16
    return [cache[i].cpu()[at] for i in (0, 2)], [x[0] for x in pages.pack(z)], z


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("K", [64, 128, 256])
def test_signs_of_elements_that_cancel(K, interleaved):
    g = torch.Generator().manual_seed(7)
    T, half = 40, K // 2
    x, c, s = (torch.rand(T, half, generator=g) + 0.5 for _ in range(3))
    y = (x.double() * c.double() / s.double()).float()                  # x c - y s is what the rounding of y leaves
    y[:, ::32] = 0.25                                                   # (and one of a block that is not small)
    sums = x.double() * c.double() - y.double() * s.double()            # (exact: 48 bits each, and close to each other)
    in_32_bits = (x.double() * c.double() - (y * s).double()).float()
    flips = (torch.signbit(sums) != torch.signbit(in_32_bits)) & (sums != 0)
    assert int(flips.sum()) > T
    k = torch.stack([x, y], dim=-1).flatten(1) if interleaved else torch.cat([x, y], dim=1)
    got, want, z = append(k[None, :, None].cuda(), torch.cat([c, s], dim=1).cuda(), interleaved=interleaved)
    assert torch.equal(z[0, :, 0, 0::2] if interleaved else z[0, :, 0, :half], sums)
    assert torch.equal(got[1], want[1]) and torch.equal(got[0], want[0])


@pytest.mark.parametrize("rotary", [0, 64])
@pytest.mark.parametrize("size,weight", [(48, -95), (49, -85), (-20, -125), (0, -60), (0, -61)])
def test_weights_next_to_the_smallest_numbers(size, weight, rotary):
    """The factor of a row times a weight is below 2^-126 in fp32, where a product keeps a few of its digits."""
    g = torch.Generator(device="cuda").manual_seed(3)
    k = torch.randn(1, 64, 4, 64, device="cuda", generator=g) * 2.0 ** size
    w = (1 + torch.randn(64, device="cuda", generator=g) / 8) * 2.0 ** weight
    w[5] = 0.0
    got, want, z = append(k, ob.rotary_table(64, rotary) if rotary else None, w, "rms")
    # (size -20: eps, 2^-20, makes the factor of a row 2^10, and keys of 2^-135 are below the least scale's codes)
    assert (float(z.abs().amax()) > 2.0 ** -118 and int((got[0] & 7).sum()) > 0) == (size >= 0)
    assert torch.equal(got[1], want[1]) and torch.equal(got[0], want[0])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("least", [0, -100, -130, -145])
def test_signs_of_the_smallest_elements_that_cancel(least, interleaved):
    """Products that fp32 rounds to a multiple of 2^-149 or to zero: the sign of what is left of two of them."""
    g = torch.Generator().manual_seed(11)
    T, half = 40, 32
    x, c, s = (torch.rand(T, half, generator=g) + 0.5 for _ in range(3))
    x = torch.ldexp(x, torch.tensor(float(least))).float()
    y = (x.double() * c.double() / s.double()).float()
    y[:, 0] = 0.25                                                      # (a block that is not small)
    y[::2, 1::4], x[1::2, 2::4] = 0.0, 0.0                              # nothing to cancel, and nothing at all
    x[::2, 1::8] = 0.0
    sums = x.double() * c.double() - y.double() * s.double()
    k = torch.stack([x, y], dim=-1).flatten(1) if interleaved else torch.cat([x, y], dim=1)
    got, want, z = append(k[None, :, None].cuda(), torch.cat([c, s], dim=1).cuda(), interleaved=interleaved)
    assert torch.equal(z[0, :, 0, 0::2] if interleaved else z[0, :, 0, :half], sums)
    assert torch.equal(got[1], want[1]) and torch.equal(got[0], want[0])
