"""Attention over a paged cache with bf16 I/O: every element of the result within the roundings of its exact interval (tests/decode_bounds.py), so
that a value that is lost or out of its place shows however long the row is."""
import math

import pytest
import torch

from tests import heads_reference as ref
from tests.decode_bounds import outside, paged
from tests.test_gpu_paged import DECODE, MANY, call, make_decode

pytestmark = pytest.mark.gpu
CASES = [c for c in DECODE + MANY if c.get("io", "bf16") == "bf16"] + [
    dict(lengths=[1531], Hq=16, Hk=4, K=256, page=16),
    dict(lengths=[4000, 900, 2049], Hq=8, Hk=4, K=128, page=64, order="token"),
    dict(lengths=[3000], Hq=4, Hk=2, K=64, page=32, spread=0.1),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for k, v in c.items() if k != "lengths" or len(v) < 9))
def test_every_element(case):
    x = make_decode(**case)
    B, K = x["q"].shape[0], x["q"].shape[2]
    want, e = paged(ref.f64(x["q"]), ref.f64(x["kc"]), ref.f64(x["vc"]), x["table"].cpu(), x["lengths"].cpu(), torch.arange(B), K ** -0.5, x["window"])
    for shares in (x["shares"], -1, 1, 3, 1000):
        o, _ = call(dict(x, shares=shares))
        bad = outside(o.double().cpu(), want, e)
        assert not bad.any(), f"shares {shares}: {int(bad.sum())} of {bad.numel()} outside"


@pytest.mark.parametrize("K", [64, 128, 256])
def test_a_value_that_is_infinite(K):
    """Where it is seen the result is infinite too, in its column alone."""
    x = make_decode([70, 41], 4, 2, K, 16)
    want, _ = call(x)
    for at, value in (((0, 3), math.inf), ((1, 40), -math.inf)):
        x["vc"][x["table"][at[0], at[1] // 16].long(), at[1] % 16, 1, 5] = value
    o, _ = call(x)
    assert bool((o[0, 2:, 5] == math.inf).all()) and bool((o[1, 2:, 5] == -math.inf).all())
    o[:, 2:, 5] = want[:, 2:, 5]
    assert torch.equal(o, want)
