"""The values that reading the 4-bit cache gives: code times scale in float32, rounded to
the type that was asked for."""
import numpy as np
import pytest
import torch

from lm_util import DEV, DT
from serve_util import Cache, rng

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("repeat", [1, 32])
def test_values_are_rounded_to_float32_first(t, repeat):
    """Scales whose products with some code fall on a half-step of the type once they
    are float32, few tokens (one at a time) and many (four at a time)."""
    from paper_2011_14504_amd import iseg
    P, page, D = 16, 16, 64
    s = np.exp2(rng(1).uniform(-8, 8, 12_000_000)).astype(np.float32)
    tie = np.zeros(len(s), bool)
    bits = {"fp16": 13, "bf16": 16, "fp32": 0}[t]                 # of float32's mantissa that the type has not
    for n in (3, 5, 6, 7):
        p = s * np.float32(n)
        tie |= (p.astype(np.float64) != s.astype(np.float64) * n) & ((p.view(np.uint32) & ((1 << bits) - 1)) == (1 << bits >> 1))
    s = s[tie][:P * page]
    assert len(s) == P * page
    cache = Cache(2, P, 1, D, page)
    cache.ks[...] = s.reshape(P, 1, page)
    cache.vs[...] = s[::-1].reshape(P, 1, page)
    slots = np.tile(np.arange(P * page), repeat)
    assert (len(slots) >= 8192) == (repeat > 1)
    k, v = iseg.kv4_read(torch.from_numpy(slots).to(DEV), cache.gpu(), D, DT[t])
    for got, n, sc in ((k, cache.kn, cache.ks), (v, cache.vn, cache.vs)):
        want = (n[:, 0, :, :D].astype(np.float32) * sc[:, 0, :, None]).reshape(-1, 1, D)
        assert torch.equal(got.cpu(), torch.from_numpy(want).to(DT[t]).repeat(repeat, 1, 1))
