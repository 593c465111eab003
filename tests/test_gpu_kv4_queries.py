"""Queries of the attention over the 4-bit cache whose elements are far apart: what
their float16 terms keep, against the formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

from lm_util import DEV, HALF, U, within
from serve_util import Cache, attention, rng, table_of, typed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("loud", [2.0 ** 12, 2.0 ** 18, 2.0 ** 24])
@pytest.mark.parametrize("n,kv,Hq,H,D", [(1, 300, 4, 1, 64), (6, 90, 8, 2, 128), (90, 200, 2, 1, 96), (140, 140, 4, 2, 128), (1, 2, 2, 2, 256)])
def test_small_elements_beside_large_ones(n, kv, Hq, H, D, loud, t):
    """Every key is 0 where a query's elements are large, so that its small ones make
    the score.  A score is off by 2 (D + 16) U of its terms (float32's two terms, 2^-23 of
    an element, among them), 2^-39 of the largest element per key element, and its
    exponential's 4 U; a weight by that above and below the fraction, and by 2^-21."""
    from paper_2011_14504_amd import iseg
    held = -(-kv // 16)
    cache = Cache(41, held, H, D, 16)
    cache.kn[..., 1:D:9] = 0
    table = table_of(42, [held], held, held)
    x = rng(43).standard_normal((n, Hq, D))
    x[..., 1::9] *= loud
    qg, qd = typed(x, t)
    out, lse = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV),
                                  torch.tensor([kv], dtype=torch.int32, device=DEV))
    o, l, s, reach, far = attention(qd, cache, table, [0, n], [kv], H, 1 / math.sqrt(D), True, 0)
    eps = 2 * (D + 16) * U * reach + 2.0 ** -39 * far + 4 * U
    within(lse, torch.from_numpy(l), torch.from_numpy(eps + 4 * U * np.abs(l) + (30 + math.log2(kv + 1)) * U), "lse")
    tol = (2 * eps[..., None] + 2.0 ** -21 + 40 * U) * s + (HALF[t] + 4 * U) * np.abs(o) + kv * 7 * 2.0 ** -31 * float(cache.vs.max())
    within(out, torch.from_numpy(o), torch.from_numpy(tol), "out")


@pytest.mark.parametrize("t", ["bf16", "fp32"])
def test_small_queries_and_large_keys(t):
    """Scores of ordinary size from queries of 2^-100 and scales of k of 2^110, and
    the other way round."""
    from paper_2011_14504_amd import iseg
    D, kv, n = 64, 150, 3
    for e in (100, -60):
        cache = Cache(44, 10, 1, D, 16)
        cache.ks *= np.float32(2.0 ** (e + 10))
        table = table_of(45, [10], 10, 10)
        qg, qd = typed(rng(46).standard_normal((n, 2, D)) * 2.0 ** (-e - 10), t)
        out, lse = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV),
                                      torch.tensor([kv], dtype=torch.int32, device=DEV))
        o, l, s, reach, far = attention(qd, cache, table, [0, n], [kv], 1, 0.125, True, 0)
        eps = 2 * (D + 16) * U * reach + 2.0 ** -25 * far + 4 * U
        within(lse, torch.from_numpy(l), torch.from_numpy(eps + 4 * U * np.abs(l) + (30 + math.log2(kv + 1)) * U), ("lse", e))
        tol = (2 * eps[..., None] + 2.0 ** -11 + 40 * U) * s + (HALF[t] + 4 * U) * np.abs(o) + kv * 7 * 2.0 ** -31 * float(cache.vs.max())
        within(out, torch.from_numpy(o), torch.from_numpy(tol), ("out", e))
