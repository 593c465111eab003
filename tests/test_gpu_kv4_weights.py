"""Softmax weights of the attention over the 4-bit cache: what their float16 terms
leave off, against the formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

from lm_util import DEV, HALF, U, within
from serve_util import Cache, attention, rng, table_of, typed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,kv,Hq,H,D", [(1, 300, 8, 2, 128), (1, 3000, 4, 1, 64), (9, 200, 8, 1, 96), (150, 420, 4, 2, 128), (300, 300, 2, 1, 256), (1, 2, 4, 4, 32)])
@pytest.mark.parametrize("size", [0.01, 0.3, 3.0])
def test_bfloat16_is_off_by_its_own_rounding(n, kv, Hq, H, D, size):
    """bfloat16 outputs: a score's error eps (2 (D + 16) U of its terms, 2^-25 of the
    query's largest element per key element, the exponential's), twice; a weight's two
    float16 terms 2^-21 and its float32 steps; at least 2^-31 of the largest scale times a
    code of up to 7; and the output's one rounding."""
    from paper_2011_14504_amd import iseg
    held = -(-kv // 32)
    cache = Cache(6, held, H, D, 32)
    table = table_of(7, [held], held, held)
    qg, qd = typed(size * rng(8).standard_normal((n, Hq, D)), "bf16")
    scale = 1 / math.sqrt(D)
    out, _ = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV),
                                torch.tensor([kv], dtype=torch.int32, device=DEV))
    o, _, s, reach, far = attention(qd, cache, table, [0, n], [kv], H, scale, True, 0)
    eps = 2 * (D + 16) * U * reach + 2.0 ** -25 * far + 4 * U
    tol = (2 * eps[..., None] + 2.0 ** -21 + 40 * U) * s + (HALF["bf16"] + 4 * U) * np.abs(o) + kv * 7 * 2.0 ** -31 * float(cache.vs.max())
    within(out, torch.from_numpy(o), torch.from_numpy(tol), "out")
