"""Requests of an attention call that pass the bounds the caller gave."""
import math

import numpy as np
import pytest
import torch

from lm_util import DEV, HALF, U, within
from serve_util import Cache, attention, rng, table_of, typed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("news,max_q", [([1000, 100], 100), ([40, 1000, 90, 3], 90), ([9, 1, 3, 2], 3), ([70, 6, 1, 2], 6), ([5, 64, 64], 64), ([5, 1, 3], 3)])
def test_requests_beyond_max_q_leave_the_others_alone(news, max_q):
    """A request of more new tokens than max_q sets the status and is left out: its
    rows keep what they held, every other request's rows are computed.  Bounds as in
    test_gpu_kv4_weights.py."""
    from paper_2011_14504_amd import iseg
    H, Hq, D, page = 1, 2, 64, 16
    kvs = [n + 30 * b for b, n in enumerate(news)]
    held = [-(-kv // page) for kv in kvs]
    P = sum(held)
    cache = Cache(51, P, H, D, page)
    table = table_of(52, held, P, max(held))
    start = np.concatenate(([0], np.cumsum(news))).astype(np.int32)
    qg, qd = typed(rng(53).standard_normal((start[-1], Hq, D)), "bf16")
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.full((int(start[-1]), Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.from_numpy(start).to(DEV), torch.tensor(kvs, dtype=torch.int32, device=DEV),
                       max_q=max_q, out=out, status=st)
    assert iseg.iseg_status_read(st) == (iseg.ISEG_DEV_RANGE if max(news) > max_q else 0)
    for b, n in enumerate(news):
        rows = slice(int(start[b]), int(start[b + 1]))
        if n > max_q:
            assert (out[rows] == 7).all()
            continue
        o, _, s, reach, far = attention(qd[rows], cache, table[b:b + 1], [0, n], [kvs[b]], H, 1 / math.sqrt(D), True, 0)
        eps = 2 * (D + 16) * U * reach + 2.0 ** -25 * far + 4 * U
        tol = (2 * eps[..., None] + 2.0 ** -21 + 40 * U) * s + (HALF["bf16"] + 4 * U) * np.abs(o) + kvs[b] * 7 * 2.0 ** -31 * float(cache.vs.max())
        within(out[rows], torch.from_numpy(o), torch.from_numpy(tol), (news, b))
