"""Attention over the 4-bit cache where blocks have long loops: so many requests and
heads that no request is split, and more keys than one look-up of the block table has."""
import math

import numpy as np
import pytest
import torch

from lm_util import DEV, HALF, U, within
from serve_util import Cache, rng, typed

pytestmark = pytest.mark.gpu


def _formula(q, K, V, vs, n, causal, window, scale):
    """q [H, G n, D] (a head's queries of token 0 first), K and V [H, kv, D], vs [H, kv]
    the scales of V, in 64 bits: out, lse, and the bounds size, reach, far, top."""
    kv = K.shape[1]
    pos = (kv - n + torch.arange(q.shape[1]) // (q.shape[1] // n))[:, None]
    j = torch.arange(kv)[None]
    hide = ((j > pos) if causal else torch.zeros_like(j > pos)) | ((j <= pos - window) if window else torch.zeros_like(j > pos))
    s = (scale * (q @ K.transpose(1, 2).contiguous())).masked_fill(hide, -math.inf)
    p = torch.softmax(s, -1)
    return (p @ V, torch.logsumexp(s, -1), p @ V.abs(), scale * (q.abs() @ K.abs().transpose(1, 2).contiguous()).amax(-1),
            scale * q.abs().amax(-1) * K.abs().sum(-1).amax(-1)[:, None], (p * vs[:, None]).amax(-1))


# B H of 2048 and more requests and heads: twice as many blocks as may be resident (256
# times up to 4), so one split; a step is 128 keys, 32 steps a look-up, so that 4300 keys
# need a second one.  G n rows: up to 16, 32 and 64 (float32 32) by one kernel each.
@pytest.mark.parametrize("B,H,G,n,D,t,causal,window", [
    (128, 16, 4, 1, 128, "bf16", True, 0), (128, 16, 1, 1, 32, "fp16", True, 0), (128, 16, 4, 1, 64, "fp32", True, 0), (256, 8, 8, 2, 64, "bf16", True, 0),
    (128, 16, 20, 1, 64, "bf16", True, 0), (128, 16, 10, 3, 128, "fp32", True, 0), (128, 16, 40, 1, 64, "bf16", True, 0), (128, 16, 13, 4, 128, "fp16", True, 0),
    (128, 16, 4, 1, 64, "bf16", True, 4400), (128, 16, 4, 3, 64, "fp16", False, 0), (128, 16, 2, 2, 96, "bf16", False, 4300), (128, 16, 2, 1, 256, "bf16", True, 0),
    (128, 16, 2, 1, 192, "fp32", True, 0)])
def test_long_loops(B, H, G, n, D, t, causal, window):
    """Bounds as in test_gpu_kv4_weights.py: a score's eps twice, weights by two terms,
    2^-34 of a row's largest weight times scale for each key and code, the output's rounding."""
    from paper_2011_14504_amd import iseg
    assert B * H >= 2048
    r, page, P = rng(B + G + D), 64, 90
    cache = Cache(D + G, P, H, D, page)
    kvs = [int(r.integers(n, 400)) for _ in range(B)]
    for b, kv in zip(r.permutation(B), (4300, 4481, 5000, 5247, 4097, 4096)):
        kvs[b] = kv
    # requests share pages, as those with one beginning do
    table = np.full((B, 83), -1, dtype=np.int32)
    for b, kv in enumerate(kvs):
        table[b, :-(-kv // page)] = r.permutation(P)[:-(-kv // page)]
    # scores that grow over the keys now and then, so that the running maximum moves late
    cache.ks *= np.where(r.random(cache.ks.shape) < 0.002, 4, 1).astype(np.float32)
    qg, qd = typed(rng(7).standard_normal((B * n, H * G, D)), t)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.arange(B + 1, dtype=torch.int32, device=DEV) * n,
                                  torch.tensor(kvs, dtype=torch.int32, device=DEV), causal=causal, window=window, max_q=n, max_kv=max(kvs), status=st)
    assert iseg.iseg_status_read(st) == 0
    K = torch.from_numpy(cache.kn[..., :D] * cache.ks.astype(np.float64)[..., None])
    V = torch.from_numpy(cache.vn[..., :D] * cache.vs.astype(np.float64)[..., None])
    vs = torch.from_numpy(cache.vs.astype(np.float64))
    out, lse, scale = out.cpu(), lse.cpu(), 1 / math.sqrt(D)
    for b, kv in enumerate(kvs):
        pages = torch.from_numpy(table[b, :-(-kv // page)]).long()
        rows = lambda x: x[pages].transpose(0, 1).flatten(1, 2)[:, :kv]  # noqa: E731
        q = torch.from_numpy(qd[b * n:(b + 1) * n]).reshape(n, H, G, D).transpose(0, 1).reshape(H, n * G, D)
        o, l, size, reach, far, top = _formula(q, rows(K), rows(V), rows(vs), n, causal, window, scale)
        eps = 2 * (D + 16) * U * reach + 2.0 ** -39 * far + 4 * U
        tol = (2 * eps + 2.0 ** -21 + 40 * U)[..., None] * size + (HALF[t] + 4 * U) * o.abs() + (kv * 7 * 2.0 ** -34 * top)[..., None] + (2.0 ** -24 if t == "fp16" else 0)
        mine = lambda x: x[b * n:(b + 1) * n].reshape(n, H, G, -1).transpose(0, 1).reshape(H, n * G, -1)  # noqa: E731
        within(mine(out), o, tol, ("out", b, kv))
        within(mine(lse)[..., 0], l, eps + 4 * U * l.abs() + (30 + math.log2(kv + 1)) * U, ("lse", b, kv))
