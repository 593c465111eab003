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


def _row(cache, table, x, h, scale, lo, hi):
    """One query over keys [lo, hi) of a request in 64 bits: its output and the bounds
    size = sum p |v|, reach and far as in serve_util.attention, top = max p_j scale of v_j."""
    K, V = cache.rows(table, hi, h)
    K, V = K[lo:], V[lo:]
    s = scale * (K @ x)
    p = np.exp(s - s.max())
    z = p.sum()
    vs = cache.vs[table][:, h].reshape(-1)[lo:hi].astype(np.float64)
    return ((p / z) @ V, (p / z) @ np.abs(V), scale * (np.abs(K) @ np.abs(x)).max(), scale * np.abs(x).max() * np.abs(K).sum(1).max(),
            (p / z * vs).max(), s.max() + math.log(z))


def _rows_close(got, cache, table, q, kv, H, window, t, what):
    """Every row's weights have the precision of its own: a score's error eps twice, two
    terms 2^-21, the float32 steps, and 2^-34 of the row's largest weight times scale for
    each key and a code of up to 7."""
    n, Hq, D = q.shape
    scale = 1 / math.sqrt(D)
    for i in range(n):
        pos = kv - n + i
        lo = max(0, pos + 1 - window) if window else 0
        for h in range(Hq):
            o, size, reach, far, top, _ = _row(cache, table, q[i, h], h * H // Hq, scale, lo, pos + 1)
            eps = 2 * (D + 16) * U * reach + 2.0 ** -25 * far + 4 * U
            tol = (2 * eps + 2.0 ** -21 + 40 * U) * size + (HALF[t] + 4 * U) * np.abs(o) + (pos + 1 - lo) * 7 * 2.0 ** -34 * top
            within(got[i, h], torch.from_numpy(o), torch.from_numpy(tol), (what, i, h))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("n,kv,Hq,H,D,window", [(5, 5, 4, 1, 64, 0), (40, 40, 2, 1, 128, 0), (100, 100, 4, 2, 64, 0), (130, 130, 2, 1, 256, 0), (7, 300, 4, 1, 64, 9),
                                                (200, 500, 2, 1, 128, 33), (3, 2500, 4, 1, 32, 2)])
def test_a_rows_weights_do_not_depend_on_other_keys(n, kv, Hq, H, D, window, t):
    """Scales of v that grow from 2^-60 to 2^40 over the tokens: an early query sees
    small ones only, whatever comes after it."""
    from paper_2011_14504_amd import iseg
    page, held = 16, -(-kv // 16)
    cache = Cache(31, held, H, D, page)
    table = table_of(32, [held], held, held)
    grow = np.exp2(np.linspace(-60, 40, held * page)).astype(np.float32).reshape(held, page)
    cache.vs[table[0]] *= grow[:, None]
    qg, qd = typed(rng(33).standard_normal((n, Hq, D)), t)
    out, _ = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV),
                                torch.tensor([kv], dtype=torch.int32, device=DEV), window=window)
    _rows_close(out, cache, table[0], qd, kv, H, window, t, (n, kv))


@pytest.mark.parametrize("t", ["bf16", "fp32"])
@pytest.mark.parametrize("n,kv,D", [(1, 300, 64), (3, 90, 128), (70, 400, 64), (1, 5000, 32)])
@pytest.mark.parametrize("small", [2.0 ** -45, 2.0 ** -60])
def test_a_small_value_with_all_the_weight(n, kv, D, small, t):
    """One key has nearly all of the weight and a value far below the others'."""
    from paper_2011_14504_amd import iseg
    page, held, at = 16, -(-kv // 16), 13
    cache = Cache(34, held, 1, D, page)
    table = table_of(35, [held], held, held)
    sign = np.where(rng(36).random(D) < 0.5, -1.0, 1.0)
    where = table[0, at // page], 0, at % page
    cache.kn[..., :D] = np.clip(cache.kn[..., :D], -2, 2)
    cache.kn[where][:D] = 7 * sign
    cache.ks[...] = 0.25
    cache.vs[where] = small
    # the key's score is 7 D / 4 q scale = 7 sqrt(D) q / 4, the others' a seventh of it at
    # most in all, nearer to 0 by far: q so that it is 90
    x = np.tile(90 / (7 * math.sqrt(D) / 4) * sign, (n, 2, 1)) * (1 + 0.01 * rng(37).random((n, 2, D)))
    qg, qd = typed(x, t)
    out, _ = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV),
                                torch.tensor([kv], dtype=torch.int32, device=DEV))
    assert (out.abs().amax(-1) > 0).all()
    _rows_close(out, cache, table[0], qd, kv, 1, 0, t, (n, kv))
