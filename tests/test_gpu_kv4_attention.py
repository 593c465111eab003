"""Attention over the 4-bit cache against its formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

from lm_util import DEV, DT, HALF, U, normal, within
from serve_util import Cache, attention, rng, table_of, typed

pytestmark = pytest.mark.gpu

# Bounds.  A score's sum of D products has an error of 2 U (a matrix
# instruction may cut where it could round) D relative to reach = scale sum |q k|,
# its factors and the argument of its exponential a few more, q's placement in
# float16 2^-25 far, far = scale max |q| sum |k| (two terms for float32: 4 U reach
# as well): eps_s.  A weight's relative error is that plus 2^-23 of the
# exponential, once above and once below the fraction, and half a step of
# float16, 2^-11 (float32: two terms, 2^-21), relative to size = sum p |v|.  Small
# weights are off by 2^-31 of the largest scale of v per key, times a code of up
# to 7.  The output is rounded once.  lse has eps_s and the roundings of its sum.


def _check(out, lse, want, t, D, keys, top, what):
    o, l, size, reach, far = want
    eps = 2 * (D + 16) * U * reach + 2.0 ** -25 * far + 4 * U
    p = 2.0 ** -21 if t == "fp32" else 2.0 ** -11
    tol = (2 * eps[..., None] + p + 40 * U) * size + (HALF[t] + 4 * U) * np.abs(o) + keys * 7 * 2.0 ** -31 * top + (2.0 ** -24 if t == "fp16" else 0)
    within(out, torch.from_numpy(o), torch.from_numpy(tol), what + " out")
    fin = np.isfinite(l)
    tol = np.where(fin, eps + 4 * U * np.abs(np.where(fin, l, 0)) + (30 + math.log2(keys + 1)) * U, 0)
    within(lse, torch.from_numpy(l), torch.from_numpy(tol), what + " lse")


def _run(seed, news, kvs, Hq, H, D, page, t, causal=True, window=0, scale=None, bounds=True, lead=0, tail=0, size=1.0, spread=0.0):
    from paper_2011_14504_amd import iseg
    held = [-(-kv // page) for kv in kvs]
    P = sum(held) + 2
    cache = Cache(seed, P, H, D, page, spread=spread)
    table = table_of(seed + 1, held, P, max(held + [1]) + 1)
    # slots that hold no token: scales of NaN, codes of anything
    for b, kv in enumerate(kvs):
        if kv % page:
            cache.ks[table[b, held[b] - 1], :, kv % page:] = np.nan
            cache.vs[table[b, held[b] - 1], :, kv % page:] = np.nan
    start = np.concatenate(([0], np.cumsum(news))).astype(np.int32) + lead
    T = int(start[-1]) + tail
    qg, qd = typed(size * rng(seed + 2).standard_normal((T, Hq, D)), t)
    scale = scale or 1 / math.sqrt(D)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.full((T, Hq, D), 7.0, dtype=DT[t], device=DEV)
    kw = dict(max_q=max(max(news), 1), max_kv=max(max(kvs), 1)) if bounds else {}
    got, lse = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.from_numpy(start).to(DEV),
                                  torch.tensor(kvs, dtype=torch.int32, device=DEV), scale=scale, causal=causal, window=window, out=out,
                                  status=st, **kw)
    assert got is out and iseg.iseg_status_read(st) == 0
    want = attention(qd, cache, table, start, kvs, H, scale, causal, window)
    mine = slice(lead, T - tail)
    assert (out[:lead] == 7).all() and (out[T - tail:] == 7).all()
    _check(out[mine], lse[mine], [w[mine] for w in want], t, D, max(kvs), float(np.nanmax(cache.vs)), str((news, kvs)))


SINGLE = [([1], [1], 1, 1, 64, 16), ([1], [15], 4, 2, 64, 16), ([1], [16], 4, 4, 128, 16), ([1], [17], 8, 1, 128, 16), ([1], [31], 3, 1, 96, 48),
          ([1], [32], 16, 1, 128, 64), ([1], [33], 6, 2, 80, 32), ([1, 1, 1], [127, 128, 129], 8, 2, 128, 64), ([1, 1], [700, 3], 8, 2, 128, 16),
          ([1], [2500], 4, 1, 32, 16), ([1, 0, 1], [200, 90, 0], 7, 1, 192, 16), ([1, 1], [400, 513], 20, 1, 256, 256), ([1], [300], 2, 2, 8, 16),
          ([1], [260], 2, 1, 24, 16), ([1, 1], [90, 300], 4, 2, 136, 80), ([1], [1300], 40, 1, 64, 32), ([1, 1, 1, 1], [5000, 1, 40, 600], 8, 2, 64, 16),
          ([1], [450], 33, 1, 256, 16)]


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", SINGLE)
def test_single_tokens(case, t):
    _run(len(str(case)), *case, t)


SEVERAL = [([5, 3], [5, 3], 4, 2, 64, 16), ([4, 4, 4], [100, 33, 64], 8, 2, 128, 16), ([2, 9], [300, 9], 8, 1, 128, 64), ([8], [1030], 8, 2, 96, 32),
           ([16, 1, 0, 5], [16, 70, 4, 200], 2, 2, 64, 48), ([3], [2], 4, 1, 64, 16), ([7, 2], [0, 5], 2, 1, 128, 16), ([64], [64], 1, 1, 32, 16),
           ([33, 1], [500, 90], 4, 4, 192, 16), ([17], [40], 8, 2, 256, 64)]
PROMPTS = [([70], [70], 4, 2, 64, 16), ([129], [129], 2, 1, 128, 16), ([200, 1, 65, 0, 9], [200, 600, 300, 8, 9], 4, 2, 128, 64), ([130], [900], 3, 1, 96, 48),
           ([64, 64], [64, 100], 8, 4, 32, 32), ([90], [250], 4, 1, 256, 16), ([150], [40], 2, 2, 80, 16), ([257], [257], 1, 1, 192, 128)]


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("case", SEVERAL + PROMPTS)
def test_several_tokens(case, t):
    _run(len(str(case)) + 7, *case, t, lead=3, tail=5)


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 7), (True, 40), (True, 10000), (False, 33), (True, 64)])
@pytest.mark.parametrize("case", [([1, 1], [300, 20], 8, 2, 128, 16), ([6, 3], [333, 70], 4, 2, 64, 32), ([100, 2], [400, 50], 2, 1, 128, 64), ([90], [30], 4, 1, 64, 16)])
def test_masks(case, causal, window):
    _run(5, *case, "bf16", causal=causal, window=window)


@pytest.mark.parametrize("case", [([1, 1], [700, 30], 8, 2, 128, 16), ([40, 3], [200, 70], 4, 2, 64, 32)])
def test_without_bounds(case):
    _run(6, *case, "bf16", bounds=False, tail=2)


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("size", [1e-3, 30.0, 3000.0])
def test_flat_and_sharp(t, size):
    """Scores near one another, and scores that leave one key."""
    _run(8, [2, 1], [150, 700], 4, 2, 64, 16, t, size=size)
    _run(9, [100], [300], 2, 1, 128, 16, t, size=size)


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
def test_values_of_very_different_size(t):
    """Scales of v over a factor of 2^20."""
    _run(10, [1, 4], [500, 300], 4, 2, 64, 16, t, spread=20.0)
    _run(11, [100], [300], 2, 1, 128, 16, t, spread=20.0)


def test_rows_of_other_sizes_stay_apart():
    """A row's queries of 2^-40 beside others of 2^40 have the precision of its own."""
    from paper_2011_14504_amd import iseg
    H, D, page, kv = 1, 64, 16, 90
    cache = Cache(3, 8, H, D, page)
    table = table_of(4, [6], 8, 6)
    qg, qd = typed(rng(5).standard_normal((1, 4, D)) * np.exp2([-40.0, 0, 30, 4])[None, :, None], "bf16")
    for scale in (0.125, 2.0 ** -30):
        out, lse = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.tensor([0, 1], dtype=torch.int32, device=DEV),
                                      torch.tensor([kv], dtype=torch.int32, device=DEV), scale=scale)
        want = attention(qd, cache, table, [0, 1], [kv], H, scale, True, 0)
        keep = want[3] < 1e4
        _check(out[torch.from_numpy(keep)], lse[torch.from_numpy(keep)], [w[keep] for w in want], "bf16", D, kv, cache.vs.max(), str(scale))


def test_not_a_number_where_it_is_seen():
    """A token of NaN reaches the rows that see it and no other; a query of NaN
    its own row."""
    from paper_2011_14504_amd import iseg
    H, D, page, n, kv = 1, 64, 16, 90, 100
    for which in ("ks", "vs"):
        cache = Cache(3, 8, H, D, page)
        table = table_of(4, [7], 8, 7)
        getattr(cache, which)[table[0, 50 // page], 0, 50 % page] = np.nan
        for rows in (n, 3):
            qg, qd = typed(rng(5).standard_normal((rows, 2, D)), "bf16")
            qg[1, 1, 3] = float("nan")
            out, lse = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.tensor([0, rows], dtype=torch.int32, device=DEV),
                                          torch.tensor([kv], dtype=torch.int32, device=DEV), window=60)
            pos = np.arange(kv - rows, kv)
            sees = torch.from_numpy((pos >= 50) & (pos - 60 < 50)).to(DEV)[:, None].expand(rows, 2).clone()
            sees[1, 1] = True
            assert torch.equal(torch.isnan(out).all(-1), sees) and torch.equal(torch.isnan(out).any(-1), sees)


def test_bad_tables_and_lengths():
    """Page ids outside the cache hide their keys, bounds that do not hold and
    wrong starts set the status; nothing is read or written beyond."""
    from paper_2011_14504_amd import iseg
    H, D, page = 2, 64, 16
    cache = Cache(3, 6, H, D, page)
    g = cache.gpu()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for n in (1, 5, 100):
        table = np.array([[0, 7, 2, -3, 4, 2 ** 30]], dtype=np.int32)
        qg, qd = typed(rng(5).standard_normal((n, 4, D)), "bf16")
        out, lse = iseg.kv4_attention(qg, g, torch.from_numpy(table).to(DEV), i32([0, n]), i32([90]), status=st)
        assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_RANGE
        iseg.iseg_status_clear(st)
        want = attention(qd, cache, table, [0, n], [90], H, 0.125, True, 0)
        _check(out, lse, want, "bf16", D, 90, cache.vs.max(), "bad pages")
    table = i32([[0, 1, 2], [3, 4, 5]])
    q = torch.ones(6, 4, D, dtype=torch.bfloat16, device=DEV)
    for start, kv, kw in (([0, 3, 6], [20, 60], {}), ([0, 3, 6], [20, -1], {}), ([0, 7, 6], [20, 20], {}), ([-1, 3, 6], [20, 20], {}),
                          ([0, 3, 9], [20, 20], {}), ([0, 3, 6], [20, 40], dict(max_kv=30)), ([0, 1, 6], [20, 20], dict(max_q=2))):
        iseg.kv4_attention(q, g, table, i32(start), i32(kv), status=st, **kw)
        assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_RANGE, (start, kv, kw)
        iseg.iseg_status_clear(st)


def test_nothing_to_see():
    """No tokens, no requests, no cached keys, an empty cache."""
    from paper_2011_14504_amd import iseg
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    c = iseg.kv4_cache(4, 2, 64, 16, DEV)
    q = torch.ones(3, 4, 64, dtype=torch.bfloat16, device=DEV)
    out, lse = iseg.kv4_attention(q, c, i32([[0], [1]]), i32([0, 2, 3]), i32([0, 0]))
    assert (out == 0).all() and (lse == -math.inf).all()
    out, lse = iseg.kv4_attention(q, iseg.kv4_cache(0, 2, 64, 16, DEV), i32([[0], [1]]), i32([0, 2, 3]), i32([0, 0]))
    assert (out == 0).all() and (lse == -math.inf).all()
    out, lse = iseg.kv4_attention(q, c, torch.empty(2, 0, dtype=torch.int32, device=DEV), i32([0, 2, 3]), i32([0, 0]))
    assert (out == 0).all() and (lse == -math.inf).all()
    out, _ = iseg.kv4_attention(q[:0], c, i32([[0]]), i32([0, 0]), i32([5]))
    assert out.shape == (0, 4, 64)
    mine = torch.full_like(q, 3.0)
    iseg.kv4_attention(q, c, torch.empty(0, 4, dtype=torch.int32, device=DEV), i32([0]), torch.empty(0, dtype=torch.int32, device=DEV), out=mine)
    assert (mine == 3).all()


def test_strides_of_queries_and_outputs():
    from paper_2011_14504_amd import iseg
    H, D, page = 2, 64, 16
    cache = Cache(3, 9, H, D, page)
    table = torch.from_numpy(table_of(4, [5, 3], 9, 5)).to(DEV)
    wide = torch.full((2, 9), 99, dtype=torch.int32, device=DEV)
    wide[:, 2:7] = table
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    for n in (1, 70):
        qkv = torch.from_numpy(rng(5).standard_normal((2 * n, 9, D + 5))).to(torch.bfloat16).to(DEV)
        q = qkv[:, 1:5, 3:D + 3]
        args = (i32([0, n, 2 * n]), i32([80, 41]))
        want, wl = iseg.kv4_attention(q.contiguous(), cache.gpu(), table, *args)
        got, gl = iseg.kv4_attention(q, cache.gpu(), wide[:, 2:7], *args)
        assert torch.equal(got, want) and torch.equal(gl, wl)
        buf = torch.full((2 * n, 7, D + 3), 5.0, dtype=torch.bfloat16, device=DEV)
        out, none = iseg.kv4_attention(q, cache.gpu(), table, *args, out=buf[:, 2:6, 1:D + 1], want_lse=False)
        assert none is None and torch.equal(out, want)
        buf[:, 2:6, 1:D + 1] = 5.0
        assert (buf == 5).all()
        by_head = q.transpose(0, 1).contiguous().transpose(0, 1)         # heads before tokens
        got, _ = iseg.kv4_attention(by_head, cache.gpu(), table, *args)
        assert torch.equal(got, want)


@pytest.mark.parametrize("gone", [-1, 1 << 30])
@pytest.mark.parametrize("n,kv,window,page", [(1, 400, 40, 16), (1, 400, 65, 16), (1, 16, 1, 16), (5, 700, 100, 16), (100, 900, 90, 16), (100, 900, 90, 48), (40, 1500, 200, 32),
                                              (1, 5000, 17, 16)])
def test_pages_behind_the_window(n, kv, window, page, gone):
    """Entries of pages whose tokens no query sees are not used."""
    from paper_2011_14504_amd import iseg
    held = -(-kv // page)
    cache = Cache(3, held + 1, 2, 64, page)
    full = table_of(4, [held], held + 1, held)
    part = full.copy()
    part[0, :max(0, kv - n + 1 - window) // page] = gone
    q = normal(5, n, 8, 64).to(torch.bfloat16).to(DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    a, b = (iseg.kv4_attention(q, cache.gpu(), torch.from_numpy(t).to(DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV),
                               torch.tensor([kv], dtype=torch.int32, device=DEV), window=window, status=st) for t in (full, part))
    assert iseg.iseg_status_read(st) == 0
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("n,kv,Hq,H,D", [(1, 300, 8, 2, 128), (1, 3000, 4, 1, 64), (9, 200, 8, 1, 96), (150, 420, 4, 2, 128), (300, 300, 2, 1, 256), (1, 2, 4, 4, 32)])
@pytest.mark.parametrize("size", [0.3, 3.0])
def test_float16_is_off_by_its_own_rounding(n, kv, Hq, H, D, size):
    """float16 outputs: the weights' part of the bound is 2^-21 (two terms), not 2^-11."""
    from paper_2011_14504_amd import iseg
    held = -(-kv // 32)
    cache = Cache(6, held, H, D, 32)
    table = table_of(7, [held], held, held)
    qg, qd = typed(size * rng(8).standard_normal((n, Hq, D)), "fp16")
    scale = 1 / math.sqrt(D)
    out, _ = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV),
                                torch.tensor([kv], dtype=torch.int32, device=DEV))
    o, _, s, reach, far = attention(qd, cache, table, [0, n], [kv], H, scale, True, 0)
    eps = 2 * (D + 16) * U * reach + 2.0 ** -25 * far + 4 * U
    tol = (2 * eps[..., None] + 2.0 ** -21 + 40 * U) * s + (HALF["fp16"] + 4 * U) * np.abs(o) + kv * 7 * 2.0 ** -31 * float(cache.vs.max()) + 2.0 ** -24
    within(out, torch.from_numpy(o), torch.from_numpy(tol), "out")


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("B,n,kv,Hq,H,D", [(1, 1500, 1500, 64, 8, 64), (8, 24, 3000, 64, 8, 64), (2, 700, 1900, 32, 8, 96), (1, 16, 9000, 64, 8, 32)])
def test_enough_rows_for_the_whole_card(B, n, kv, Hq, H, D, t):
    """Tiles of 256 rows, whole and in splits, and of 128 in splits; the formula by
    matrices."""
    from paper_2011_14504_amd import iseg
    page, G = 64, Hq // H
    held = -(-kv // page)
    cache = Cache(11, B * held, H, D, page)
    table = table_of(12, [held] * B, B * held, held)
    qg, qd = typed(rng(13).standard_normal((B * n, Hq, D)), t)
    start = np.arange(B + 1) * n
    out, lse = iseg.kv4_attention(qg, cache.gpu(), torch.from_numpy(table).to(DEV), torch.from_numpy(start.astype(np.int32)).to(DEV),
                                  torch.full((B,), kv, dtype=torch.int32, device=DEV), max_q=n, max_kv=kv)
    scale, want = 1 / math.sqrt(D), [np.zeros((B * n, Hq, D)), np.zeros((B * n, Hq)), np.zeros((B * n, Hq, D)), np.zeros((B * n, Hq)), np.zeros((B * n, Hq))]
    unseen = torch.arange(kv)[None] > torch.arange(kv - n, kv)[:, None]
    for b in range(B):
        rows = slice(b * n, (b + 1) * n)
        for h in range(Hq):
            K, V = (torch.from_numpy(x) for x in cache.rows(table[b], kv, h // G))
            x = torch.from_numpy(qd[rows, h])
            s = (scale * (x @ K.t())).masked_fill(unseen, -math.inf)
            p = torch.softmax(s, -1)
            of = (p @ V, torch.logsumexp(s, -1), p @ V.abs(), scale * (x.abs() @ K.abs().t()).amax(-1), scale * x.abs().amax(-1) * K.abs().sum(1).max())
            for w, y in zip(want, of):
                w[rows, h] = y.numpy()
    _check(out, lse, want, t, D, kv, float(cache.vs.max()), str((B, n, kv)))
