"""Log probabilities, entropies, alternatives and their gradient against the
formulas in 64 bits: vocabularies on both sides of the vector, block and split
sizes, ties, banned tokens, empty rows, tokens that are not given."""
import math

import pytest
import torch

from lm_util import DEV, DT, HALF, TINY, U, normal, strided, within

pytestmark = pytest.mark.gpu

# (M, V, type, gap, top_k, tokens' type)
CASES = [
    (1, 1, "fp32", 0, 1, torch.int64), (2, 2, "bf16", 0, 2, torch.int32), (3, 7, "fp16", 1, 7, torch.int64), (5, 64, "fp32", 0, 64, torch.int64),
    (4, 100, "bf16", 0, 20, torch.int64), (3, 1000, "fp32", 5, 5, torch.int32), (2, 2047, "bf16", 0, 64, torch.int64), (2, 2049, "bf16", 1, 3, torch.int64),
    (1, 8192, "fp32", 0, 20, torch.int64), (3, 8193, "fp16", 3, 20, torch.int64), (1, 50021, "bf16", 0, 20, torch.int64),
    (2, 65536, "fp32", 0, 64, torch.int32), (1, 131072, "bf16", 0, 20, torch.int64), (40, 20000, "bf16", 0, 5, torch.int64), (1, 262147, "fp32", 0, 1, torch.int64),
    (1, 600007, "bf16", 0, 1, torch.int64), (1, 300000, "fp32", 0, 64, torch.int64), (20, 50000, "fp32", 1, 64, torch.int64), (600, 1003, "fp16", 0, 64, torch.int32),
    (1100, 300, "bf16", 4, 4, torch.int64), (1030, 5000, "fp32", 0, 0, torch.int64), (2, 100003, "fp16", 0, 0, torch.int64),
]


def _reference(x, tok, k):
    """x float64, the definition with its special rows."""
    lse = torch.logsumexp(x, 1)
    empty = torch.isinf(x).all(1) & (x < 0).all(1)
    p = torch.exp(x - lse[:, None])
    p[empty] = 0
    ent = -torch.xlogy(p, p).sum(1)
    given = tok >= 0
    lp = x.gather(1, tok.long().clamp_min(0)[:, None])[:, 0] - lse
    lp = torch.where(empty, torch.full_like(lp, -math.inf), lp)
    lp = torch.where(given, lp, torch.zeros_like(lp))
    val, ids = torch.sort(x, dim=1, descending=True, stable=True)
    tlp = val[:, :k] - lse[:, None]
    tlp[empty] = -math.inf
    return lp, lse, ent, ids[:, :k].int(), tlp


def _check_fwd(iseg, x, xg, tok, k, t, status=0):
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = iseg.logprob_fwd(xg, tok.to(DEV), top_k=k, status=st)
    assert iseg.iseg_status_read(st) == status
    lp, lse, ent, ids, tlp = _reference(x.double(), tok, k)
    V = x.shape[1]
    # a thread adds at most V / 256 exponentials (more when a row is cut), 8 +
    # 256 joins follow; each exponential is off by 2 (|d| + 1) half-steps, and
    # e^d |d| stays below 0.37
    n = (V // 256 + 300) * U
    m = x.double().amax(1).clamp(min=-1e30, max=1e30)
    logs = torch.where(torch.isfinite(lse), lse - m, torch.zeros_like(lse))
    fin = lambda v: torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v))
    within(got[0], lp, n + 3 * U * (fin(lp) + logs.abs() + 1), "logprob")
    within(got[1], lse, n + 2 * U * (m.abs() + logs.abs()), "lse")
    within(got[2], ent, 3 * n * (1 + ent + logs.abs()), "entropy")
    if k:
        assert torch.equal(got[3].cpu(), ids)
        within(got[4], tlp, n + 3 * U * (fin(tlp) + logs[:, None].abs() + 1), "top_logprob")
    else:
        assert got[3] is None and got[4] is None
    no = iseg.logprob_fwd(xg, tok.to(DEV), top_k=k, want_entropy=False)
    assert no[2] is None and torch.equal(no[0], got[0]) and torch.equal(no[1], got[1])
    return got


def _inputs(case):
    M, V, t, gap, k, tt = case
    x = (normal(M + V, M, V) * 3 + normal(V, M, 1)).to(DT[t])
    tok = (normal(5, M).abs() * 1e9).long() % V
    if M > 2:
        tok[1] = -100
    return x, tok.to(tt)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case):
    from paper_2011_14504_amd import iseg
    M, V, t, gap, k, tt = case
    print(f"[logprob fwd] {case}", flush=True)
    x, tok = _inputs(case)
    _check_fwd(iseg, x, strided(x, V + gap, float("nan")), tok, k, t)


@pytest.mark.parametrize("t", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [9, 3001, 40000])
def test_ties_masks_and_empty_rows(V, t):
    from paper_2011_14504_amd import iseg
    print(f"[logprob masks] {V} {t}", flush=True)
    low = torch.finfo(DT[t]).min
    x = (normal(V, 12, V) * 2).to(DT[t])
    x[0] = 0                                             # every logit equal
    x[1] = -math.inf                                     # nothing left
    x[2] = low                                           # the type's lowest value everywhere
    x[3, 1:] = -math.inf                                 # one left
    x[4, : V // 2] = low                                 # half masked by it
    x[5, ::2] = -math.inf
    x[6] = (torch.arange(V) % 3).to(DT[t])               # many ties
    x[7] = torch.arange(V).to(DT[t]) / V                 # rising
    x[8] = -torch.arange(V).to(DT[t]) / V                # falling
    x[9] = torch.tensor(-0.0)
    x[9, ::3] = 0.0                                      # the two zeros are equal
    x[10, V // 2] = 300.0 if t != "fp16" else 200.0      # one token takes everything
    x[11, V - 1] = -math.inf
    tok = torch.tensor([V - 1, 0, V // 2, 0, 0, 1, 2, V - 1, 0, 1, V // 2, V - 1])
    _check_fwd(iseg, x, x.to(DEV), tok, min(V, 20), t)
    one = _check_fwd(iseg, x[1:2], x[1:2].to(DEV), tok[1:2], min(V, 64), t)       # cut over several blocks
    assert torch.equal(one[3].cpu()[0], torch.arange(min(V, 64), dtype=torch.int32))
    _check_fwd(iseg, x[6:8], x[6:8].to(DEV), tok[6:8], min(V, 64), t)
    _check_fwd(iseg, x[0:1], x[0:1].to(DEV), tok[0:1], min(V, 64), t)


def test_large_offsets():
    from paper_2011_14504_amd import iseg
    x = normal(3, 4, 5000).float() + torch.tensor([1e4, -1e4, 3e37, -3e37])[:, None]
    x[2, 5] = -3e38
    _check_fwd(iseg, x, x.to(DEV), torch.tensor([1, 2, 3, 4]), 10, "fp32")


def test_bad_tokens_and_values():
    from paper_2011_14504_amd import iseg
    for V in (100, 30000):
        x = normal(1, 5, V).float()
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        tok = torch.tensor([0, V, 2, V - 1, 1 << 40])
        lp, lse, ent, ids, tlp = iseg.logprob_fwd(x.to(DEV), tok.to(DEV), top_k=3, status=st)
        assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_RANGE
        assert torch.isnan(lp.cpu()).tolist() == [False, True, False, False, True]
        ref = _reference(x.double(), tok.clamp_max(V - 1), 3)
        assert torch.equal(ids.cpu(), ref[3])
        iseg.iseg_status_clear(st)
        d = iseg.logprob_bwd(x.to(DEV), tok.to(DEV), lse, ent, torch.ones(5, device=DEV), status=st)
        assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_RANGE
        assert not bool(d[1].any()) and not bool(d[4].any())
        iseg.iseg_status_clear(st)
        for bad in (math.nan, math.inf):
            y = x.clone()
            y[2, V // 3] = bad
            y[3] = bad
            lp, lse, ent, ids, tlp = iseg.logprob_fwd(y.to(DEV), torch.zeros(5, dtype=torch.int64, device=DEV), top_k=64, status=st)
            assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
            iseg.iseg_status_clear(st)
            for v in (lp, lse, ent, tlp[:, 0]):
                assert torch.isnan(v.cpu()).tolist() == [False, False, True, True, False]
            assert bool(((ids >= 0) & (ids < V)).all())


def _check_bwd(iseg, x, xg, tok, lse, ent, glp, gh, t):
    d = iseg.logprob_bwd(xg, tok.to(DEV), lse.to(DEV), None if ent is None else ent.to(DEV),
                         None if glp is None else glp.to(DEV), None if gh is None else gh.to(DEV))
    M, V = x.shape
    l64 = lse.double()[:, None]
    lpv = x.double() - l64
    p = torch.exp(lpv)
    p[torch.isinf(lse) & (lse < 0)] = 0
    lpc = lpv.clamp_min(-1e6)
    lpc[torch.isnan(lpc)] = 0
    g = glp.double() if glp is not None else torch.zeros(M, dtype=torch.float64)
    g = torch.where(tok >= 0, g, torch.zeros_like(g))
    h = gh.double() if gh is not None else torch.zeros(M, dtype=torch.float64)
    e = ent.double() if ent is not None else torch.zeros(M, dtype=torch.float64)
    want = -p * (g[:, None] + h[:, None] * (lpc + e[:, None]))
    size = p * (g.abs()[:, None] + h.abs()[:, None] * (lpc.abs() + e.abs()[:, None]))
    rows = (tok >= 0) & ~(torch.isinf(lse) & (lse < 0))
    want[rows.nonzero()[:, 0], tok[rows].long()] += g[rows]
    # p within 2 |log p| + 3 half-steps, the factor and products 5 more; a p
    # below 2^-126 may count as 0; the token's own addition one more
    tol = U * size * (2 * lpc.abs() + 8) + U * want.abs() \
        + 2.0 ** -126 * (g.abs()[:, None] + h.abs()[:, None] * (200 + e.abs()[:, None]))
    within(d, want, tol + HALF[t] * (want.abs() + tol) + TINY[t], "dlogits")
    assert d.dtype == x.dtype and d.shape == x.shape


@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(case):
    from paper_2011_14504_amd import iseg
    M, V, t, gap, k, tt = case
    print(f"[logprob bwd] {case}", flush=True)
    x, tok = _inputs(case)
    xg = strided(x, V + gap, float("nan"))
    _, lse, ent, _, _ = (v if v is None else v.float() for v in _reference(x.double(), tok, 1))
    glp, gh = normal(8, M).float(), normal(9, M).float() * 0.1
    _check_bwd(iseg, x, xg, tok, lse, ent, glp, gh, t)
    _check_bwd(iseg, x, xg, tok, lse, None, glp, None, t)
    _check_bwd(iseg, x, xg, tok, lse, ent, None, gh, t)


def test_backward_masks():
    from paper_2011_14504_amd import iseg
    for t in ("fp32", "bf16"):
        x = normal(1, 5, 3001).to(DT[t])
        x[0] = -math.inf
        x[1, ::2] = -math.inf
        x[2, 7:] = torch.finfo(DT[t]).min
        x[3, 1:] = -math.inf
        tok = torch.tensor([4, 0, 3000, 0, -1])              # a banned token among them
        _, lse, ent, _, _ = (v.float() for v in _reference(x.double(), tok, 1))
        _check_bwd(iseg, x, x.to(DEV), tok, lse, ent, normal(8, 5).float(), normal(9, 5).float(), t)


def test_backward_against_differences():
    from paper_2011_14504_amd import iseg
    x, tok = normal(1, 3, 40).float(), torch.tensor([3, -1, 39])
    glp, gh = normal(2, 3).float(), normal(3, 3).float()
    lp, lse, ent, _, _ = iseg.logprob_fwd(x.to(DEV), tok.to(DEV))
    d = iseg.logprob_bwd(x.to(DEV), tok.to(DEV), lse, ent, glp.to(DEV), gh.to(DEV)).cpu()

    def loss(x):
        r = _reference(x, tok, 1)
        return float((r[0] * glp.double() + r[2] * gh.double()).sum())

    h = 1e-5
    x8 = x.double()
    for m in range(3):
        for v in range(0, 40, 3):
            keep = float(x8[m, v])
            x8[m, v] = keep + h
            up = loss(x8)
            x8[m, v] = keep - h
            dn = loss(x8)
            x8[m, v] = keep
            # rounding of the losses over 2 h and h^2 times a third derivative
            assert abs((up - dn) / (2 * h) - float(d[m, v])) < 1e-6, (m, v)


def test_backward_leaves_what_lies_between_rows():
    from paper_2011_14504_amd import iseg
    x = normal(1, 4, 77).to(torch.bfloat16)
    tok = torch.tensor([1, 2, 3, 4])
    lp, lse, ent, _, _ = iseg.logprob_fwd(x.to(DEV), tok.to(DEV))
    out = torch.full((6, 90), 3.0, dtype=torch.bfloat16, device=DEV)
    g = iseg.LogprobGeom(4, 77, 77, 90, iseg.ISEG_BF16, iseg.ISEG_I64, 0, 0)
    one = torch.ones(4, device=DEV)
    iseg.iseg_logprob_bwd(x.to(DEV), tok.to(DEV), lse, ent, one, None, g, out)
    assert torch.equal(out[:4, :77], iseg.logprob_bwd(x.to(DEV), tok.to(DEV), lse, ent, one))
    assert bool((out[4:] == 3).all()) and bool((out[:, 77:] == 3).all())


def test_shapes_and_empty():
    from paper_2011_14504_amd import iseg
    x = normal(1, 2, 3, 50).float().to(DEV)
    tok = torch.tensor([[1, 2, 3], [4, 5, -1]], device=DEV)
    got = iseg.logprob_fwd(x, tok, top_k=4)
    assert got[0].shape == (2, 3) and got[3].shape == (2, 3, 4)
    flat = iseg.logprob_fwd(x.reshape(6, 50), tok.reshape(6), top_k=4)
    assert torch.equal(got[4].reshape(6, 4), flat[4]) and torch.equal(got[2].reshape(6), flat[2])
    d = iseg.logprob_bwd(x, tok, got[1], got[2], torch.ones(2, 3, device=DEV))
    assert d.shape == x.shape
    e = iseg.logprob_fwd(torch.empty(0, 9, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), top_k=2)
    assert e[0].shape == (0,) and e[3].shape == (0, 2)
    z = torch.empty(0, device=DEV)
    assert iseg.logprob_bwd(torch.empty(0, 9, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), z, z, z).shape == (0, 9)
