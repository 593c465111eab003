"""The gradient of log probabilities and entropies of rows far from zero, where
a float32 log-sum has lost more than the gradient may: against the formulas of
the logits themselves in 64 bits."""
import math

import pytest
import torch

from lm_util import DEV, DT, HALF, TINY, U, normal, within

pytestmark = pytest.mark.gpu


def _exact(x, tok, g, h):
    """(gradient, its terms' magnitude, log p, entropy) in 64 bits, from the
    logits: differences to the largest one first, so nothing is lost far out."""
    d = x.double() - x.double().amax(1, keepdim=True)
    lp = d - torch.log(torch.exp(d).sum(1, keepdim=True))
    p = torch.exp(lp)
    lpc = torch.where(p > 0, lp, torch.zeros_like(lp))
    ent = -(p * lpc).sum(1, keepdim=True)
    g = torch.where(tok >= 0, g.double(), torch.zeros_like(g, dtype=torch.float64))[:, None]
    h = h.double()[:, None]
    want = -p * (g + h * (lpc + ent))
    rows = (tok >= 0).nonzero()[:, 0]
    want[rows, tok[rows]] += g[rows, 0]
    return want, p * (g.abs() + h.abs() * (lpc.abs() + ent)), p, lpc, ent, h.abs()


@pytest.mark.parametrize("t", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [7, 3001, 40000])
def test_backward_of_far_rows(V, t):
    """Rows filled with the type's lowest value (a mask that leaves nothing), or
    half filled, all of one huge value, and logits around plus and minus 300 and
    far more."""
    from paper_2011_14504_amd import iseg
    print(f"[logprob far rows] {V} {t}", flush=True)
    low = torch.finfo(DT[t]).min
    far = [300.0, -300.0, 2000.0, -9000.0] + ([] if t == "fp16" else [1e6, -3e37])
    x = normal(V, 4 + len(far), V) * 2
    x[0] = low
    x[1, V // 2:] = low
    x[2] = low
    x[2, ::2] = -math.inf
    x[3] = -low
    x[4:] += torch.tensor(far, dtype=torch.float64)[:, None]
    x = x.to(DT[t])
    M = len(x)
    tok = (normal(5, M).abs() * 1e6).long() % V
    tok[2], tok[5] = 1, -1                               # a banned token, and none
    g, h = normal(8, M).float(), normal(9, M).float()
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    lp, lse, ent, _, _ = iseg.logprob_fwd(x.to(DEV), tok.to(DEV), status=st)
    d = iseg.logprob_bwd(x.to(DEV), tok.to(DEV), lse, ent, g.to(DEV), h.to(DEV), status=st)
    assert iseg.iseg_status_read(st) == 0
    want, size, p, lpc, H, ha = _exact(x, tok, g, h)
    # the sum of a row as in the forward: V / 256 + 300 half-steps; log p takes
    # 2 |log p| more from its difference and its own rounding, its exponential
    # 2 |log p| + 3, the factor and products 5; the given entropy is off by
    # three times the sum's error relative to 1 + H + log V
    n = (V // 256 + 300) * U
    tol = size * (n + U * (4 * lpc.abs() + 8)) + p * ha * (4 * n * (1 + H + math.log(V)) + 2 * U * lpc.abs()) \
        + 2 * U * want.abs() + 2.0 ** -126 * (1 + ha * (200 + H)) * 4
    within(d, want, tol + HALF[t] * (want.abs() + tol) + TINY[t], "dlogits")
    only = iseg.logprob_bwd(x.to(DEV), tok.to(DEV), lse, None, g.to(DEV))
    want, size, p, lpc, H, ha = _exact(x, tok, g, torch.zeros(M))
    tol = size * (n + U * (4 * lpc.abs() + 8)) + 2 * U * want.abs() + 2.0 ** -124
    within(only, want, tol + HALF[t] * (want.abs() + tol) + TINY[t], "dlogits without entropy")


@pytest.mark.parametrize("V", [100, 40000])
def test_backward_of_a_part_of_a_vocabulary(V):
    """An lse that is not the row's own is taken as given, near zero and far
    from it: here the log-sum over two parts of a vocabulary, of which one has
    next to nothing (or nothing) of the probability."""
    from paper_2011_14504_amd import iseg
    x = normal(V, 6, 2 * V).float() + torch.tensor([0., 300., -300., 2000., -9000., 400.])[:, None]
    x[1, V:] -= 3                                        # the other part's share still shows in float32
    x[5, V:] = -math.inf
    tok = torch.full((6,), 3)
    lse = torch.logsumexp(x.double(), 1).float()
    g = normal(8, 6).float()
    for half in (x[:, :V], x[:, V:]):
        d = iseg.logprob_bwd(half.to(DEV), tok.to(DEV), lse.to(DEV), None, g.to(DEV))
        lp = half.double() - lse.double()[:, None]
        p = torch.exp(lp)
        want = -p * g.double()[:, None]
        want[:, 3] += g.double()
        # p within 2 |log p| + 3 half-steps, the products 5 more; an lse within
        # its rounding (and 2^-14 for the sum's) of the part's own may be taken for that
        size = p * g.double().abs()[:, None]
        lpc = torch.where(p > 0, lp.abs(), torch.zeros_like(lp))
        slack = 2 * U * lse.double().abs() + 2.0 ** -14
        own = (torch.logsumexp(half.double(), 1) - lse.double()).abs() <= slack
        e = U * (2 * lpc + 8) + (own * slack)[:, None]
        within(d, want, size * e + 2 * U * want.abs() + 2.0 ** -124, "dlogits")
