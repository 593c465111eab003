"""Probabilities that are none among the drafts that were accepted."""
import numpy as np
import pytest
import torch

from lm_util import DEV, DT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("S", [3, 130])
def test_accepted_drafts_of_no_probability(S, t):
    """An accepted draft's probabilities of infinity or below zero set the status; those
    of drafts after the first refused one, and of tokens that were not drafted, do not."""
    from paper_2011_14504_amd import iseg
    B, V = 4, 600
    g = lambda v, d=torch.int32: torch.as_tensor(v, dtype=d, device=DEV)  # noqa: E731
    tok = torch.arange(S)[None].expand(B, S) % V
    at = S - 2
    for p_bad, q_bad, said in ((float("inf"), 0.001, True), (0.001, -0.5, True), (0.001, -float("inf"), True), (0.001, 0.001, False)):
        p, q = torch.full((B, S + 1, V), 1 / V), torch.full((B, S, V), 1 / V)
        p[2, at, at % V], q[2, at, at % V] = p_bad, q_bad
        run = lambda n, u, st: iseg.verify_drafts(p.to(DT[t]).to(DEV), q.to(DT[t]).to(DEV), g(tok), g([n] * B), g(u, torch.float32),  # noqa: E731
                                                  g([0.5] * B, torch.float32), status=st)
        u = np.full((B, S), 0.25)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        _, acc = run(S, u, st)
        assert acc.tolist() == [S] * B and iseg.iseg_status_read(st) == (iseg.ISEG_DEV_NONFINITE if said else 0), (p_bad, q_bad)
        # the draft before it refused: 1 / V is not above 1 times 1 / V, nor what follows it
        # a row that is used
        u[:, at - 1] = 1.0
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        _, acc = run(S, u, st)
        assert acc.tolist() == [at - 1] * B and iseg.iseg_status_read(st) == 0, (p_bad, q_bad)
        # not drafted
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        _, acc = run(at - 1, np.full((B, S), 0.25), st)
        assert acc.tolist() == [at - 1] * B and iseg.iseg_status_read(st) == 0, (p_bad, q_bad)
