"""Drafted tokens against the target's probabilities: every decision against a
loop in 64 bits."""
import numpy as np
import pytest
import torch

from lm_util import DEV, DT
from serve_util import rng

pytestmark = pytest.mark.gpu


def _loop(p, q, tokens, n_draft, u, us):
    """p [B, S + 1, V], q [B, S, V] or None: (tokens out, accepted)."""
    B, S1, V = p.shape
    out, acc = np.full((B, S1), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        i, n = 0, min(max(int(n_draft[b]), 0), S1 - 1)
        while i < n:
            x = int(tokens[b, i])
            ok = 0 <= x < V
            qx = (q[b, i, x] if q is not None else 1.0) if ok else 0.0
            if not (ok and float(u[b, i]) * qx < p[b, i, x]):
                break
            out[b, i] = x
            i += 1
        rest = p[b, i].copy()
        if i < n:
            if q is not None:
                rest = np.maximum(rest - q[b, i], 0)
            elif 0 <= tokens[b, i] < V:
                rest[tokens[b, i]] = max(rest[tokens[b, i]] - 1, 0)
        if not rest.any():
            rest = p[b, i]
        c = np.cumsum(rest)
        if c[-1] > 0:
            out[b, i] = int(np.argmax(c > float(us[b]) * c[-1]))
        acc[b] = i
    return out, acc


def _inputs(seed, B, S, V, t, onehot=False, near=0.7):
    r = rng(seed)
    z = r.standard_normal((B, S + 1, V)) * 2

    def soft(z):
        e = np.exp(z - z.max(-1, keepdims=True))
        return torch.from_numpy(e / e.sum(-1, keepdims=True)).to(DT[t])

    p = soft(z)
    q = soft(z[:, :S] + near * r.standard_normal((B, S, V)))
    tok = np.zeros((B, S), np.int64)
    for b in range(B):
        for i in range(S):
            w = q[b, i].double().numpy()
            tok[b, i] = min(np.searchsorted(np.cumsum(w), r.random() * w.sum(), side="right"), V - 1)
    n = np.where(r.random(B) < 0.6, S, r.integers(0, S + 1, B)).astype(np.int32)
    return p, None if onehot else q, tok, n, r.random((B, S)).astype(np.float32), r.random(B).astype(np.float32)


def _compare(p, q, tok, n, u, us, status=0, dtype=torch.int32):
    from paper_2011_14504_amd import iseg
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    g = lambda v: torch.from_numpy(np.asarray(v)).to(DEV)  # noqa: E731
    out, acc = iseg.verify_drafts(p.to(DEV), None if q is None else q.to(DEV), g(tok).to(dtype), g(n), g(u), g(us), status=st)
    assert iseg.iseg_status_read(st) == status
    wo, wa = _loop(p.double().numpy(), None if q is None else q.double().numpy(), tok, n, u, us)
    assert np.array_equal(acc.cpu().numpy(), wa)
    assert np.array_equal(out.cpu().numpy(), wo), (out.cpu().numpy()[(out.cpu().numpy() != wo).any(1)], wo[(out.cpu().numpy() != wo).any(1)])
    return out, acc


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("onehot", [False, True])
@pytest.mark.parametrize("B,S,V", [(1, 1, 1), (1, 0, 50), (1, 4, 1003), (5, 3, 2), (7, 2, 2048), (3, 8, 2049), (40, 5, 777), (2, 70, 300), (4, 3, 50021),
                                   (300, 2, 5000), (1, 2, 270001)])
def test_against_the_loop(B, S, V, onehot, t):
    near = 0.7 if V > 3 else 2.0
    _compare(*_inputs(B + S + V, B, S, V, t, onehot, near), dtype=torch.int64 if S % 2 else torch.int32)


def test_edges_of_the_random_numbers():
    """u of 0 and just below 1, a token without mass on either side."""
    p, q, tok, n, u, us = _inputs(3, 6, 3, 300, "fp32")
    n[:] = 3
    big = np.float32(1 - 2.0 ** -24)
    for a in (np.float32(0), big):
        for b in (np.float32(0), big):
            _compare(p, q, tok, n, np.full_like(u, a), np.full_like(us, b))
    p2, q2 = p.clone(), q.clone()
    p2[:, :, :7] = 0                      # nothing at the front, nothing at the end
    p2[:, :, -5:] = 0
    q2[torch.arange(6)[:, None], torch.arange(3)[None], torch.from_numpy(tok)] = 0       # drafted against all odds: stands if p > 0
    for b in (np.float32(0), big):
        out, _ = _compare(p2, q2, tok, n, np.zeros_like(u), np.full_like(us, b))
    tok2 = tok.copy()
    tok2[:, 0] = 3                        # p is 0 there: refused whatever u says
    out, acc = _compare(p2, q, tok2, n, np.zeros_like(u), us)
    assert (acc == 0).all()


def test_equal_distributions_leave_no_remainder():
    """p = q: a draft is refused only by u q >= p, never here; with a u outside
    its range the remainder is empty and the target's row is used."""
    p, q, tok, n, u, us = _inputs(4, 5, 2, 400, "fp32")
    n[:] = 2
    q = p[:, :2].clone()
    _, acc = _compare(p, q, tok, n, u, us)
    assert (acc == 2).all()
    _, acc = _compare(p, q, tok, n, np.ones_like(u), us)
    assert (acc == 0).all()


def test_counts_and_tokens_out_of_range():
    from paper_2011_14504_amd import iseg
    for onehot in (False, True):
        p, q, tok, n, u, us = _inputs(5, 4, 3, 200, "fp32", onehot)
        _compare(p, q, tok, np.array([-1, 4, 100, 2], np.int32), u, us, iseg.ISEG_DEV_RANGE)
        t = tok.copy()
        t[:, 0] = [200, -1, 2 ** 31 - 1, -2 ** 31]
        _compare(p, q, t, np.full(4, 3, np.int32), u, us, iseg.ISEG_DEV_RANGE)


def test_rows_without_mass_and_of_nan():
    from paper_2011_14504_amd import iseg
    p, q, tok, n, u, us = _inputs(6, 3, 2, 3000, "fp32")
    n[:] = 0
    p[1, 0] = 0
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    g = lambda v: torch.from_numpy(np.asarray(v)).to(DEV)  # noqa: E731
    run = lambda: iseg.verify_drafts(p.to(DEV), q.to(DEV), g(tok).int(), g(n), g(u), g(us), status=st)  # noqa: E731
    out, _ = run()
    assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_RANGE and int(out[1, 0]) == -1 and (out[[0, 2], 0] >= 0).all()
    for v in (float("nan"), float("inf"), -0.5):
        p[1, 0] = 0.1
        p[1, 0, 2500] = v
        iseg.iseg_status_clear(st)
        out, _ = run()
        assert iseg.iseg_status_read(st) & iseg.ISEG_DEV_NONFINITE and -1 <= int(out[1, 0]) < 3000


def test_strided_rows():
    from paper_2011_14504_amd import iseg
    p, q, tok, n, u, us = _inputs(7, 6, 3, 1001, "bf16")
    want = _compare(p, q, tok, n, u, us)
    buf = torch.full((6, 9, 1013), float("nan"), dtype=torch.bfloat16, device=DEV)
    buf[:, 1:8:2, 5:1006] = p.to(DEV)
    buf[:, 2:8:2, 3:1004] = q.to(DEV)
    g = lambda v: torch.from_numpy(np.asarray(v)).to(DEV)  # noqa: E731
    out, acc = iseg.verify_drafts(buf[:, 1:8:2, 5:1006], buf[:, 2:8:2, 3:1004], g(tok), g(n), g(u), g(us))
    assert torch.equal(out, want[0]) and torch.equal(acc, want[1])


def test_the_tokens_follow_the_target():
    """Over many draws the first token has the target's distribution, whatever the
    drafts came from: its counts within six deviations."""
    from paper_2011_14504_amd import iseg
    B, V = 60000, 8
    r = rng(8)
    p = torch.tensor(r.dirichlet(np.ones(V)), dtype=torch.float32).expand(B, 2, V)
    q = torch.tensor(r.dirichlet(np.ones(V)), dtype=torch.float32).expand(B, 1, V)
    tok = torch.from_numpy(np.minimum(np.searchsorted(np.cumsum(q[0, 0].double().numpy()), r.random((B, 1))), V - 1))
    out, _ = iseg.verify_drafts(p.to(DEV), q.to(DEV), tok.to(DEV), torch.ones(B, dtype=torch.int32, device=DEV),
                                torch.from_numpy(r.random((B, 1)).astype(np.float32)).to(DEV), torch.from_numpy(r.random(B).astype(np.float32)).to(DEV))
    c = torch.bincount(out[:, 0].cpu(), minlength=V).double()
    w = p[0, 0].double() * B
    assert ((c - w).abs() <= 6 * (w * (1 - p[0, 0].double())).sqrt() + 1).all()


def test_no_requests():
    from paper_2011_14504_amd import iseg
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    out, acc = iseg.verify_drafts(torch.empty(0, 3, 10, device=DEV), None, none.view(0, 2), none, torch.empty(0, 2, device=DEV), torch.empty(0, device=DEV))
    assert out.shape == (0, 3) and acc.shape == (0,)
