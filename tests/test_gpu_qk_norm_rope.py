"""Norms of queries and keys with the rotation of their positions, and the
backward, against the formulas in 64 bits and against differences."""
import math

import numpy as np
import pytest
import torch

from lm_util import DEV, DT, HALF, TINY, U, normal, within

pytestmark = pytest.mark.gpu


def _turn(x, pos, freq, pairs, mscale, back=False):
    """float64 rotation of the first 2 len(freq) columns of x [T, H, D]."""
    R = 2 * len(freq)
    a = pos.double()[:, None, None] * freq.double()
    c, s = a.cos() * mscale, a.sin() * mscale * (-1 if back else 1)
    y = x.clone()
    u, v = (x[..., 0:R:2], x[..., 1:R:2]) if pairs else (x[..., :R // 2], x[..., R // 2:R])
    p, q = u * c - v * s, u * s + v * c
    if pairs:
        y[..., 0:R:2], y[..., 1:R:2] = p, q
    else:
        y[..., :R // 2], y[..., R // 2:R] = p, q
    return y


def _forward(x, gamma, pos, freq, pairs, norm, eps, mscale):
    if norm:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
        x = x * gamma if gamma is not None else x
    return _turn(x, pos, freq, pairs, mscale)


def _backward(dy, x, gamma, pos, freq, pairs, norm, eps, mscale):
    g = _turn(dy, pos, freq, pairs, mscale, True)
    if not norm:
        return g, None
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xh = x * r
    h = g * gamma if gamma is not None else g
    return r * (h - xh * (h * xh).mean(-1, keepdim=True)), (g * xh).sum((0, 1))


def _room(x, freq, pairs, mscale):
    """|x| with each rotated pair's elements replaced by mscale times the sum of both."""
    R = 2 * len(freq)
    y = x.abs().clone()
    if pairs:
        y[..., 0:R:2] = y[..., 1:R:2] = abs(mscale) * (x[..., 0:R:2].abs() + x[..., 1:R:2].abs())
    else:
        y[..., :R // 2] = y[..., R // 2:R] = abs(mscale) * (x[..., :R // 2].abs() + x[..., R // 2:R].abs())
    return y


def _inputs(seed, T, Hq, Hk, D, R, t, far=False):
    r = np.random.default_rng(seed)
    q, k, dq, dk = (normal(seed + i, T, h, D).to(DT[t]) for i, h in enumerate((Hq, Hk, Hq, Hk)))
    pos = torch.from_numpy(r.integers(-2 ** 31 if far else 0, 2 ** 31 if far else 20000, T))
    freq = (10000.0 ** (-2 * torch.arange(R // 2, dtype=torch.float64) / max(R, 1))).float()
    return q, k, dq, dk, pos, freq


# A sine is off by its angle's error, 2^-22 of a turn at most far out (2^31
# radians are 2^28.3 turns, of which 64 bits leave 2^-23.7; rounded to 2^-25 of a
# turn) and 2^-25 of a turn near 0, and a few U: SINE.  A norm's factor: D / 2 + 8
# roundings of a sum of squares at most, halved by the root, and a few more.
SINE = 2 * math.pi * 2.0 ** -25 + 4 * U
FAR = 2 * math.pi * 2.0 ** -22 + 4 * U

CASES = [(1, 1, 1, 64, 64), (7, 4, 2, 128, 128), (3, 3, 0, 96, 64), (130, 2, 1, 80, 40), (33, 5, 2, 80, 80), (5, 0, 3, 256, 128), (9, 2, 2, 6, 4),
         (4, 2, 1, 33, 16), (600, 8, 2, 64, 32), (21, 7, 1, 192, 96), (2, 130, 1, 128, 0), (10, 2, 2, 512, 512), (6, 3, 1, 500, 250), (70, 1, 1, 1, 0),
         (1100, 4, 4, 32, 32), (12, 2, 1, 40, 24), (8, 1, 1, 300, 300)]


@pytest.mark.parametrize("t", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_forward_and_backward(case, pairs, t):
    from paper_2011_14504_amd import iseg
    T, Hq, Hk, D, R = case
    for k, (norm, pt, far) in enumerate(((True, t, False), (True, "fp32", True), (False, None, False), (True, None, False))):
        q, kk, dq, dk, pos, freq = _inputs(T + D, *case, t, far)
        sine = FAR if far else SINE
        mscale, eps = (1.0, 1e-6) if k % 2 == 0 else (1.25, 1e-3)
        gq, gk = ((1 + 0.3 * normal(i, D)).to(DT[pt]) if pt else None for i in (50, 51))
        g = lambda v: None if v is None else v.to(DEV)  # noqa: E731
        some = lambda v, h: g(v) if h else None  # noqa: E731
        args = (g(pos) if far else g(pos).int(), g(freq) if R else None)
        kw = dict(gamma_q=some(gq, Hq), gamma_k=some(gk, Hk), eps=eps, pairs=pairs, norm=norm, mscale=mscale)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        ys = iseg.qk_norm_rope_fwd(some(q, Hq), some(kk, Hk), *args, status=st, **kw)
        assert iseg.iseg_status_read(st) == 0
        ds = iseg.qk_norm_rope_bwd(some(dq, Hq), some(dk, Hk), some(q, Hq), some(kk, Hk), *args, **kw)
        for i, (x, dy, gamma, H) in enumerate(((q, dq, gq, Hq), (kk, dk, gk, Hk))):
            if not H:
                assert ys[i] is None and ds[i] is None and ds[2 + i] is None
                continue
            x, dy = x.double(), dy.double()
            gm = gamma.double() if gamma is not None else torch.ones(D, dtype=torch.float64)
            rel = (D / 2 + 12) * U if norm else 0.0
            want = _forward(x, gm, pos, freq, pairs, norm, eps, mscale)
            n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gm if norm else x
            room = _room(n, freq, pairs, mscale)
            within(ys[i], want, (rel + sine + 4 * U) * room + HALF[t] * want.abs() + TINY[t], ("y", case, k))
            dx, dgamma = _backward(dy, x, gm, pos, freq, pairs, norm, eps, mscale)
            gr = _room(dy, freq, pairs, mscale)
            if norm:
                r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
                xh = (x * r).abs()
                h = gr * gm.abs()
                size = r * (h + xh * (h * xh).mean(-1, keepdim=True))
                tol = ((D / 2 + 12) * U + 4 * rel + sine + 8 * U) * size
            else:
                tol = (sine + 4 * U) * gr
            within(ds[i], dx, tol + HALF[t] * dx.abs() + TINY[t], ("dx", case, k))
            if norm:
                # a block's rows one after another, the blocks in turn: T H roundings at most
                all_ = (gr * xh).sum((0, 1))
                half = HALF[pt or t]
                within(ds[2 + i], dgamma, (T * H * U + rel + sine + 8 * U) * all_ + half * dgamma.abs() + TINY[pt or t], ("dgamma", case, k))
            else:
                assert ds[2 + i] is None


@pytest.mark.parametrize("pairs", [False, True])
def test_gradient_against_differences(pairs):
    """d/dx and d/dgamma of a random projection of y, by central differences of the
    64-bit formula."""
    from paper_2011_14504_amd import iseg
    T, H, D, R = 3, 2, 16, 8
    q, _, dq, _, pos, freq = _inputs(1, T, H, 1, D, R, "fp32")
    gamma = (1 + 0.3 * normal(9, D)).float()
    got = iseg.qk_norm_rope_bwd(dq.to(DEV), None, q.to(DEV), None, pos.to(DEV), freq.to(DEV), gamma_q=gamma.to(DEV), eps=1e-3, pairs=pairs, mscale=0.9)

    def f(x, gm):
        return float((_forward(x, gm, pos, freq, pairs, True, 1e-3, 0.9) * dq.double()).sum())

    x0, g0, h = q.double(), gamma.double(), 1e-5
    for at in ((0, 0, 0), (1, 1, 5), (2, 0, 9), (2, 1, 15), (0, 1, 3)):
        e = torch.zeros_like(x0)
        e[at] = h
        # the differences' own error: h^2 of third derivatives of order 1, and 2^-50 / h
        assert abs((f(x0 + e, g0) - f(x0 - e, g0)) / (2 * h) - float(got[0][at])) < 1e-5
    for d in range(0, D, 3):
        e = torch.zeros_like(g0)
        e[d] = h
        assert abs((f(x0, g0 + e) - f(x0, g0 - e)) / (2 * h) - float(got[2][d])) < 1e-5


def test_strided_in_place_and_broadcast():
    from paper_2011_14504_amd import iseg
    for D, R in ((128, 128), (80, 40)):
        T, Hq, Hk = 37, 4, 2
        qkv = normal(3, T, Hq + 2 * Hk, D).to(torch.bfloat16).to(DEV)
        pos, freq = torch.arange(T, device=DEV), iseg.rope_frequencies(R, device=DEV)
        gamma = torch.ones(D, device=DEV)
        q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
        want = iseg.qk_norm_rope_fwd(q.contiguous(), k.contiguous(), pos, freq, gamma, gamma)
        got = iseg.qk_norm_rope_fwd(q, k, pos, freq, gamma, gamma)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        for a, b in zip(iseg.qk_norm_rope_bwd(q, k, k[:, :1].expand(T, Hq, D), q[:, :Hk], pos, freq, gamma, gamma),
                        iseg.qk_norm_rope_bwd(q.contiguous(), k.contiguous(), k[:, :1].expand(T, Hq, D).contiguous(), q[:, :Hk].contiguous(), pos, freq,
                                              gamma, gamma)):
            assert torch.equal(a, b)
        odd = torch.empty(T * Hq * D + 1, dtype=torch.bfloat16, device=DEV)[1:].view(T, Hq, D).copy_(q)
        assert torch.equal(iseg.qk_norm_rope_fwd(odd, None, pos, freq, gamma)[0], want[0])
        by_head = q.transpose(0, 1).contiguous().transpose(0, 1)
        assert torch.equal(iseg.qk_norm_rope_fwd(by_head, None, pos, freq, gamma)[0], want[0])
        v = qkv[:, Hq + Hk:].clone()
        out = iseg.qk_norm_rope_fwd(q, k, pos, freq, gamma, gamma, in_place=True)
        assert out[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, Hq + Hk:], v)


def test_rotations_compose_and_shift():
    """The product of a query and a key depends on the distance of their positions."""
    from paper_2011_14504_amd import iseg
    D, T = 128, 9
    q, k = (normal(i, 1, 2, D).float().expand(T, 2, D).contiguous().to(DEV) for i in (1, 2))
    freq = iseg.rope_frequencies(D, base=500000.0, device=DEV)
    base = torch.arange(T, device=DEV) * 1234567
    a, _ = iseg.qk_norm_rope_fwd(q, None, base + 77, freq)
    b, _ = iseg.qk_norm_rope_fwd(k, None, base, freq)
    s = (a.double() * b.double()).sum(-1)
    size = a.double().norm(dim=-1) * b.double().norm(dim=-1)
    assert ((s - s[:1]).abs() <= (4 * SINE + 20 * U) * size).all()


def test_frequencies():
    from paper_2011_14504_amd import iseg
    f = iseg.rope_frequencies(8, base=100.0, device="cpu")
    assert torch.equal(f, torch.tensor([1.0, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.float64).float())
    assert torch.equal(iseg.rope_frequencies(8, 100.0, factor=4.0, device="cpu"), (f.double() / 4).float())
    g = iseg.rope_frequencies(64, 10000.0, factor=8.0, stretch=(4096, 1.0, 32.0), device="cpu")
    h = iseg.rope_frequencies(64, 10000.0, device="cpu")
    turns = 4096 * h.double() / (2 * math.pi)
    assert torch.equal(g[turns > 32.01], h[turns > 32.01])
    low = turns < 0.99
    assert torch.equal(g[low], (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64) / 8).float()[low])
    mid = (turns > 1.01) & (turns < 31.99)
    assert (g[mid] < h[mid]).all() and (g[mid] > h[mid] / 8).all()


def test_rows_of_nan_and_of_zeros():
    from paper_2011_14504_amd import iseg
    q = normal(1, 4, 2, 64).float().to(DEV)
    q[1, 0] = 0
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    pos, freq = torch.arange(4, device=DEV), iseg.rope_frequencies(64, device=DEV)
    y, _ = iseg.qk_norm_rope_fwd(q, None, pos, freq, status=st)
    assert iseg.iseg_status_read(st) == 0 and (y[1, 0] == 0).all()
    clean = y.clone()
    q[2, 1, 7] = float("inf")
    y, _ = iseg.qk_norm_rope_fwd(q, None, pos, freq, status=st)
    assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
    keep = torch.ones(4, 2, dtype=torch.bool, device=DEV)
    keep[2, 1] = False
    assert torch.equal(y[keep], clean[keep])


def test_no_tokens():
    from paper_2011_14504_amd import iseg
    q = torch.empty(0, 2, 64, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    freq = iseg.rope_frequencies(64, device=DEV)
    y, _ = iseg.qk_norm_rope_fwd(q, None, none, freq)
    assert y.shape == (0, 2, 64)
    dq, _, dg, _ = iseg.qk_norm_rope_bwd(q, None, q, None, none, freq, gamma_q=torch.ones(64, device=DEV))
    assert dq.shape == (0, 2, 64) and (dg == 0).all()
