"""Shared parts of the tests of the language-model operators: types, their
rounding units, inputs from numpy seeds and the formulas in 64 bits."""
import numpy as np
import torch

U = 2.0 ** -24                                   # half a step of float32, relative
DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
HALF = {k: torch.finfo(t).eps / 2 for k, t in DT.items()}
TINY = {"fp32": 2.0 ** -149, "fp16": 2.0 ** -24, "bf16": 2.0 ** -133}   # smallest subnormal

DEV = "cuda:0"


def normal(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape))


def codes(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).integers(-128, 128, shape, dtype=np.int8))


def strided(x, ld, fill):
    """x on the GPU in rows ld apart; the gaps hold `fill`."""
    buf = torch.full((x.shape[0], ld), fill, dtype=x.dtype)
    buf[:, :x.shape[1]] = x
    return buf.to(DEV)[:, :x.shape[1]]


def within(got, want, tol, what):
    """|got - want| <= tol everywhere, NaN and infinities in the same places."""
    got, want = got.double().cpu(), want.double()
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fin & ~torch.isnan(want)], want[~fin & ~torch.isnan(want)]), what
    tol = torch.as_tensor(tol, dtype=torch.float64).expand(want.shape)
    bad = (got - want).abs()[fin] - tol[fin]
    if bad.numel():
        i = int(bad.argmax())
        assert bad[i] <= 0, (what, "off by", float((got - want).abs()[fin][i]), "allowed", float(tol[fin][i]),
                             "value", float(want[fin][i]))


def quantized(v, bits, pow2):
    """(codes, float32 scales) of the rows of v (float64)."""
    lim = 2 ** (bits - 1) - 1
    big = v.abs().amax(1) if v.shape[1] else torch.zeros(v.shape[0], dtype=torch.float64)
    if pow2:
        _, e = torch.frexp(big)
        s = torch.ldexp(torch.ones_like(big), e + 1 - bits)
    else:
        s = big / lim
    s = s.float().clamp_min(2.0 ** -126)
    s = torch.where(big > 0, s, torch.ones_like(s))
    q = torch.floor(v / s.double()[:, None] + 0.5).clamp(-lim, lim)
    return q.to(torch.int8), s
