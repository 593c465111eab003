"""Serving operators at sizes whose blocks take several turns: the backward of norm and
rotation with more groups of tokens than blocks, verification with several pieces of a
row to a wave."""
import pytest
import torch

from lm_util import DEV, DT, HALF, TINY, U, normal, within
from test_gpu_qk_norm_rope import SINE, _backward, _inputs, _room
from test_gpu_verify import _compare
from test_gpu_verify import _inputs as _drafts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,Hq,Hk,D,R,t,pairs", [(4100, 32, 8, 128, 128, "bf16", False), (8195, 24, 3, 96, 96, "fp32", False), (9001, 32, 16, 64, 32, "fp16", True),
                                                 (2500, 130, 1, 40, 24, "bf16", False), (2101, 64, 128, 33, 16, "fp32", True)])
def test_backward_of_more_tokens_than_blocks(T, Hq, Hk, D, R, t, pairs):
    """More than 1024 groups of tokens, the last one partly filled.  gamma's gradient: a
    group of lanes adds up its rows of a turn (130 over four groups at most, by single
    elements; 128 over 16 and more by vectors) over up to three turns, 14 additions join
    lanes, waves and blocks: CHAIN roundings."""
    from paper_2011_14504_amd import iseg
    CHAIN = 3 * 33 + 14 if Hq == 130 or Hk == 128 else 3 * 8 + 14
    q, kk, dq, dk, pos, freq = _inputs(T + D, T, Hq, Hk, D, R, t)
    gq, gk = ((1 + 0.3 * normal(i, D)).to(DT[t]) for i in (50, 51))
    g = lambda v: v.to(DEV)  # noqa: E731
    ds = iseg.qk_norm_rope_bwd(g(dq), g(dk), g(q), g(kk), g(pos), g(freq), gamma_q=g(gq), gamma_k=g(gk), eps=1e-6, pairs=pairs)
    rel = (D / 2 + 12) * U
    for i, (x, dy, gamma) in enumerate(((q, dq, gq), (kk, dk, gk))):
        x, dy, gm = x.double(), dy.double(), gamma.double()
        dx, dgamma = _backward(dy, x, gm, pos, freq, pairs, True, 1e-6, 1.0)
        gr = _room(dy, freq, pairs, 1.0)
        r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        xh = (x * r).abs()
        h = gr * gm.abs()
        size = r * (h + xh * (h * xh).mean(-1, keepdim=True))
        within(ds[i], dx, ((D / 2 + 12) * U + 4 * rel + SINE + 8 * U) * size + HALF[t] * dx.abs() + TINY[t], ("dx", i))
        within(ds[2 + i], dgamma, (CHAIN * U + rel + SINE + 8 * U) * (gr * xh).sum((0, 1)) + HALF[t] * dgamma.abs() + TINY[t], ("dgamma", i))


@pytest.mark.parametrize("B,S,V,t,onehot", [(64, 2, 131072, "fp32", False), (70, 1, 131001, "fp32", True), (64, 1, 130995, "bf16", False), (150, 1, 70003, "fp16", False),
                                            (30, 1, 300001, "fp32", False)])
def test_verification_of_several_pieces_to_a_wave(B, S, V, t, onehot):
    """B times a row's pieces (of 256 float32 or 512 16-bit values, twice that in the
    last case) is 16384 or more."""
    _compare(*_drafts(B + V, B, S, V, t, onehot))
