"""How the helpers of the language-model operators take their arguments."""
import pytest
import torch

from lm_util import DEV, codes, normal


def _calls(iseg, dev):
    """Every helper with a valid call's arguments by name."""
    x, q = normal(1, 6, 48).float().to(dev), codes(2, 6, 48).to(dev)
    w, v, tok = codes(3, 20, 48).to(dev), (normal(4, 6).abs() + 0.1).float().to(dev), torch.arange(6).to(dev)
    dy = normal(5, 6, 20).float().to(dev)
    return [
        (iseg.layernorm_fwd, dict(x=x, gamma=None, beta=None, eps=1e-5, status=None)),
        (iseg.layernorm_bwd, dict(dy=x, x=x, gamma=None, mean=v, rstd=v, want_params=True)),
        (iseg.quantize_rows, dict(x=x, bits=8, scale_mode=iseg.ISEG_SCALE_MAX, mul=None, status=None)),
        (iseg.quantize_cols, dict(x=x, bits=8, scale_mode=iseg.ISEG_SCALE_MAX, mul=None, want_sums=True, status=None)),
        (iseg.transpose_i8, dict(codes=q)),
        (iseg.matmul_i8, dict(a=q, b=w, a_scale=v, b_scale=None, bias=None, out_dtype=torch.float32)),
        (iseg.linear_i8_fwd, dict(x=x, w=w, w_scale=None, bias=None, bits=8, scale_mode=iseg.ISEG_SCALE_MAX, out_dtype=None, status=None)),
        (iseg.linear_i8_bwd, dict(dy=dy, a=q, a_scale=v, w=w, w_scale=None, w_t=None, bits=8, scale_mode=iseg.ISEG_SCALE_MAX, out_dtype=None,
                                  want_input=True, want_weight=True, want_bias=True, status=None)),
        (iseg.logprob_fwd, dict(logits=x, tokens=tok, top_k=3, want_entropy=True, status=None)),
        (iseg.logprob_bwd, dict(logits=x, tokens=tok, lse=v, entropy=v, g_logprob=v, g_entropy=v, status=None)),
    ]


@pytest.mark.parametrize("n", range(10))
def test_arguments_by_name(n):
    """The first argument may be named too: the call gets as far as its refusal
    of CPU tensors, the last of its checks."""
    from paper_2011_14504_amd import iseg
    f, kw = _calls(iseg, "cpu")[n]
    with pytest.raises(ValueError, match="GPU tensors expected"):
        f(**kw)
    with pytest.raises(TypeError, match=next(iter(kw))):
        f(**{k: v for k, v in list(kw.items())[1:]})


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16, torch.float32])
def test_layernorm_parameter_type(monkeypatch, t):
    """The type that the kernels are chosen by: the parameters', and x's own
    without any (float32 parameters beside 16-bit rows of more than 16384
    columns take more passes over the row)."""
    from paper_2011_14504_amd import iseg
    seen = []
    monkeypatch.setattr(iseg, "_gpu", lambda x, *ts: None)
    monkeypatch.setattr(iseg, "iseg_layernorm_fwd", lambda x, g, b, geom, *rest: seen.append(geom.p_dtype))
    x, one = torch.zeros(2, 20000, dtype=t), torch.ones(20000)
    iseg.layernorm_fwd(x)
    iseg.layernorm_fwd(x, one)
    iseg.layernorm_fwd(x, None, one.half())
    assert seen == [iseg._FLOATS[t], iseg.ISEG_F32, iseg.ISEG_F16]


@pytest.mark.gpu
@pytest.mark.parametrize("C", [100, 9000, 20000, 40000])
def test_layernorm_without_parameters_is_that_of_ones_and_zeros(C):
    from paper_2011_14504_amd import iseg
    x = (normal(C, 5, C) + 0.5).to(torch.bfloat16).to(DEV)
    one = torch.ones(C, dtype=torch.bfloat16, device=DEV)
    for a, b in zip(iseg.layernorm_fwd(x), iseg.layernorm_fwd(x, one, 0 * one)):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(10))
def test_arguments_by_name_give_the_same(n):
    from paper_2011_14504_amd import iseg
    f, kw = _calls(iseg, DEV)[n]
    for a, b in zip(f(**kw), f(*kw.values())):
        assert (a is None and b is None) or torch.equal(a, b)
