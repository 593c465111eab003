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
    monkeypatch.setattr(iseg, "_gpu", lambda x, *ts, **kw: None)
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


# (helper, arguments that replace a valid call's, the refusal's words): every
# check is told apart by its own message, so that no later one can stand in
REFUSALS = [
    ("layernorm_fwd", dict(x=torch.zeros(4, 32).double()), "x: float32, float16 or bfloat16"),
    ("layernorm_fwd", dict(x=torch.zeros(())), "x: at least one dimension"),
    ("layernorm_fwd", dict(x=torch.zeros(4, 0)), "x: empty rows"),
    ("layernorm_fwd", dict(gamma=torch.zeros(31)), "gamma: 48 elements of torch.float32"),
    ("layernorm_fwd", dict(beta=torch.zeros(49)), "beta: 48 elements"),
    ("layernorm_fwd", dict(gamma=torch.zeros(48).double()), "gamma, beta: float32, float16 or bfloat16"),
    ("layernorm_fwd", dict(gamma=torch.zeros(48).half(), beta=torch.zeros(48)), "beta: 48 elements of torch.float16"),
    ("layernorm_fwd", dict(eps=0.0), "eps: positive and finite"),
    ("layernorm_fwd", dict(eps=-1.0), "eps: positive and finite"),
    ("layernorm_fwd", dict(eps=float("nan")), "eps: positive and finite"),
    ("layernorm_fwd", dict(eps=float("inf")), "eps: positive and finite"),
    ("layernorm_bwd", dict(x=torch.zeros(6, 48).double()), "x: float32, float16 or bfloat16"),
    ("layernorm_bwd", dict(dy=torch.zeros(6, 48).half()), "dy: x's shape and type"),
    ("layernorm_bwd", dict(dy=torch.zeros(5, 48)), "dy: x's shape and type"),
    ("layernorm_bwd", dict(dy=torch.zeros(6, 0), x=torch.zeros(6, 0)), "x: empty rows"),
    ("layernorm_bwd", dict(gamma=torch.zeros(47)), "gamma: 48 elements"),
    ("layernorm_bwd", dict(gamma=torch.zeros(48).double()), "gamma: float32, float16 or bfloat16"),
    ("layernorm_bwd", dict(mean=torch.zeros(6).double()), "mean: 6 elements of torch.float32"),
    ("layernorm_bwd", dict(mean=torch.zeros(5)), "mean: 6 elements"),
    ("layernorm_bwd", dict(rstd=torch.zeros(7)), "rstd: 6 elements"),
    ("quantize_rows", dict(x=torch.zeros(6, 48, dtype=torch.int8)), "x: float32, float16 or bfloat16"),
    ("quantize_rows", dict(bits=9), "bits: 2 to 8"), ("quantize_rows", dict(bits=1), "bits: 2 to 8"),
    ("quantize_rows", dict(scale_mode=2), "scale_mode: ISEG_SCALE_MAX or"),
    ("quantize_rows", dict(mul=torch.ones(6)), "mul: 48 elements"),
    ("quantize_rows", dict(mul=torch.ones(48).half()), "mul: 48 elements of torch.float32"),
    ("quantize_cols", dict(x=torch.zeros(6, 48).double()), "x: float32, float16 or bfloat16"),
    ("quantize_cols", dict(bits=9), "bits: 2 to 8"), ("quantize_cols", dict(bits=1), "bits: 2 to 8"),
    ("quantize_cols", dict(scale_mode=-1), "scale_mode: ISEG_SCALE_MAX or"),
    ("quantize_cols", dict(mul=torch.ones(48)), "mul: 6 elements"),
    ("transpose_i8", dict(codes=torch.zeros(6, 48)), "codes: an int8 matrix"),
    ("transpose_i8", dict(codes=torch.zeros(48, dtype=torch.int8)), "codes: an int8 matrix"),
    ("matmul_i8", dict(a=torch.zeros(6, 48)), "a: an int8 matrix"),
    ("matmul_i8", dict(b=torch.zeros(20, 48)), "b: an int8 matrix"),
    ("matmul_i8", dict(b=torch.zeros(20, 47, dtype=torch.int8)), "a and b: rows of one length"),
    ("matmul_i8", dict(a=torch.zeros(1, 131072, dtype=torch.int8), b=torch.zeros(1, 131072, dtype=torch.int8)), "a and b: rows of at most 131071"),
    ("matmul_i8", dict(a_scale=torch.zeros(20)), "a_scale: 6 elements"),
    ("matmul_i8", dict(b_scale=torch.zeros(6)), "b_scale: 20 elements"),
    ("matmul_i8", dict(b_scale=torch.zeros(20).double()), "b_scale: 20 elements of torch.float32"),
    ("matmul_i8", dict(bias=torch.zeros(19)), "bias: 20 elements"),
    ("matmul_i8", dict(out_dtype=torch.int32), "out_dtype: float32, float16 or bfloat16"),
    ("linear_i8_fwd", dict(x=torch.zeros(6, 48, dtype=torch.int8)), "(x|out_dtype): float32, float16 or bfloat16"),
    ("linear_i8_fwd", dict(x=torch.zeros(())), "x and w: rows of one length"),
    ("linear_i8_fwd", dict(w=torch.zeros(20, 47, dtype=torch.int8)), "x and w: rows of one length"),
    ("linear_i8_fwd", dict(w=torch.zeros(20, 48)), "w: an int8 matrix"),
    ("linear_i8_fwd", dict(x=torch.zeros(1, 131072), w=torch.zeros(1, 131072, dtype=torch.int8)), "x and w: rows of at most 131071"),
    ("linear_i8_fwd", dict(w_scale=torch.zeros(6)), "w_scale: 20 elements"),
    ("linear_i8_fwd", dict(bias=torch.zeros(20).half()), "bias: 20 elements of torch.float32"),
    ("linear_i8_fwd", dict(bits=1), "bits: 2 to 8"), ("linear_i8_fwd", dict(scale_mode=2), "scale_mode: ISEG_SCALE_MAX or"),
    ("linear_i8_fwd", dict(out_dtype=torch.int8), "out_dtype: float32, float16 or bfloat16"),
    ("linear_i8_bwd", dict(dy=torch.zeros(6, 20).double()), "dy: float32, float16 or bfloat16"),
    ("linear_i8_bwd", dict(dy=torch.zeros(5, 20)), "expected"),
    ("linear_i8_bwd", dict(a=torch.zeros(6, 48)), "a: an int8 matrix"),
    ("linear_i8_bwd", dict(a=torch.zeros(6, 47, dtype=torch.int8)), r"dy \[..., N\], a \[M, K\] and w \[N, K\] expected"),
    ("linear_i8_bwd", dict(w=torch.zeros(21, 48, dtype=torch.int8)), r"dy \[..., N\], a \[M, K\] and w \[N, K\] expected"),
    ("linear_i8_bwd", dict(w=torch.zeros(20, 48)), "w: an int8 matrix"),
    ("linear_i8_bwd", dict(w_t=torch.zeros(20, 48, dtype=torch.int8)), "w_t: the transposed w"),
    ("linear_i8_bwd", dict(w_t=torch.zeros(48, 20)), "w_t: an int8 matrix"),
    ("linear_i8_bwd", dict(a_scale=torch.zeros(20)), "a_scale: 6 elements"),
    ("linear_i8_bwd", dict(w_scale=torch.zeros(6)), "w_scale: 20 elements"),
    ("linear_i8_bwd", dict(bits=9), "bits: 2 to 8"), ("linear_i8_bwd", dict(scale_mode=3), "scale_mode: ISEG_SCALE_MAX or"),
    ("linear_i8_bwd", dict(out_dtype=torch.int32), "out_dtype: float32, float16 or bfloat16"),
    ("linear_i8_bwd", dict(dy=torch.zeros(1, 131072), a=torch.zeros(1, 1, dtype=torch.int8), a_scale=None, w=torch.zeros(131072, 1, dtype=torch.int8)),
     "dy: reductions of at most 131071"),
    ("linear_i8_bwd", dict(dy=torch.zeros(131072, 1), a=torch.zeros(131072, 1, dtype=torch.int8), a_scale=None, w=torch.zeros(1, 1, dtype=torch.int8)),
     "dy: reductions of at most 131071"),
    ("logprob_fwd", dict(logits=torch.zeros(6, 48).double()), "logits: float32, float16 or bfloat16"),
    ("logprob_fwd", dict(logits=torch.zeros(6, 0), top_k=0), "logits: empty rows"),
    ("logprob_fwd", dict(tokens=torch.zeros(5, dtype=torch.int64)), "tokens: int32 or int64 of the logits' leading shape"),
    ("logprob_fwd", dict(tokens=torch.zeros(6)), "tokens: int32 or int64"),
    ("logprob_fwd", dict(top_k=49), "top_k: 0 to 64"), ("logprob_fwd", dict(top_k=-1), "top_k: 0 to 64"),
    ("logprob_fwd", dict(logits=torch.zeros(6, 100), top_k=65), "top_k: 0 to 64"),
    ("logprob_bwd", dict(logits=torch.zeros(6, 48, dtype=torch.int32)), "logits: float32, float16 or bfloat16"),
    ("logprob_bwd", dict(logits=torch.zeros(6, 0)), "logits: empty rows"),
    ("logprob_bwd", dict(tokens=torch.zeros(2, 3, dtype=torch.int64)), "tokens: int32 or int64"),
    ("logprob_bwd", dict(g_logprob=None, g_entropy=None), "g_logprob or g_entropy expected"),
    ("logprob_bwd", dict(lse=None), "the forward's lse and"),
    ("logprob_bwd", dict(entropy=None), "with g_entropy, its entropy expected"),
    ("logprob_bwd", dict(lse=torch.zeros(5)), "lse: 6 elements"),
    ("logprob_bwd", dict(entropy=torch.zeros(6).double()), "entropy: 6 elements of torch.float32"),
    ("logprob_bwd", dict(g_logprob=torch.zeros(7)), "g_logprob: 6 elements"),
    ("logprob_bwd", dict(g_entropy=torch.zeros(6).half()), "g_entropy: 6 elements of torch.float32"),
] + [(name, dict(status=st), "status: an int32 word") for st in (torch.zeros(1), torch.zeros(4, dtype=torch.uint8), torch.zeros(0, dtype=torch.int32))
     for name in ("layernorm_fwd", "quantize_rows", "quantize_cols", "linear_i8_fwd", "linear_i8_bwd", "logprob_fwd", "logprob_bwd")]


@pytest.mark.parametrize("i", range(len(REFUSALS)), ids=lambda i: f"{REFUSALS[i][0]}-{i}")
def test_refusals_by_their_message(i):
    from paper_2011_14504_amd import iseg
    name, bad, words = REFUSALS[i]
    f, kw = next((f, kw) for f, kw in _calls(iseg, "cpu") if f.__name__ == name)
    with pytest.raises(ValueError, match=words):
        f(**{**kw, **bad})


@pytest.mark.gpu
@pytest.mark.parametrize("n", range(10))
def test_tensors_elsewhere(n):
    """Every tensor of a call has to be on the first one's device."""
    from paper_2011_14504_amd import iseg
    f, kw = _calls(iseg, DEV)[n]
    f(**kw)
    first = next(iter(kw))
    for k in [k for k, v in kw.items() if isinstance(v, torch.Tensor)]:
        if k in ("mean", "rstd", "a_scale", "lse", "entropy", "g_logprob", "g_entropy"):
            words = f"{k}: 6 elements of torch.float32 on cuda:0"
        elif k == "tokens":
            words = "tokens: on the logits' device"
        else:                                            # a vector beside the first tensor may notice first
            words = "GPU tensors|(a_scale|mean): 6 elements of torch.float32 on cpu|tokens: on the logits' device" if k == first \
                else "GPU tensors on one device|(mean): 6 elements of torch.float32 on cpu"
        with pytest.raises(ValueError, match=words):
            f(**{**kw, k: kw[k].cpu()})
    if "status" in kw:
        with pytest.raises(ValueError, match="GPU tensors on one device"):
            f(**{**kw, "status": torch.zeros(1, dtype=torch.int32)})
