"""Operators of language models on the integer dataflow, as measurable cases.

  norm    layer normalization, forward and backward
  matmul  int8 x int8 products with a scale for each token and each channel
  linear  a linear layer in integers: its input quantized per token, then the
          product with int8 weights; and its backward, which quantizes the
          error per token and per channel for the two products of the gradients
  logprob log probabilities of given tokens with the entropy and the most
          likely alternatives of each row, and their gradient

`run` computes them in elementary torch operations, or, where `own` is true,
by the calls that a program makes of paper_2011_14504_amd.iseg.
"""
import math

import torch

own = False

DEV = "cuda:0"
_DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_ES = {"bf16": 2, "fp16": 2, "fp32": 4}
_EPS = 1e-5
_MAX_WORK = 2 * 8192 ** 3           # of a drawn product
_MAX_ELEMS = 16384 * 4096           # of a drawn row operator


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _norm(way, M, C, t, ld, **kw):
    return dict(op="norm", way=way, M=M, C=C, t=t, ld=ld, **kw)


def _product(op, way, M, N, K, t, bias, **kw):
    return dict(op=op, way=way, M=M, N=N, K=K, t=t, bias=bias, **kw)


def _logprob(way, M, V, t, ld, k, mask, **kw):
    return dict(op="logprob", way=way, M=M, V=V, t=t, ld=ld, k=k, mask=mask, **kw)


def listed():
    return [
        # four tokens of a decoding step: one launch and its latency
        _norm("fwd", 4, 2048, "bf16", 2048, name="norm-fwd-4x2048"),
        # the tokens of a large training batch, bound by memory
        _norm("fwd", 16384, 4096, "bf16", 4096, name="norm-fwd-16384x4096"),
        # the backward of a training batch at odd sizes in fp32
        _norm("bwd", 5003, 1537, "fp32", 1537, name="norm-bwd-5003x1537-fp32"),
        # a decoding step of eight tokens through a wide layer: the weights' bytes
        _product("matmul", "fwd", 8, 12288, 4096, "bf16", False, name="matmul-8x12288x4096"),
        # odd sizes whose rows start off every alignment
        _product("matmul", "fwd", 509, 1001, 1543, "fp32", True, name="matmul-509x1001x1543"),
        # a long prompt or a training batch through a large square layer
        _product("matmul", "fwd", 8192, 8192, 8192, "bf16", False, name="matmul-8192x8192x8192"),
        # one token through a whole linear layer, its quantizer included
        _product("linear", "fwd", 1, 4096, 4096, "bf16", True, name="linear-1x4096x4096"),
        # an ordinary prompt through a linear layer that widens
        _product("linear", "fwd", 2048, 8192, 2048, "fp16", True, name="linear-2048x8192x2048"),
        # the backward of a linear layer in a training step
        _product("linear", "bwd", 4096, 4096, 4096, "bf16", True, name="linear-bwd-4096x4096x4096"),
        # the tokens of a decoding step, with the twenty best alternatives
        _logprob("fwd", 4, 131072, "bf16", 131072, 20, False, name="logprob-4x131072-top20"),
        # the scoring of given texts over a padded vocabulary of odd size, in
        # which some tokens are banned and some positions hold no token
        _logprob("fwd", 2048, 50021, "fp32", 50048, 5, True, name="logprob-2048x50021-top5"),
        # the gradient of log probabilities and entropies in a training step
        _logprob("bwd", 4096, 32768, "bf16", 32768, 0, False, name="logprob-bwd-4096x32768"),
    ]


def _logu(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dim(rng, lo, hi):
    """A size of [lo, hi]: half of them multiples of 64, the others as they fall."""
    n = _logu(rng, lo, hi)
    return min(hi, max(lo, (n + 63) // 64 * 64)) if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(("norm", "matmul", "linear", "logprob"))
    t = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if op == "norm":
        C = _dim(rng, 64, 16384)
        M = _logu(rng, 1, max(1, min(65536, _MAX_ELEMS // C)))
        return _norm(rng.choice(("fwd", "bwd")), M, C, t, C + rng.choice((0, 0, 8, 24)))
    if op == "logprob":
        V = _dim(rng, 1000, 262144)
        M = _logu(rng, 1, max(1, min(8192, _MAX_ELEMS // V)))
        way = rng.choice(("fwd", "fwd", "bwd"))
        return _logprob(way, M, V, t, V + rng.choice((0, 0, 7, 64)), rng.choice((0, 1, 5, 20)) if way == "fwd" else 0,
                        rng.random() < 0.5)
    while True:
        way = "bwd" if op == "linear" and rng.random() < 0.4 else "fwd"
        M = _logu(rng, 1, 16) if way == "fwd" and rng.random() < 0.4 else _dim(rng, 16, 8192)
        N, K = _dim(rng, 256, 16384), _dim(rng, 256, 16384)
        if M * N * K * (4 if way == "bwd" else 2) <= _MAX_WORK // 2:
            return _product(op, way, M, N, K, t, rng.random() < 0.5)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _codes(gen, rows, cols):
    """Bell-shaped int8 codes whose rows reach the end of the range."""
    n = torch.randn(rows, cols, device=DEV, generator=gen) * 32
    return n.round_().clamp_(-127, 127).to(torch.int8)


def _strided(x, ld):
    """x in rows that are ld apart."""
    buf = torch.zeros(x.shape[0], ld, dtype=x.dtype, device=x.device)
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt = _DT[case["t"]]

    def randn(*shape):
        return torch.randn(*shape, device=DEV, generator=gen)

    st = dict(case=case)
    if case["op"] == "norm":
        M, C = case["M"], case["C"]
        # a residual stream: an offset and a scale of each row's own, and a few loud channels
        loud = 1 + 9 * (torch.rand(C, device=DEV, generator=gen) < 0.01).float()
        x = randn(M, C) * loud * (0.5 + torch.rand(M, 1, device=DEV, generator=gen)) + 0.2 * randn(M, 1)
        st["x"] = _strided(x.to(dt), case["ld"])
        st["gamma"] = (1 + 0.1 * randn(C)).to(dt)
        st["beta"] = (0.1 * randn(C)).to(dt)
        if case["way"] == "bwd":
            st["dy"] = (randn(M, C) * 1e-2).to(dt)
            xd = st["x"].double()
            mean = xd.mean(1)
            st["mean"] = mean.float()
            st["rstd"] = (((xd - mean[:, None]) ** 2).mean(1) + _EPS).rsqrt().float()
    elif case["op"] in ("matmul", "linear"):
        M, N, K = case["M"], case["N"], case["K"]
        st["w"] = _codes(gen, N, K)
        st["w_scale"] = (0.5 + torch.rand(N, device=DEV, generator=gen)) / (32 * math.sqrt(K))
        st["bias"] = 0.1 * randn(N) if case["bias"] else None
        if case["op"] == "matmul" or case["way"] == "bwd":
            st["a"] = _codes(gen, M, K)
            st["a_scale"] = (0.5 + torch.rand(M, device=DEV, generator=gen)) / 32
        else:
            st["x"] = (randn(M, K) * (0.5 + torch.rand(M, 1, device=DEV, generator=gen))).to(dt)
        if case["way"] == "bwd":
            st["dy"] = (randn(M, N) * 1e-3).to(dt)
    else:
        M, V = case["M"], case["V"]
        x = randn(M, V) * 2.5
        st["tokens"] = torch.randint(V, (M,), device=DEV, generator=gen)
        # a model that has learnt something: the given token is often a likely one
        rows = torch.arange(M, device=DEV)
        x[rows, st["tokens"]] += 12 * torch.rand(M, device=DEV, generator=gen)
        if case["mask"]:
            banned = torch.rand(V, device=DEV, generator=gen) < 0.05
            x[:, banned] = -math.inf
            st["tokens"][torch.rand(M, device=DEV, generator=gen) < 0.1] = -100
        st["logits"] = _strided(x.to(dt), case["ld"])
        if case["way"] == "bwd":
            p = torch.log_softmax(st["logits"].double(), 1)
            st["lse"] = torch.logsumexp(st["logits"].double(), 1).float()
            st["entropy"] = -(p.exp() * p.clamp_min(-1e9)).sum(1).float()
            st["g_logprob"] = randn(M) / M
            st["g_entropy"] = -0.01 * torch.rand(M, device=DEV, generator=gen) / M
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["op"] == "norm":
        return _plain_norm(case, state)
    if case["op"] == "logprob":
        return _plain_logprob(case, state)
    return _plain_product(case, state)


def _run_own(case, st):
    from paper_2011_14504_amd import iseg
    dt = _DT[case["t"]]
    if case["op"] == "norm":
        if case["way"] == "fwd":
            return iseg.layernorm_fwd(st["x"], st["gamma"], st["beta"], eps=_EPS)
        return iseg.layernorm_bwd(st["dy"], st["x"], st["gamma"], st["mean"], st["rstd"])
    if case["op"] == "matmul":
        return iseg.matmul_i8(st["a"], st["w"], st["a_scale"], st["w_scale"], st["bias"], out_dtype=dt)
    if case["op"] == "linear":
        if case["way"] == "fwd":
            return iseg.linear_i8_fwd(st["x"], st["w"], st["w_scale"], st["bias"])[0]
        # a training step changes the weights after each backward, so their
        # transposition is part of every call
        return iseg.linear_i8_bwd(st["dy"], st["a"], st["a_scale"], st["w"], st["w_scale"],
                                  want_bias=case["bias"])[:3 if case["bias"] else 2]
    if case["way"] == "fwd":
        out = iseg.logprob_fwd(st["logits"], st["tokens"], top_k=case["k"])
        return out if case["k"] else out[:3]
    return iseg.logprob_bwd(st["logits"], st["tokens"], st["lse"], st["entropy"], st["g_logprob"], st["g_entropy"])


def _plain_norm(case, st):
    x, gamma = st["x"].float(), st["gamma"].float()
    dt = _DT[case["t"]]
    if case["way"] == "fwd":
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = torch.rsqrt((d * d).mean(1) + _EPS)
        return (d * rstd[:, None] * gamma + st["beta"].float()).to(dt), mean, rstd
    dy = st["dy"].float()
    xhat = (x - st["mean"][:, None]) * st["rstd"][:, None]
    g = dy * gamma
    dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * st["rstd"][:, None]
    return dx.to(dt), (dy * xhat).sum(0).to(dt), dy.sum(0).to(dt)


def _quantize(t):
    """Codes and scales of the rows of t (float64: half-steps are decided exactly)."""
    big = t.abs().amax(1)
    s = torch.where(big > 0, (big / 127).float().clamp_min(2.0 ** -126), torch.ones_like(big, dtype=torch.float32))
    return torch.floor(t / s.double()[:, None] + 0.5).clamp(-127, 127).float(), s


def _sums(a, b):
    """a b^T of codes held in float32: exact over 1024 products, added in int32."""
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.int32, device=a.device)
    for k in range(0, a.shape[1], 1024):
        out += (a[:, k:k + 1024] @ b[:, k:k + 1024].t()).to(torch.int32)
    return out.float()


def _plain_product(case, st):
    dt = _DT[case["t"]]
    w = st["w"].float()
    if case["way"] == "bwd":
        a, dy = st["a"].float(), st["dy"].double()
        q, s = _quantize(dy * st["w_scale"].double())
        da = _sums(q, w.t()) * s[:, None]
        q, s = _quantize((dy * st["a_scale"].double()[:, None]).t())
        dw = _sums(q, a.t()) * s[:, None]
        out = (da.to(dt), dw.to(dt))
        return out + (st["dy"].float().sum(0),) if case["bias"] else out
    if case["op"] == "linear":
        a, s = _quantize(st["x"].double())
    else:
        a, s = st["a"].float(), st["a_scale"]
    y = _sums(a, w) * s[:, None] * st["w_scale"]
    if case["bias"]:
        y = y + st["bias"]
    return y.to(dt)


def _plain_logprob(case, st):
    x, tok = st["logits"].float(), st["tokens"]
    if case["way"] == "bwd":
        lp = x - st["lse"][:, None]
        p = torch.exp(lp)
        lp = torch.where(p > 0, lp, torch.zeros_like(lp))
        g = torch.where(tok >= 0, st["g_logprob"], torch.zeros_like(st["g_logprob"]))
        dx = -p * (g[:, None] + st["g_entropy"][:, None] * (lp + st["entropy"][:, None]))
        hit = torch.arange(x.shape[1], device=x.device) == tok[:, None]
        return (dx + torch.where(hit, g[:, None], torch.zeros_like(dx))).to(_DT[case["t"]])
    m = x.amax(1)
    d = x - m[:, None]
    e = torch.exp(d)
    s = e.sum(1)
    logs = torch.log(s)
    entropy = logs - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1) / s
    at = d.gather(1, tok.clamp_min(0)[:, None])[:, 0]
    logprob = torch.where(tok >= 0, at - logs, torch.zeros_like(at))
    out = (logprob, m + logs, entropy)
    if case["k"] == 0:
        return out
    ids = torch.arange(x.shape[1], device=x.device, dtype=torch.int32)
    top, left = [], d.clone()
    for _ in range(case["k"]):
        best = left.amax(1, keepdim=True)
        i = torch.where(left == best, ids, x.shape[1]).amin(1)
        top.append(i)
        left.scatter_(1, i.long()[:, None], -math.inf)
    top = torch.stack(top, 1)
    return out + (top, d.gather(1, top.long()) - logs[:, None])


# ---------------------------------------------------------------------------
# work and the definition in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    es = _ES[case["t"]]
    if case["op"] == "norm":
        n = case["M"] * case["C"]
        if case["way"] == "fwd":
            return {"bytes": 2 * n * es + 8 * case["M"] + 2 * case["C"] * es, "flops": 8 * n}
        return {"bytes": 3 * n * es + 8 * case["M"] + 3 * case["C"] * es, "flops": 14 * n}
    if case["op"] == "logprob":
        n = case["M"] * case["V"]
        if case["way"] == "fwd":
            return {"bytes": n * es + case["M"] * (20 + 8 * case["k"]), "flops": 6 * n}
        return {"bytes": 2 * n * es + 24 * case["M"], "flops": 8 * n}
    M, N, K = case["M"], case["N"], case["K"]
    bias = 4 * N if case["bias"] else 0
    if case["way"] == "bwd":
        return {"bytes": M * N * es + (M * K + N * K) * (1 + es) + 4 * (M + N) + bias, "flops": 4 * M * N * K}
    a = M * K * es if case["op"] == "linear" else M * K + 4 * M
    return {"bytes": a + N * K + M * N * es + 4 * N + bias, "flops": 2 * M * N * K}


def exact(case, seed):
    st = prepare(case, seed)
    f8 = torch.float64
    if case["op"] == "norm":
        x, gamma = st["x"].to(f8), st["gamma"].to(f8)
        if case["way"] == "fwd":
            var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
            y = (x - mean) / torch.sqrt(var + _EPS) * gamma + st["beta"].to(f8)
            return y, mean[:, 0], 1 / torch.sqrt(var[:, 0] + _EPS)
        dy, r = st["dy"].to(f8), st["rstd"].to(f8)[:, None]
        xhat = (x - st["mean"].to(f8)[:, None]) * r
        C = x.shape[1]
        g = dy * gamma
        proj = (g.sum(1, keepdim=True) + xhat * (g * xhat).sum(1, keepdim=True)) / C
        return (g - proj) * r, torch.einsum("mc,mc->c", dy, xhat), torch.ones(len(dy), dtype=f8, device=DEV) @ dy
    if case["op"] == "logprob":
        x = st["logits"].to(f8)
        tok = st["tokens"]
        given = tok >= 0
        if case["way"] == "bwd":
            p = torch.exp(x - st["lse"].to(f8)[:, None])
            log_p = torch.log(p.clamp_min(1e-300))
            g = st["g_logprob"].to(f8) * given
            onehot = torch.zeros_like(p)
            onehot[given.nonzero()[:, 0], tok[given]] = 1
            return g[:, None] * (onehot - p) - st["g_entropy"].to(f8)[:, None] * p * (log_p + st["entropy"].to(f8)[:, None])
        lse = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[:, None])
        entropy = -torch.xlogy(p, p).sum(1)
        lp = x[torch.arange(len(tok), device=DEV), tok.clamp_min(0)] - lse
        out = (torch.where(given, lp, torch.zeros_like(lp)), lse, entropy)
        if case["k"] == 0:
            return out
        val, ids = torch.sort(x, dim=1, descending=True, stable=True)
        return out + (ids[:, :case["k"]].to(torch.int32), val[:, :case["k"]] - lse[:, None])
    w, sw = st["w"].to(f8), st["w_scale"].to(f8)

    def codes(v):
        """Row v rounded half up onto 255 levels: values and not codes."""
        top = v.abs().max(dim=1, keepdim=True).values
        step = torch.maximum((top / 127).to(torch.float32), torch.tensor(2.0 ** -126, device=DEV)).to(f8)
        return torch.minimum(torch.ceil(torch.floor(2 * v / step) / 2), torch.tensor(127.0, dtype=f8, device=DEV)) * step

    if case["way"] == "bwd":
        dy, a = st["dy"].to(f8), st["a"].to(f8)
        da = codes(dy * sw) @ w
        dw = codes((dy * st["a_scale"].to(f8)[:, None]).t().contiguous()) @ a
        return (da, dw, dy.sum(0)) if case["bias"] else (da, dw)
    a = codes(st["x"].to(f8)) if case["op"] == "linear" else st["a"].to(f8) * st["a_scale"].to(f8)[:, None]
    y = a @ w.t() * sw
    return y + st["bias"].to(f8) if case["bias"] else y
