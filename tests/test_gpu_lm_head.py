"""The language-model operators as they are used together: a training step of a
norm, an integer linear layer and the log probabilities of given tokens against
the same chain in 64 bits; serving a token at a time; captured graphs, several
streams and the step tape; rows farther apart than 32 bits reach."""
import pytest
import torch

from lm_util import DEV, HALF, U, codes, normal, quantized, within

pytestmark = pytest.mark.gpu


def _model(seed, D, V, dtype):
    w = normal(seed, V, D).float() / D ** 0.5
    wq, ws = quantized(w.double(), 8, False)
    return dict(gamma=(1 + 0.1 * normal(seed + 1, D)).to(dtype).to(DEV), beta=(0.1 * normal(seed + 2, D)).to(dtype).to(DEV),
                w=wq.to(DEV), ws=ws.to(DEV), bias=(0.1 * normal(seed + 3, V)).float().to(DEV))


def _step(iseg, p, x, tokens, g_lp, g_h, out_dtype=torch.float32, status=None):
    """Forward and backward of norm -> linear -> log probabilities."""
    y, mean, rstd = iseg.layernorm_fwd(x, p["gamma"], p["beta"], status=status)
    logits, q, s = iseg.linear_i8_fwd(y, p["w"], p["ws"], p["bias"], out_dtype=out_dtype, status=status)
    lp, lse, ent, ids, tlp = iseg.logprob_fwd(logits, tokens, top_k=4, status=status)
    dl = iseg.logprob_bwd(logits, tokens, lse, ent, g_lp, g_h, status=status)
    dy, dw, db = iseg.linear_i8_bwd(dl, q, s, p["w"], p["ws"], w_t=p.get("w_t"), want_bias=True, out_dtype=y.dtype, status=status)
    dx, dgamma, dbeta = iseg.layernorm_bwd(dy.view(x.shape), x, p["gamma"], mean, rstd)
    return dict(y=y, mean=mean, rstd=rstd, logits=logits, q=q, s=s, lp=lp, lse=lse, ent=ent, ids=ids, tlp=tlp, dl=dl, dy=dy, dw=dw,
                db=db, dx=dx, dgamma=dgamma, dbeta=dbeta)


@pytest.mark.parametrize("M,D,V", [(1, 64, 100), (7, 96, 1000), (130, 256, 517), (300, 512, 2048)])
def test_training_step(M, D, V):
    from paper_2011_14504_amd import iseg
    p = _model(M, D, V, torch.float32)
    x, tokens = normal(5, M, D).float(), (normal(6, M).abs() * 1e6).long() % V
    if M > 2:
        tokens[2] = -1
    g_lp, g_h = normal(7, M).float() / M, 0.01 * normal(8, M).float() / M
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    r = _step(iseg, p, x.to(DEV), tokens.to(DEV), g_lp.to(DEV), g_h.to(DEV), status=st)
    assert iseg.iseg_status_read(st) == 0
    c = {k: v.cpu() for k, v in r.items()}
    pc = {k: v.cpu() for k, v in p.items()}
    # every stage against the formulas in 64 bits on the stage before it: the
    # quantizers between them round, so a difference is not carried through them
    gamma, beta, w, ws, bias = (pc[k].double() for k in ("gamma", "beta", "w", "ws", "bias"))
    xd = x.double()
    mean = xd.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((xd - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    xh = (xd - mean) * rstd
    within(c["y"], xh * gamma + beta, 100 * U * (xh.abs() + 1) * gamma.abs() + 2 * U * (xh * gamma + beta).abs(), "y")
    q, s = quantized(c["y"].double(), 8, False)
    assert torch.equal(c["q"], q) and torch.equal(c["s"], s)
    prod = (q.double() @ w.t()) * s.double()[:, None] * ws
    within(c["logits"], prod + bias, 4 * U * (prod.abs() + bias.abs()), "logits")
    l = c["logits"].double()
    lse = torch.logsumexp(l, 1)
    lp = l - lse[:, None]
    pr = lp.exp()
    ent = -(pr * lp).sum(1)
    given = tokens >= 0
    at = torch.where(given, lp.gather(1, tokens.clamp_min(0)[:, None])[:, 0], torch.zeros(M, dtype=torch.float64))
    within(c["lp"], at, 400 * U * (1 + at.abs()), "logprob")
    within(c["ent"], ent, 1200 * U * (1 + ent), "entropy")
    val, ids = torch.sort(l, dim=1, descending=True, stable=True)
    assert torch.equal(c["ids"], ids[:, :4].int())
    g = g_lp.double() * given
    dl = -pr * (g[:, None] + g_h.double()[:, None] * (lp + ent[:, None]))
    size = pr * (g.abs()[:, None] + g_h.double().abs()[:, None] * (lp.abs() + ent[:, None]))
    dl[given.nonzero()[:, 0], tokens[given]] += g[given]
    # the kernel's own lse and entropy enter: their errors are those bounded above
    within(c["dl"], dl, 2000 * U * size + 2 * U * dl.abs(), "dlogits")
    q2, s2 = quantized(c["dl"].double() * ws, 8, False)
    dy = (q2.double() @ w) * s2.double()[:, None]
    within(c["dy"], dy, 4 * U * dy.abs(), "dy")
    q3, s3 = quantized((c["dl"].double() * s.double()[:, None]).t().contiguous(), 8, False)
    dw = (q3.double() @ q.double()) * s3.double()[:, None]
    within(c["dw"], dw, 4 * U * dw.abs(), "dw")
    within(c["db"], c["dl"].double().sum(0), (M + 4) * U * c["dl"].double().abs().sum(0), "dbias")
    gg = c["dy"].double() * gamma
    want = rstd * (gg - gg.mean(1, keepdim=True) - xh * (gg * xh).mean(1, keepdim=True))
    scale = rstd * (gg.abs() + (1 + xh.abs()) * (gg.abs() * (1 + xh.abs())).mean(1, keepdim=True))
    within(c["dx"], want, 200 * U * scale, "dx")
    t = c["dy"].double() * xh
    within(c["dgamma"], t.sum(0), 300 * U * (t.abs() + c["dy"].double().abs()).sum(0), "dgamma")
    within(c["dbeta"], c["dy"].double().sum(0), 300 * U * c["dy"].double().abs().sum(0), "dbeta")


def test_tokens_one_at_a_time_give_the_batch():
    """Serving: a token alone and in a batch has the same logits, log
    probabilities up to the order of a sum, and alternatives."""
    from paper_2011_14504_amd import iseg
    D, V, M = 384, 5000, 40
    p = _model(3, D, V, torch.bfloat16)
    x = normal(9, M, D).to(torch.bfloat16).to(DEV)
    tok = ((normal(10, M).abs() * 1e6).long() % V).to(DEV)

    def run(rows):
        y, _, _ = iseg.layernorm_fwd(x[rows], p["gamma"], p["beta"])
        lg, _, _ = iseg.linear_i8_fwd(y, p["w"], p["ws"], p["bias"], out_dtype=torch.float32)
        return (lg,) + iseg.logprob_fwd(lg, tok[rows], top_k=8)

    whole = run(slice(0, M))
    for i in (0, 1, 17, M - 1):
        one = run(slice(i, i + 1))
        assert torch.equal(one[0][0], whole[0][i]) and torch.equal(one[4][0], whole[4][i])
        for k in (1, 2, 3, 5):
            within(one[k][0], whole[k][i].double().cpu(), 800 * U * (1 + whole[k][i].double().abs().cpu()), k)


def test_captured_steps_replay():
    """Two captured training steps replay like eager ones, each several times,
    with eager work and synchronizations between, and both at once."""
    from paper_2011_14504_amd import iseg
    M, D, V = 200, 320, 3001
    p = _model(1, D, V, torch.bfloat16)
    p["w_t"] = iseg.transpose_i8(p["w"])
    bufs = []
    for k in range(2):
        b = dict(x=torch.zeros(M, D, dtype=torch.bfloat16, device=DEV), tok=torch.zeros(M, dtype=torch.int64, device=DEV),
                 g=torch.zeros(M, device=DEV), h=torch.zeros(M, device=DEV))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            _step(iseg, p, b["x"], b["tok"], b["g"], b["h"], torch.bfloat16)
        torch.cuda.current_stream().wait_stream(s)
        b["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(b["graph"]):
            b["out"] = _step(iseg, p, b["x"], b["tok"], b["g"], b["h"], torch.bfloat16)
        bufs.append(b)

    def load(b, seed):
        b["x"].copy_(normal(seed, M, D))
        b["tok"].copy_((normal(seed + 1, M).abs() * 1e6).long() % V)
        b["g"].copy_(normal(seed + 2, M) / M)
        b["h"].copy_(0.01 * normal(seed + 3, M) / M)
        return _step(iseg, p, b["x"], b["tok"], b["g"], b["h"], torch.bfloat16)

    for rep in range(3):
        for k, b in enumerate(bufs):
            want = load(b, 100 * rep + 10 * k)
            b["graph"].replay()
            torch.cuda.synchronize()
            for n in want:
                assert torch.equal(b["out"][n], want[n]), (rep, k, n)
    # both at once, on streams of their own
    want = [load(b, 900 + 10 * k) for k, b in enumerate(bufs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in bufs]
    for _ in range(3):
        for b, s in zip(bufs, streams):
            with torch.cuda.stream(s):
                b["graph"].replay()
    torch.cuda.synchronize()
    for b, w in zip(bufs, want):
        for n in w:
            assert torch.equal(b["out"][n], w[n]), n


def test_streams_at_once():
    from paper_2011_14504_amd import iseg
    M, D, V = 150, 200, 4099
    p = _model(2, D, V, torch.bfloat16)
    ins = []
    for k in range(4):
        ins.append((normal(k, M, D).to(torch.bfloat16).to(DEV), ((normal(k + 9, M).abs() * 1e6).long() % V).to(DEV),
                    (normal(k + 20, M) / M).float().to(DEV), (normal(k + 30, M) / M).float().to(DEV)))
    want = [_step(iseg, p, *i, torch.bfloat16) for i in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    for _ in range(3):
        got = []
        for i, s in zip(ins, streams):
            with torch.cuda.stream(s):
                got.append(_step(iseg, p, *i, torch.bfloat16))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for n in w:
                assert torch.equal(g[n], w[n]), n


def test_tape_replays_a_step():
    from paper_2011_14504_amd import iseg
    M, D, V = 33, 128, 500
    p = _model(4, D, V, torch.float32)
    p["w_t"] = iseg.transpose_i8(p["w"])
    x, tok = normal(1, M, D).float().to(DEV), ((normal(2, M).abs() * 1e6).long() % V).to(DEV)
    g, h = (normal(3, M) / M).float().to(DEV), (normal(4, M) / M).float().to(DEV)
    tape = iseg.Tape(0)
    with tape:
        out = _step(iseg, p, x, tok, g, h)
    assert tape.size() == 6                     # three forward, three backward
    for seed in (50, 60):
        x.copy_(normal(seed, M, D))
        tok.copy_((normal(seed + 1, M).abs() * 1e6).long() % V)
        tape.run(0)
        torch.cuda.synchronize()
        want = _step(iseg, p, x, tok, g, h)
        for n in want:
            assert torch.equal(out[n], want[n]), n
    with pytest.raises(iseg.IsegError):
        with iseg.Tape(0):
            iseg.layernorm_fwd(x.t())           # would copy outside the recorded calls
    tape.close()


@pytest.mark.parametrize("C", [300, 5, 40000])
def test_rows_past_32_bits(C):
    """Row strides whose last rows start past 2^31 elements and 2^32 bytes."""
    from paper_2011_14504_amd import iseg
    M, ld = 40, 1 << 26
    buf = torch.empty(M * ld, dtype=torch.bfloat16, device=DEV)
    x = buf.view(M, ld)[:, :C]
    x.copy_(normal(1, M, C))
    xc = x.contiguous()
    for a, b in zip(iseg.layernorm_fwd(x), iseg.layernorm_fwd(xc)):
        assert torch.equal(a, b)
    _, mean, rstd = iseg.layernorm_fwd(xc)
    for a, b in zip(iseg.layernorm_bwd(x, x, None, mean, rstd), iseg.layernorm_bwd(xc, xc, None, mean, rstd)):
        assert torch.equal(a, b)
    for f in (iseg.quantize_rows, iseg.quantize_cols):
        for a, b in zip(f(x)[:2], f(xc)[:2]):
            assert torch.equal(a, b)
    tok = torch.arange(M, device=DEV) % C
    got, want = iseg.logprob_fwd(x, tok, top_k=5), iseg.logprob_fwd(xc, tok, top_k=5)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    one = torch.ones(M, device=DEV)
    assert torch.equal(iseg.logprob_bwd(x, tok, got[1], got[2], one, one), iseg.logprob_bwd(xc, tok, got[1], got[2], one, one))
    cb = buf.view(torch.int8)[: M * (ld * 2)].view(M, ld * 2)
    a = cb[:, :C]
    a.copy_(codes(2, M, C))
    ac = a.contiguous()
    want = (ac.double() @ ac.double().t()).float()
    assert torch.equal(iseg.matmul_i8(a, a), want) and torch.equal(iseg.matmul_i8(a[:20], a), want[:20])
    off = cb[:, 3:C]                              # off 16 bytes: packed first
    assert torch.equal(iseg.matmul_i8(off, off), (ac[:, 3:].double() @ ac[:, 3:].double().t()).float())
    assert torch.equal(iseg.transpose_i8(a), ac.t())
