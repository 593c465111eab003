"""int8 products with row scales, the row and column quantizers and the
transposition, against integer arithmetic and the formulas in 64 bits."""
import pytest
import torch

from lm_util import DEV, DT, HALF, TINY, U, codes, normal, quantized, strided, within

pytestmark = pytest.mark.gpu

# (M, N, K, out type, gap of a's rows, gap of b's rows, scales and bias)
PRODUCTS = [
    (1, 1, 1, "fp32", 0, 0, True), (1, 5, 3, "bf16", 0, 0, False), (2, 64, 64, "fp32", 0, 0, True), (7, 100, 17, "fp16", 0, 0, True),
    (1, 1000, 4096, "bf16", 0, 0, True), (3, 513, 1000, "fp32", 8, 0, True), (8, 4096, 2048, "bf16", 0, 0, True),
    (16, 300, 8192, "fp32", 16, 32, False), (17, 128, 640, "bf16", 0, 0, True), (31, 77, 65, "fp32", 1, 2, True), (33, 130, 129, "fp16", 15, 15, True),
    (64, 64, 63, "fp32", 0, 1, True), (65, 65, 4097, "fp32", 0, 0, True), (100, 1003, 1536, "bf16", 0, 0, True),
    (128, 128, 128, "fp32", 0, 0, False), (129, 257, 192, "fp32", 16, 16, True), (255, 256, 512, "bf16", 0, 0, True),
    (256, 512, 1024, "bf16", 0, 0, True), (300, 700, 1543, "fp32", 0, 0, True), (513, 1025, 336, "fp16", 0, 0, True), (1000, 2000, 80, "fp32", 0, 0, True),
    (520, 512, 4096, "bf16", 64, 0, True), (1, 64, 131071, "fp32", 0, 0, False), (40, 70, 131071, "fp32", 1, 0, False),
    (5, 6, 0, "fp32", 0, 0, True), (2049, 33, 48, "bf16", 0, 0, False), (4096, 64, 16, "fp32", 0, 0, True),
]


def _sums(a, b):
    """Exact int64 sums through float64 (products below 2^31, sums below 2^53)."""
    return a.double() @ b.double().t()


def _operand(seed, rows, K, gap):
    return strided(codes(seed, rows, K), K + gap, 77) if gap else codes(seed, rows, K).to(DEV)


@pytest.mark.parametrize("case", PRODUCTS, ids=str)
def test_product(case):
    from paper_2011_14504_amd import iseg
    M, N, K, t, ga, gb, full = case
    print(f"[matmul_i8] {case}", flush=True)
    a, b = _operand(M + K, M, K, ga), _operand(N + 2 * K, N, K, gb)
    sa = (normal(1, M).abs() + 0.1).float() if full else None
    sb = (normal(2, N).abs() * 1e-4 + 1e-5).float() if full else None
    bias = normal(3, N).float() if full else None
    got = iseg.matmul_i8(a, b, *(None if v is None else v.to(DEV) for v in (sa, sb, bias)), out_dtype=DT[t])
    want = _sums(a.cpu(), b.cpu())
    if full:
        want = want * sa.double()[:, None] * sb.double()
    if t == "fp16":
        assert want.abs().max() < 6e4
    # the sum's rounding and two products': 3 half-steps; the bias's addition one more
    e = 3 * U * want.abs()
    if full:
        want = want + bias.double()
        e = e + U * want.abs()
    if t == "fp32" and not full:
        assert torch.equal(got.cpu(), want.float())          # one rounding of an exact sum
    within(got, want, e + HALF[t] * (want.abs() + e) + TINY[t], "product")
    assert got.dtype == DT[t] and got.shape == (M, N)


# sizes that reach every way a product is run: few rows, each tile, a reduction
# in parts; with whole and broken tiles and reductions, and rows off 16 bytes
PATHS = [(11, 416, 14279), (1, 33, 1025), (32, 700, 2307), (15, 9000, 300), (16, 20, 8200), (20, 100, 500), (32, 5000, 272), (33, 20, 2050), (40, 40, 9000), (64, 2048, 4096), (512, 1024, 1536), (1024, 2048, 400),
         (1000, 2050, 130), (1500, 2048, 1000), (2048, 2048, 128), (4000, 4100, 160), (4096, 8192, 256), (4100, 4100, 1), (260, 16000, 100), (2300, 3700, 1100), (3712, 2200, 300), (3200, 3200, 2000), (1900, 6100, 400)]


@pytest.mark.parametrize("case", PATHS, ids=str)
def test_every_path_of_a_product(case):
    from paper_2011_14504_amd import iseg
    M, N, K = case
    print(f"[matmul_i8 paths] {case}", flush=True)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(M + N + K)
    a, b = (torch.randint(-128, 128, (r, K), dtype=torch.int8, device=DEV, generator=gen) for r in (M, N))
    want = (a.double() @ b.double().t()).float()
    pad = (K + 15) // 16 * 16
    for la, lb, off in ((pad, pad, 0), (K, pad + 16, 0), (pad, pad + 32, 16), (pad + 1, K, 3), (pad, pad, 5)):
        ba = torch.full((M * la + off,), 99, dtype=torch.int8, device=DEV)
        bb = torch.full((N * lb + off,), -99, dtype=torch.int8, device=DEV)
        va, vb = (t[off:].view(r, l)[:, :K] for t, r, l in ((ba, M, la), (bb, N, lb)))
        va.copy_(a)
        vb.copy_(b)
        assert torch.equal(iseg.matmul_i8(va, vb), want), (la, lb, off)


def test_product_extremes():
    """-128 codes at the longest reduction: the sums reach 2^31 - 2^14."""
    from paper_2011_14504_amd import iseg
    a = torch.full((3, 131071), -128, dtype=torch.int8, device=DEV)
    got = iseg.matmul_i8(a, a)
    assert torch.equal(got.cpu().double(), torch.full((3, 3), 131071.0 * 16384))


def test_product_scales_one_by_one():
    from paper_2011_14504_amd import iseg
    a, b = codes(1, 20, 96).to(DEV), codes(2, 30, 96).to(DEV)
    s = _sums(a.cpu(), b.cpu())
    sa, sb, bias = normal(1, 20).float(), normal(2, 30).float(), normal(3, 30).float()
    within(iseg.matmul_i8(a, b, sa.to(DEV)), s * sa.double()[:, None], 2 * U * (s * sa.double()[:, None]).abs(), "sa")
    within(iseg.matmul_i8(a, b, None, sb.to(DEV)), s * sb.double(), 2 * U * (s * sb.double()).abs(), "sb")
    within(iseg.matmul_i8(a, b, None, None, bias.to(DEV)), s + bias.double(), 2 * U * (s.abs() + bias.double().abs()), "bias")


def test_product_leaves_what_lies_beside_its_output():
    from paper_2011_14504_amd import iseg
    for M, N, K in ((3, 50, 64), (70, 50, 64), (200, 300, 256)):
        a, b = codes(1, M, K).to(DEV), codes(2, N, K).to(DEV)
        out = torch.full((M + 2, N + 9), 7.0, device=DEV)
        g = iseg.MatmulGeom(M, N, K, K, K, N + 9, iseg.ISEG_F32, 0)
        ws = torch.empty(max(iseg.lib().iseg_matmul_i8_ws(iseg.C.byref(g)), 256), dtype=torch.uint8, device=DEV)
        iseg.iseg_matmul_i8(a, None, b, None, None, g, out, ws)
        assert torch.equal(out[:M, :N].cpu().double(), _sums(a.cpu(), b.cpu()))
        assert bool((out[M:] == 7).all()) and bool((out[:, N:] == 7).all())


# (M, C, type, gap, bits, power-of-two scale, with mul)
QUANT = [
    (1, 1, "fp32", 0, 8, False, False), (3, 17, "bf16", 0, 8, False, True), (5, 64, "fp16", 3, 8, True, False), (64, 63, "fp32", 1, 8, False, True),
    (65, 130, "bf16", 0, 4, True, True), (1, 4096, "bf16", 0, 8, False, False), (300, 1000, "fp32", 0, 8, False, False),
    (130, 2052, "bf16", 4, 8, False, True), (9, 8193, "fp16", 0, 8, False, False), (7, 16384, "bf16", 0, 8, True, False),
    (6, 2100, "fp32", 0, 8, False, True), (4, 4104, "fp32", 0, 8, False, False), (5, 6148, "fp32", 2, 8, False, True), (4, 12300, "bf16", 0, 8, False, True),
    (1000, 72, "fp32", 0, 8, True, True), (4100, 33, "bf16", 0, 8, False, True), (3, 20000, "fp32", 0, 2, False, False), (2, 40003, "bf16", 0, 8, False, True),
    (300, 9001, "bf16", 1, 8, False, True), (70, 12000, "fp32", 0, 8, False, False), (3, 16383, "fp32", 0, 8, False, True), (3, 16389, "fp32", 0, 8, False, True),
    (3, 24581, "bf16", 0, 8, False, False), (3, 32768, "fp16", 0, 8, True, False), (3, 40000, "bf16", 0, 8, False, False), (70000, 3, "fp32", 1, 8, False, True),
    (3, 32760, "bf16", 0, 8, False, True), (5, 20001, "fp16", 0, 8, False, True), (600, 16384, "bf16", 0, 8, False, True), (2100, 700, "fp32", 0, 8, False, True),
]


def _quant_input(case):
    M, C, t, gap, bits, pow2, with_mul = case
    x = (normal(M + 3 * C, M, C) * torch.exp(2 * normal(7, M, 1))).to(DT[t])
    if M > 2:
        x[1] = 0                                             # a row of zeros
        x[2] = x[2].sign()                                   # ties of the largest magnitude
    if C > 4:
        x[:, 3] = 0                                          # a column of zeros
    return x


@pytest.mark.parametrize("case", QUANT, ids=str)
def test_quantize_rows(case):
    from paper_2011_14504_amd import iseg
    M, C, t, gap, bits, pow2, with_mul = case
    print(f"[quantize_rows] {case}", flush=True)
    x = _quant_input(case)
    mul = (normal(4, C).abs() * 0.3 + 0.01).float() if with_mul else None
    q, s = iseg.quantize_rows(strided(x, C + gap, float("inf")), bits, iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX,
                              None if mul is None else mul.to(DEV))
    wq, ws = quantized(x.double() * (mul.double() if with_mul else 1.0), bits, pow2)
    assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)


@pytest.mark.parametrize("case", QUANT, ids=str)
def test_quantize_cols(case):
    from paper_2011_14504_amd import iseg
    M, C, t, gap, bits, pow2, with_mul = case
    print(f"[quantize_cols] {case}", flush=True)
    x = _quant_input(case)
    mul = (normal(4, M).abs() * 0.3 + 0.01).float() if with_mul else None
    xg = strided(x, C + gap, float("inf"))
    q, s, sums = iseg.quantize_cols(xg, bits, iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX,
                                    None if mul is None else mul.to(DEV), want_sums=True)
    v = x.double() * (mul.double()[:, None] if with_mul else 1.0)
    wq, ws = quantized(v.t().contiguous(), bits, pow2)
    assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)
    within(sums, x.double().sum(0), (M + 4) * U * x.double().abs().sum(0), "sums")
    q2, s2, none = iseg.quantize_cols(xg, bits, iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX,
                                      None if mul is None else mul.to(DEV))
    assert none is None and torch.equal(q2, q) and torch.equal(s2, s)


def test_quantize_decides_half_steps_exactly():
    """Values on, just below and just above every half-step of a scale that is
    no power of two and of one that is."""
    from paper_2011_14504_amd import iseg
    for big in (127.0, 100.3, 1e-3, 3.7e30, 2e-36):
        s = (torch.tensor(big, dtype=torch.float64).float().double() / 127).float().double()
        half = ((torch.arange(-127, 127).double() + 0.5) * s).float()
        row = torch.cat([half, torch.nextafter(half, torch.tensor(1e38)), torch.nextafter(half, torch.tensor(-1e38)),
                         torch.tensor([big])])
        x = torch.stack([row, row.flip(0)])
        for pow2 in (False, True):
            wq, ws = quantized(x.double(), 8, pow2)
            mode = iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX
            q, sc = iseg.quantize_rows(x.to(DEV), 8, mode)
            assert torch.equal(sc.cpu(), ws) and torch.equal(q.cpu(), wq), big
            q, sc, _ = iseg.quantize_cols(x.t().contiguous().to(DEV), 8, mode)
            assert torch.equal(sc.cpu(), ws) and torch.equal(q.cpu(), wq), big


def test_quantize_products_near_half_steps():
    """x mul on half-steps where the float32 product is not: the exact product decides."""
    from paper_2011_14504_amd import iseg
    gen = torch.Generator().manual_seed(3)
    for C in (5, 200, 3000):
        mul = (torch.rand(C, generator=gen) + 0.5).float()
        n = torch.randint(-127, 127, (40, C), generator=gen).double() + 0.5
        x = (n * 0.01 / mul.double()).float()
        x[:, 0] = (1.27 / mul[0].double()).float() * (1 + 2.0 ** -23 * torch.arange(40))
        wq, ws = quantized(x.double() * mul.double(), 8, False)
        q, s = iseg.quantize_rows(x.to(DEV), mul=mul.to(DEV))
        assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)
        q, s, _ = iseg.quantize_cols(x.t().contiguous().to(DEV), mul=mul.to(DEV))
        assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)


def test_quantize_tiny_huge_and_non_finite():
    from paper_2011_14504_amd import iseg
    x = torch.zeros(6, 40)
    x[0, 3], x[0, 5] = 1e-44, -3e-45                     # scale held at 2^-126
    x[1, 0], x[1, 1] = 3.4e38, -1.2e38
    x[2, 7] = 2.0 ** -120
    x[3, 9], x[3, 10] = -0.0, 1.0
    x[4] = normal(1, 40).float()
    x[5] = normal(2, 40).float() * 1e-39
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for pow2 in (False, True):
        mode = iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX
        wq, ws = quantized(x.double(), 8, pow2)
        q, s = iseg.quantize_rows(x.to(DEV), 8, mode, status=st)
        assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)
        q, s, _ = iseg.quantize_cols(x.t().contiguous().to(DEV), 8, mode, status=st)
        assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)
    assert iseg.iseg_status_read(st) == 0
    for bad in (float("nan"), float("inf"), -float("inf")):
        y = x.clone()
        y[4, 39] = bad
        wq, ws = quantized(x.double(), 8, False)
        q, s = iseg.quantize_rows(y.to(DEV), status=st)
        assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
        iseg.iseg_status_clear(st)
        keep = [0, 1, 2, 3, 5]
        assert torch.equal(s.cpu()[keep], ws[keep]) and torch.equal(q.cpu()[keep], wq[keep])
        assert bool(torch.isnan(s[4])) and not bool(q[4].any())
        q, s, _ = iseg.quantize_cols(y.t().contiguous().to(DEV), status=st)
        assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
        iseg.iseg_status_clear(st)
        assert torch.equal(s.cpu()[keep], ws[keep]) and torch.equal(q.cpu()[keep], wq[keep])
        assert bool(torch.isnan(s[4])) and not bool(q[4].any())
    # a product with mul that leaves float32: no scale
    q, s = iseg.quantize_rows(torch.full((1, 4), 3e38, device=DEV), mul=torch.full((4,), 1e30, device=DEV), status=st)
    assert bool(torch.isnan(s[0])) and iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
    # and one that leaves it below
    q, s = iseg.quantize_rows(torch.full((1, 4), 1e-38, device=DEV), mul=torch.full((4,), 1e-30, device=DEV))
    assert float(s[0]) == 2.0 ** -126 and not bool(q.any())
    q, s, _ = iseg.quantize_cols(torch.full((3, 9), 1e-38, device=DEV), mul=torch.full((3,), 1e-30, device=DEV))
    assert bool((s == 2.0 ** -126).all()) and not bool(q.any())
    # float32 products past the range whose scale is inside it
    for C in (3, 40):
        x = torch.full((3, C), 1e38, dtype=torch.float64)
        x[1, 0], x[2] = 3e38, -2.9e38
        mul = torch.linspace(60, 100, C, dtype=torch.float64).float()
        wq, ws = quantized(x.float().double() * mul.double(), 8, False)
        q, s = iseg.quantize_rows(x.float().to(DEV), mul=mul.to(DEV))
        assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)
        q, s, _ = iseg.quantize_cols(x.float().t().contiguous().to(DEV), mul=mul.to(DEV))
        assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)


@pytest.mark.parametrize("C", [3, 200, 1500, 5000, 9000, 33000])
def test_quantize_products_out_of_float_range(C):
    """Rows whose largest product is subnormal, 0 or infinite in float32, zero
    rows, and infinities that meet a zero."""
    from paper_2011_14504_amd import iseg
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    x = normal(1, 5, C).float()
    mul = (normal(2, C).abs() + 0.1).float()
    x[0] *= 1e-42
    x[1] = 0
    x[2] *= 1e-22
    x[3] = x[3].clamp(-3, 3) * 1e38
    for scale in (1.0, 1e-24):
        m = (mul * scale).float()
        wq, ws = quantized(x.double() * m.double(), 8, False)
        q, s = iseg.quantize_rows(x.to(DEV), mul=m.to(DEV), status=st)
        assert torch.equal(s.cpu(), ws) and torch.equal(q.cpu(), wq)
    assert iseg.iseg_status_read(st) == 0
    m = mul.clone()
    m[C // 2] = float("inf")
    q, s = iseg.quantize_rows(x.to(DEV), mul=m.to(DEV), status=st)
    assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
    assert bool(torch.isnan(s).all()) and not bool(q.any())


def test_linear_backward_empty():
    from paper_2011_14504_amd import iseg
    w, one = codes(1, 5, 16).to(DEV), torch.ones(5, device=DEV)
    dx, dw, db = iseg.linear_i8_bwd(torch.empty(0, 5, device=DEV), torch.empty(0, 16, dtype=torch.int8, device=DEV), one[:0], w, one, want_bias=True)
    assert dx.shape == (0, 16) and torch.equal(dw.cpu(), torch.zeros(5, 16)) and torch.equal(db.cpu(), torch.zeros(5))
    dx, dw, db = iseg.linear_i8_bwd(torch.empty(3, 0, device=DEV), torch.ones(3, 16, dtype=torch.int8, device=DEV), one[:3], w[:0], one[:0], want_bias=True)
    assert torch.equal(dx.cpu(), torch.zeros(3, 16)) and dw.shape == (0, 16) and db.shape == (0,)
    dx, dw, db = iseg.linear_i8_bwd(torch.ones(3, 5, device=DEV), torch.empty(3, 0, dtype=torch.int8, device=DEV), one[:3], torch.empty(5, 0, dtype=torch.int8, device=DEV), one,
                                    want_bias=True)
    assert dx.shape == (3, 0) and dw.shape == (5, 0) and torch.equal(db.cpu(), torch.full((5,), 3.0))


def test_linear_modes_strides_and_status():
    from paper_2011_14504_amd import iseg
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for M, K in ((2, 777), (40, 777)):
        x, w = normal(1, M, K).float(), codes(2, 50, K).clamp_min(-127)
        xg, wg = strided(x, K + 5, float("nan")), strided(w, K + 7, 99)
        for bits, pow2 in ((8, True), (4, False), (2, False)):
            y, q, s = iseg.linear_i8_fwd(xg, wg, None, None, bits, iseg.ISEG_SCALE_POW2 if pow2 else iseg.ISEG_SCALE_MAX, status=st)
            wq, ws = quantized(x.double(), bits, pow2)
            assert torch.equal(q.cpu(), wq) and torch.equal(s.cpu(), ws)
            p = _sums(wq, w) * ws.double()[:, None]
            within(y, p, 3 * U * p.abs(), "y")
        assert iseg.iseg_status_read(st) == 0
        x[1, 3] = float("nan")
        y, q, s = iseg.linear_i8_fwd(x.to(DEV), wg, status=st)
        assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
        iseg.iseg_status_clear(st)
        assert torch.isnan(y[1]).all() and bool(torch.isfinite(y[0]).all()) and not bool(q[1].any())
        y3, q3, _ = iseg.linear_i8_fwd(x.to(DEV).view(1, M, K), wg)
        assert y3.shape == (1, M, 50) and q3.shape == (M, K) and torch.equal(q3, q)
    y, q, s = iseg.linear_i8_fwd(torch.empty(0, 16, device=DEV), wg[:, :16])
    assert y.shape == (0, 50) and s.shape == (0,)
    y, q, s = iseg.linear_i8_fwd(torch.ones(3, 16, device=DEV), torch.empty(0, 16, dtype=torch.int8, device=DEV))
    assert y.shape == (3, 0) and bool((q == 127).all())
    y, q, s = iseg.linear_i8_fwd(torch.empty(3, 0, device=DEV), torch.empty(5, 0, dtype=torch.int8, device=DEV), None, torch.arange(5., device=DEV))
    assert torch.equal(y.cpu(), torch.arange(5.).expand(3, 5)) and bool((s == 1).all())


@pytest.mark.parametrize("C", [3, 300, 9000, 40000])
def test_every_row_width_leaves_gaps_and_flags(C):
    from paper_2011_14504_amd import iseg
    M, ld, st = 11, C + 13, torch.zeros(1, dtype=torch.int32, device=DEV)
    x = normal(C, M, C).float()
    mul = (normal(2, C).abs() + 0.1).float()
    xg = strided(x, ld, float("nan"))
    for m in (None, mul):
        wq, ws = quantized(x.double() * (1.0 if m is None else m.double()), 8, False)
        q = torch.full((M + 2, ld), 55, dtype=torch.int8, device=DEV)
        s = torch.full((M + 3,), 7.0, device=DEV)
        md = None if m is None else m.to(DEV)
        iseg.iseg_quantize_rows(xg, iseg.ISEG_F32, M, C, ld, md, 8, iseg.ISEG_SCALE_MAX, q, ld, s, st)
        assert torch.equal(q[:M, :C].cpu(), wq) and bool((q[M:] == 55).all()) and bool((q[:, C:] == 55).all())
        assert torch.equal(s[:M].cpu(), ws) and bool((s[M:] == 7).all()) and iseg.iseg_status_read(st) == 0
        for bad in (float("nan"), -float("inf")):
            z = x.clone()
            z[4, C - 1] = bad
            q, s = iseg.quantize_rows(z.to(DEV), mul=md, status=st)
            assert iseg.iseg_status_read(st) == iseg.ISEG_DEV_NONFINITE
            iseg.iseg_status_clear(st)
            keep = [i for i in range(M) if i != 4]
            assert torch.equal(q.cpu()[keep], wq[keep]) and bool(torch.isnan(s[4])) and not bool(q[4].any())


def test_quantize_empty():
    from paper_2011_14504_amd import iseg
    q, s = iseg.quantize_rows(torch.empty(0, 8, device=DEV))
    assert q.shape == (0, 8) and s.shape == (0,)
    q, s = iseg.quantize_rows(torch.empty(3, 0, device=DEV))
    assert q.shape == (3, 0) and torch.equal(s.cpu(), torch.ones(3))
    q, s, sums = iseg.quantize_cols(torch.empty(0, 5, device=DEV), want_sums=True)
    assert q.shape == (5, 0) and torch.equal(s.cpu(), torch.ones(5)) and torch.equal(sums.cpu(), torch.zeros(5))
    assert iseg.quantize_cols(torch.empty(4, 0, device=DEV))[0].shape == (0, 4)
    a = torch.empty(0, 16, dtype=torch.int8, device=DEV)
    b = codes(1, 4, 16).to(DEV)
    assert iseg.matmul_i8(a, b).shape == (0, 4) and iseg.matmul_i8(b, a).shape == (4, 0)
    assert iseg.transpose_i8(a).shape == (16, 0)


@pytest.mark.parametrize("shape", [(1, 1), (1, 100), (100, 1), (64, 64), (65, 63), (130, 257), (1000, 48), (33, 4100)], ids=str)
def test_transpose(shape):
    from paper_2011_14504_amd import iseg
    M, C = shape
    x = codes(M, M, C)
    for gap in (0, 5, 16):
        t = iseg.transpose_i8(strided(x, C + gap, 99))
        assert torch.equal(t.cpu(), x.t())
    out = torch.full((C + 1, M + 20), 55, dtype=torch.int8, device=DEV)
    iseg.iseg_transpose_i8(x.to(DEV), M, C, C, out, M + 20)
    assert torch.equal(out[:C, :M].cpu(), x.t())
    assert bool((out[C:] == 55).all()) and bool((out[:, M:] == 55).all())


# (M, N, K, type)
LINEAR = [(1, 40, 30, "fp32"), (1, 4096, 4096, "bf16"), (1, 9000, 1024, "fp16"), (2, 100, 4100, "bf16"), (3, 33, 5000, "fp32"), (4, 100, 4096, "bf16"), (16, 64, 1000, "fp16"),
          (16, 8200, 512, "fp32"), (17, 64, 256, "bf16"), (1, 20, 3, "fp32"), (2, 20, 7, "bf16"), (1, 64, 16384, "bf16"), (1, 50, 16390, "fp32"),
          (1, 100, 8, "bf16"), (1, 8193, 8192, "bf16"), (1, 17, 8191, "fp32"), (1, 9, 2049, "fp16"), (5, 64, 128, "bf16"), (70, 100, 99, "fp16"), (128, 256, 192, "bf16"), (257, 129, 512, "fp32"),
          (50, 5, 100, "bf16"), (300, 3, 64, "fp32"), (129, 64, 300, "bf16"), (127, 65, 1000, "fp16"), (1100, 200, 130, "bf16")]


@pytest.mark.parametrize("case", LINEAR, ids=str)
def test_linear_forward_and_backward(case):
    from paper_2011_14504_amd import iseg
    M, N, K, t = case
    x, w = normal(1, M, K).to(DT[t]), codes(2, N, K).clamp_min(-127)
    ws, bias, dy = (normal(3, N).abs() * 1e-3 + 1e-4).float(), normal(4, N).float(), normal(5, M, N).to(DT[t])
    y, qa, sa = iseg.linear_i8_fwd(x.to(DEV), w.to(DEV), ws.to(DEV), bias.to(DEV))
    wqa, wsa = quantized(x.double(), 8, False)
    assert torch.equal(qa.cpu(), wqa) and torch.equal(sa.cpu(), wsa)
    p = _sums(wqa, w) * wsa.double()[:, None] * ws.double()
    want = p + bias.double()
    within(y, want, 4 * U * (p.abs() + want.abs()) + HALF[t] * want.abs() * (1 + 8 * U) + TINY[t] + 4 * U * HALF[t], "y")
    wt = iseg.transpose_i8(w.to(DEV))
    for kw in ({}, {"w_t": wt}):
        dx, dw, db = iseg.linear_i8_bwd(dy.to(DEV), qa, sa, w.to(DEV), ws.to(DEV), want_bias=True, **kw)
        q, s = quantized(dy.double() * ws.double(), 8, False)
        p = (q.double() @ w.double()) * s.double()[:, None]
        within(dx, p, 3 * U * p.abs() + HALF[t] * p.abs() * (1 + 4 * U) + TINY[t], "dx")
        q, s = quantized((dy.double() * wsa.double()[:, None]).t().contiguous(), 8, False)
        p = (q.double() @ wqa.double()) * s.double()[:, None]
        within(dw, p, 3 * U * p.abs() + HALF[t] * p.abs() * (1 + 4 * U) + TINY[t], "dw")
        within(db, dy.double().sum(0), (M + 4) * U * dy.double().abs().sum(0), "dbias")
    # the same bits as its two parts, whichever way it is run
    q2, s2 = iseg.quantize_rows(x.to(DEV))
    assert torch.equal(iseg.matmul_i8(q2, w.to(DEV), s2, ws.to(DEV), bias.to(DEV), DT[t]), y)
    wide = torch.zeros(K, N + 5, dtype=torch.int8, device=DEV)
    wide[:, 5:] = wt
    again = iseg.linear_i8_bwd(dy.to(DEV), strided(wqa, K + 3, 9), sa, strided(w, K + 1, 9), ws.to(DEV), w_t=wide[:, 5:], want_bias=True)
    for g, e in zip(again, (dx, dw, db)):
        assert torch.equal(g, e)
    q3, s3, db3 = iseg.quantize_cols(dy.to(DEV), mul=sa, want_sums=True)
    assert torch.equal(db3, db)
    no = iseg.linear_i8_bwd(dy.to(DEV), qa, sa, w.to(DEV), ws.to(DEV), want_weight=False, want_bias=True)
    assert no[1] is None and torch.equal(no[0], dx) and torch.equal(no[2], db)
    only = iseg.linear_i8_bwd(dy.to(DEV), qa, sa, w.to(DEV), ws.to(DEV), want_input=False)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)
